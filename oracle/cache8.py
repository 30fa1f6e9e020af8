"""CPU oracle, in 64 bits, of rotary positions and of the cache of pages that holds keys and values in 8 bits.

Written from the definitions that ``include/dkv.h`` states, without the library: values in place of codes, Python lists in place
of device memory, one row after the other.  Pinned by hand-worked cases, brute force over all codes and invariants
(``tests/test_oracle_cache8.py``)."""
import math

import numpy as np

LARGEST = {"e4m3": 448.0, "int8": 127.0}
SMALLEST_SCALE = 2.0 ** -126


def scale_for(values, kind):
    """The smallest power of two, not below 2^-126, whose largest code covers every finite value."""
    x = np.abs(np.asarray(values, dtype=np.float64))
    most = x[np.isfinite(x)].max(initial=0.0)
    s = SMALLEST_SCALE
    while s * LARGEST[kind] < most:
        s *= 2.0
    return s


def nearest(x, kind):
    """The code numbers next to x (already divided by the scale): ties to even, beyond the largest the largest, NaN 0."""
    x = np.nan_to_num(np.asarray(x, dtype=np.float64), nan=0.0, posinf=np.inf, neginf=-np.inf)
    x = np.clip(x, -LARGEST[kind], LARGEST[kind])
    if kind == "int8":
        return np.rint(x)
    exponent = np.maximum(np.frexp(x)[1] - 1, -6)            # of the power of two at or below |x|; e4m3's subnormals share 2^-6
    step = np.ldexp(1.0, exponent - 3)
    return np.rint(x / step) * step


def step_at(x, scale, kind):
    """Distance of neighbouring values around x."""
    if kind == "int8":
        return np.full_like(np.asarray(x, dtype=np.float64), scale)
    return np.ldexp(1.0, np.maximum(np.frexp(np.asarray(x, dtype=np.float64) / scale)[1] - 1, -6) - 3) * scale


class NoPages(Exception):
    pass


class Cache:
    """Sequences of pages.  A page is {"scale": [2][Hkv], "code": [2][Hkv][R][D]}; free pages are those that no sequence holds."""

    def __init__(self, n_pages, R, n_seqs, max_pages, Hkv, D, kind):
        self.n_pages, self.R, self.max_pages, self.Hkv, self.D, self.kind = n_pages, R, max_pages, Hkv, D, kind
        self.pages = [None] * n_pages
        self.table = [[] for _ in range(n_seqs)]
        self.len = [0] * n_seqs

    def refs(self):
        r = [0] * self.n_pages
        for t in self.table:
            for p in t:
                r[p] += 1
        return r

    def _new_page(self):
        return {"scale": np.full((2, self.Hkv), SMALLEST_SCALE), "code": np.zeros((2, self.Hkv, self.R, self.D))}

    def _take(self, needs):
        """Lowest free pages in order; None from the first that cannot be served on."""
        free = [p for p, n in enumerate(self.refs()) if n == 0]
        got, served = [], True
        for need in needs:
            served = served and need <= len(free)
            got.append(free[:need] if served else None)
            free = free[need:] if served else free
        return got

    def reserve(self, seqs, adds):
        """Which sequences could not be served: (no free pages, table full)."""
        refs, plans = self.refs(), []
        for s, add in zip(seqs, adds):
            pages = -(-(self.len[s] + add) // self.R)
            if add <= 0 or pages > self.max_pages:
                plans.append((0, False))
                continue
            copies = self.len[s] % self.R != 0 and refs[self.table[s][self.len[s] // self.R]] > 1
            plans.append((max(0, pages - len(self.table[s])) + copies, copies))
        full = [s for s, add in zip(seqs, adds) if -(-(self.len[s] + add) // self.R) > self.max_pages]
        none = []
        for s, got, (need, copies) in zip(seqs, self._take([n for n, _ in plans]), plans):
            if got is None:
                none += [s] if need else []
                continue
            for p in got:
                self.pages[p] = self._new_page()
            if copies:
                old = self.table[s][self.len[s] // self.R]
                self.pages[got[0]] = {w: x.copy() for w, x in self.pages[old].items()}
                self.table[s][self.len[s] // self.R] = got[0]
                got = got[1:]
            self.table[s] += got
        return none, full

    def append(self, s, k, v):
        """Rows k, v [Hkv, rows, D] behind those of sequence s; False (and nothing done) without room."""
        add, at = k.shape[1], self.len[s]
        if at + add > len(self.table[s]) * self.R:
            return False
        if add and at % self.R and self.refs()[self.table[s][at // self.R]] != 1:
            return False
        while add:
            page, r = self.pages[self.table[s][at // self.R]], at % self.R
            take = min(add, self.R - r)
            for w, x in enumerate((k, v)):
                for h in range(self.Hkv):
                    new, old = x[h, :take], page["scale"][w, h]
                    scale = scale_for(new, self.kind)
                    if r:
                        scale = max(scale, old)
                        page["code"][w, h, :r] = nearest(page["code"][w, h, :r] * old / scale, self.kind)
                    page["scale"][w, h] = scale
                    page["code"][w, h, r:r + take] = nearest(np.asarray(new, dtype=np.float64) / scale, self.kind)
            k, v = k[:, take:], v[:, take:]
            add, at = add - take, at + take
            self.len[s] = at
        return True

    def rows(self, s, which):
        """[Hkv, len, D]."""
        got = [self.pages[p]["code"][which] * self.pages[p]["scale"][which][:, None, None] for p in self.table[s]]
        return np.concatenate(got, axis=1)[:, :self.len[s]] if got else np.zeros((self.Hkv, 0, self.D))

    def scales(self, s, which):
        """[Hkv, len], a row's scale."""
        got = [np.repeat(self.pages[p]["scale"][which][:, None], self.R, axis=1) for p in self.table[s]]
        return np.concatenate(got, axis=1)[:, :self.len[s]] if got else np.zeros((self.Hkv, 0))

    def trim(self, s, rows):
        self.len[s] = max(0, min(self.len[s], rows))
        del self.table[s][-(-self.len[s] // self.R):]

    def fork(self, pairs):
        for _, t in pairs:
            self.table[t] = []
        for f, t in pairs:
            self.table[t], self.len[t] = self.table[f][:-(-self.len[f] // self.R)], self.len[f]

    def compact(self, seqs, idx):
        """Sequence seqs[i] keeps rows idx[i] [Hkv][count]; those that could not be served."""
        got, none = self._take([-(-len(x[0]) // self.R) for x in idx]), []
        keep = [[np.stack([self.rows(s, w)[h][list(x[h])] for h in range(self.Hkv)]) for w in range(2)] for s, x in zip(seqs, idx)]
        for s, x, pages, rows in zip(seqs, idx, got, keep):
            if pages is None:
                none += [s] if len(x[0]) else []
                if len(x[0]):
                    continue
                pages = []
            for j, p in enumerate(pages):
                self.pages[p] = self._new_page()
                part = slice(j * self.R, (j + 1) * self.R)
                for w in range(2):
                    for h in range(self.Hkv):
                        r = rows[w][h][part]
                        self.pages[p]["scale"][w, h] = scale_for(r, self.kind)
                        self.pages[p]["code"][w, h, :len(r)] = nearest(r / self.pages[p]["scale"][w, h], self.kind)
            self.table[s], self.len[s] = list(pages), len(x[0])
        return none

    def attend(self, s, q, causal):
        """q [Hq, nq, D]: (out [Hq, nq, D], lse [Hq, nq])."""
        return attention(q, self.rows(s, 0), self.rows(s, 1), causal)


def attention(q, k, v, causal):
    q, (Hq, nq, D) = np.asarray(q, dtype=np.float64), q.shape
    out, lse = np.zeros((Hq, nq, D)), np.full((Hq, nq), -np.inf)
    for hq in range(Hq):
        h = hq // (Hq // k.shape[0])
        for j in range(nq):
            seen = k.shape[1] - (nq - 1 - j if causal else 0)
            if seen <= 0:
                continue
            z = k[h, :seen] @ q[hq, j] / math.sqrt(D)
            e = np.exp(z - z.max())
            out[hq, j] = e @ v[h, :seen] / e.sum()
            lse[hq, j] = z.max() + math.log(e.sum())
    return out, lse


def frequencies(rot, theta, scaling="none", factor=1.0, low=1.0, high=4.0, trained=8192.0):
    """Radians a position of every pair, and the amplitude."""
    f = [theta ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [x / factor for x in f], 1.0
    if scaling == "base":
        return frequencies(rot, theta * factor ** (rot / (rot - 2)))
    if scaling == "wavelength":
        w = [min(1.0, max(0.0, (trained * x / (2 * math.pi) - low) / (high - low))) for x in f]
        return [x / factor * (1 - b) + x * b for x, b in zip(f, w)], 1.0
    if scaling == "ramp":
        x, y = (rot * math.log(trained / (2 * math.pi * b)) / (2 * math.log(theta)) for b in (high, low))
        x, y = max(0, math.floor(x)), min(rot - 1, math.ceil(y))
        r = [min(1.0, max(0.0, (i - x) / max(y - x, 0.001))) for i in range(rot // 2)]
        return [a / factor * b + a * (1 - b) for a, b in zip(f, r)], 0.1 * math.log(factor) + 1
    return f, 1.0


def rotate(x, pos, freq, amplitude, layout, transpose=False):
    """x [.., tokens, D], pos [.., tokens]."""
    x = np.asarray(x, dtype=np.float64)
    got, rot = x.copy(), 2 * len(freq)
    for i, f in enumerate(freq):
        a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
        t = np.asarray(pos, dtype=np.float64) * f * (-1 if transpose else 1)
        c, s = amplitude * np.cos(t), amplitude * np.sin(t)
        got[..., a] = x[..., a] * c - x[..., b] * s
        got[..., b] = x[..., a] * s + x[..., b] * c
    return got
