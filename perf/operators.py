"""The operators of generation after a compressed prompt, as cases with seeded inputs: their plain forms, and the calls of
the library that do the same.

A compressed prompt goes on living in a cache of pages that holds keys and values in 8 bits, with one power of two as the
scale of every (page, KV head, keys or values).  The uses are

``rotate``   rotary positions of a projection's queries and keys, token-major in and head-major out, or the gradient the
             other way (``dkv_rotate``)
``attend``   new queries attend to the cache (``dkv_cache8_attend``)
``step``     one layer's part of a decoding step with ``nq`` drafted tokens: room for them, their rows written (which may
             raise a page's scale), causal attention, and the drafted rows dropped again (``dkv_cache8_reserve``,
             ``dkv_cache8_append``, ``dkv_cache8_attend``, ``dkv_cache8_trim``)
``fill``     finished sequences make room for new ones: pages freed, compressed rows written, their keys rotated on the way
             where the case says so, and read back as 16-bit rows (``dkv_cache8_trim``, ``.._reserve``, ``.._append``,
             ``.._read``)
``evict``    sequences are forked and the forks cut to ``keep`` rows that each head chooses (``dkv_cache8_fork``,
             ``dkv_cache8_compact``, ``dkv_cache8_read``)

``prepare`` makes the inputs and the cache, ``run`` is one pass.
"""
import math

import torch

own = False

#: Largest magnitude of a code of either kind.
LARGEST = {"e4m3": 448.0, "int8": 127.0}
IO = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SCALINGS = ("none", "linear", "base", "wavelength", "ramp")


def _rotate(name, B, T, Hq, Hk, D, rot, layout, scaling, factor, io, backward=False, start=0):
    c = dict(use="rotate", B=B, T=T, Hq=Hq, Hk=Hk, D=D, rot=rot, layout=layout, scaling=scaling, factor=factor, io=io,
             backward=backward, start=start)
    return dict(c, name=name) if name else c


def _cache(name, use, n, Hkv, G, D, rows, ragged, kind, io, R, nq=1, causal=False, rot=0, layout="half", keep=0):
    c = dict(use=use, n=n, Hkv=Hkv, G=G, D=D, rows=rows, ragged=ragged, kind=kind, io=io, R=R, nq=nq, causal=causal, rot=rot,
             layout=layout, keep=keep)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoding step's queries and keys of sixteen sequences, 32/8 heads, as they leave the projection: latency
        _rotate("rotate_step", 16, 1, 32, 8, 128, 128, "half", "none", 1.0, "bf16", start=20000),
        # a whole 32K prompt of the same model, its context extended by wavelength
        _rotate("rotate_prompt", 1, 32768, 32, 8, 128, 128, "half", "wavelength", 8.0, "bf16"),
        # training: the gradient of three prompts of 5003 tokens, 18/6 heads of 64, neighbouring pairs, half of each head
        _rotate("rotate_grad", 3, 5003, 18, 6, 64, 32, "pairs", "ramp", 4.0, "f32", True),
        # the shortest call: one sequence, one layer, 160 kept rows and the window of a prompt compressed hard
        _cache("attend_one", "attend", 1, 8, 4, 128, 160, False, "e4m3", "bf16", 32),
        # drafted tokens verified against a whole 32K cache of one sequence: 16 query rows a KV head
        _cache("attend_32k_draft", "attend", 1, 8, 4, 128, 32768, False, "int8", "bf16", 64, nq=4, causal=True),
        # 33 sequences of every length up to 5003 rows, one of them empty, 18/6 heads of 64
        _cache("attend_ragged", "attend", 33, 6, 3, 64, 5003, True, "int8", "f16", 32),
        # a serving batch over long caches: 64 sequences of 8K rows, the most bytes
        _cache("attend_batch", "attend", 64, 8, 4, 128, 8192, False, "e4m3", "bf16", 32),
        # one layer's part of a step of 32 sequences with caches of the large budget, two drafted tokens each
        _cache("step_draft", "step", 32, 8, 4, 128, 1090, True, "int8", "bf16", 32, nq=2, causal=True),
        # the compressed cache of a 32-layer model moves into pages: 544 rows a head and layer
        _cache("fill_layers", "fill", 32, 8, 4, 128, 544, False, "e4m3", "bf16", 32),
        # long prompts move in uncompressed, keys rotated on the way: odd lengths, half of each head rotated
        _cache("fill_rotated", "fill", 5, 6, 3, 64, 16001, True, "int8", "f16", 64, rot=32, layout="pairs"),
        # four beams' forks cut to 128 rows of some 700: latency
        _cache("evict_beams", "evict", 4, 8, 4, 128, 700, False, "e4m3", "bf16", 32, keep=128),
        # 28 layers with 4 KV heads cut from 8K rows to 1000
        _cache("evict_layers", "evict", 28, 4, 7, 128, 8192, True, "int8", "bf16", 64, keep=1000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    use = rng.choice(["rotate", "attend", "attend", "attend", "step", "fill", "evict"])
    if use == "rotate":
        while True:
            B, T = _log_int(rng, 1, 32), _log_int(rng, 1, 32768)
            Hk, G, D = rng.choice([1, 2, 4, 6, 8]), rng.choice([1, 2, 3, 4, 7, 8]), rng.choice([64, 80, 96, 128, 128, 256])
            if B * T * (G + 1) * Hk * D <= 32768 * 40 * 128:
                break
        return _rotate("", B, T, G * Hk, Hk, D, rng.choice([D, D, D // 2, 10]), rng.choice(["half", "pairs"]),
                       rng.choice(SCALINGS), rng.choice([2.0, 4.0, 8.0, 10.5]), rng.choice(["bf16", "bf16", "f16", "f32"]),
                       rng.choice([False, False, True]), rng.choice([0, 0, 1000, 100000, 1000000]))
    while True:
        n, Hkv, D, rows = _log_int(rng, 1, 96), rng.choice([1, 2, 4, 6, 8]), rng.choice([64, 128, 128]), _log_int(rng, 1, 40000)
        if n * Hkv * D * rows <= {"attend": 64 * 8 * 128 * 8192, "step": 32 * 8 * 128 * 8192}.get(use, 28 * 4 * 128 * 8192):
            break
    nq = rng.choice([1, 1, 1, 2, 3, 5, 8]) if use in ("attend", "step") else 1
    rot = rng.choice([0, D, D // 2]) if use == "fill" else 0
    return _cache("", use, n, Hkv, rng.choice([1, 2, 3, 4, 4, 7, 8]), D, rows, rng.choice([False, True, True]),
                  rng.choice(["e4m3", "int8"]), rng.choice(["bf16", "bf16", "f16"]), rng.choice([32, 32, 64, 128]), nq,
                  use == "step" or rng.choice([False, True]), rot, rng.choice(["half", "pairs"]),
                  max(1, _log_int(rng, 1, rows)) if use == "evict" else 0)


def _lengths(c):
    """Rows that each sequence holds: all of them, or every length (an empty sequence last where there are three)."""
    if not c["ragged"]:
        return [c["rows"]] * c["n"]
    some = [c["rows"]] + [1 + int((c["rows"] - 1) * (i * 0.6180339887498949 % 1)) for i in range(1, c["n"])]
    return some[:-1] + [0] if c["n"] > 2 else some


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _rows(g, c, n, rows):
    """Keys with four outlier channels a head and values of a size of their own a head, [n, Hkv, rows, D]."""
    shape, t = (n, c["Hkv"], rows, c["D"]), IO[c["io"]]
    k, v = (torch.randn(shape, generator=g, device="cuda", dtype=t) for _ in range(2))
    channels = torch.rand((c["Hkv"], c["D"]), generator=g, device="cuda").topk(4, dim=1).indices
    k *= torch.ones((c["Hkv"], c["D"]), device="cuda").scatter_(1, channels, 6.0).to(t)[None, :, None, :]
    v *= (0.25 + torch.rand((c["Hkv"], 1, 1), generator=g, device="cuda")).to(t)
    return k, v


def _inputs(c, seed):
    """The tensors that a case starts from, the same for every form of it."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    if c["use"] == "rotate":
        width = (c["Hq"] + 2 * c["Hk"]) * c["D"]
        x = torch.randn((c["B"], c["T"], width), generator=g, device="cuda", dtype=torch.float32).to(IO[c["io"]])
        first = c["start"] + torch.randint(0, 1000, (c["B"], 1), generator=g, device="cuda", dtype=torch.int32)
        return {"x": x, "pos": (first + torch.arange(c["T"], device="cuda", dtype=torch.int32)).to(torch.int32).contiguous()}
    n, D, lens = c["n"], c["D"], torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
    k, v = _rows(g, c, n, c["rows"])
    got = {"k": k, "v": v, "lens": lens}
    if c["use"] in ("attend", "step"):
        mean = torch.randn((n, c["Hkv"] * c["G"], 1, D), generator=g, device="cuda")
        q = torch.randn((n, c["Hkv"] * c["G"], c["nq"], D), generator=g, device="cuda") + 0.5 * mean
        got["q"] = q.to(IO[c["io"]])
    if c["use"] == "step":                       # now and then a drafted token raises its page's scale
        got["k_new"], got["v_new"] = (2.0 * x for x in _rows(g, c, n, c["nq"]))
    if c["use"] == "fill" and c["rot"]:
        got["pos0"] = torch.randint(0, 100000, (n,), generator=g, device="cuda", dtype=torch.int32)
    if c["use"] == "evict":                      # every head keeps rows of its own, best first
        w = torch.rand((n, c["Hkv"], c["rows"]), generator=g, device="cuda")
        w.masked_fill_(torch.arange(c["rows"], device="cuda") >= lens[:, None, None], -1.0)
        got["idx"] = w.topk(min(c["keep"], c["rows"]), dim=2).indices.to(torch.int32).contiguous()
        got["n_keep"] = lens.clamp(max=c["keep"])
    return got


def _pages(c, rows):
    return -(-rows // c["R"])


# ---- rotary positions ---------------------------------------------------------------------------------------------------
#: Base, bands of the scalings and the context length that they extend.
THETA, LOW, HIGH, FAST, TRAINED = 500000.0, 1.0, 4.0, 32.0, 8192.0


def _frequencies(rot, scaling, factor):
    """Radians a position, one for each pair, in 64 bits; and what multiplies cosine and sine."""
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    if scaling == "base":
        return (THETA * factor ** (rot / (rot - 2))) ** (-2.0 * i / rot), 1.0
    f = THETA ** (-2.0 * i / rot)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "wavelength":
        waves = TRAINED * f / (2.0 * math.pi)
        blend = ((waves - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
        return f / factor * (1.0 - blend) + f * blend, 1.0
    if scaling == "ramp":
        at = [rot * math.log(TRAINED / (2.0 * math.pi * b)) / (2.0 * math.log(THETA)) for b in (FAST, LOW)]
        lo, hi = max(0, math.floor(at[0])), min(rot - 1, math.ceil(at[1]))
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f / factor * ramp + f * (1.0 - ramp), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _plain_rotate(x, pos, freq, amplitude, rot, layout, backward=False):
    """x [.., tokens, D] turned by pos [.., tokens] (broadcast over heads); angles in 64 bits, the rest in 32."""
    angle = pos.double().unsqueeze(-1) * freq
    c, s = (amplitude * torch.cos(angle)).float(), (amplitude * torch.sin(angle)).float()
    s = -s if backward else s
    x = x.float()
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    a, b = a * c - b * s, a * s + b * c
    turned = torch.cat([a, b], -1) if layout == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _views(s, c):
    """Queries and keys of the projection as [B, heads, tokens, D]."""
    heads = s["x"].view(c["B"], c["T"], -1, c["D"]).transpose(1, 2)
    return heads[:, :c["Hq"]], heads[:, c["Hq"]:c["Hq"] + c["Hk"]]


# ---- the cache, plain form ------------------------------------------------------------------------------------------------
def _scale_for(most, kind):
    """The smallest power of two, not below 2^-126, that is at least most / LARGEST[kind]."""
    fraction, exponent = torch.frexp(most)
    top, at = math.frexp(LARGEST[kind])
    e = (exponent - at + (fraction > top)).clamp(min=-126)
    return torch.where(most > 0, torch.ldexp(torch.ones_like(most), e), torch.full_like(most, 2.0 ** -126))


def _code(x, kind):
    """x, already divided by its scale, as codes: clamped, rounded to the nearest, ties to even; NaN is 0."""
    x = torch.nan_to_num(x, nan=0.0, posinf=LARGEST[kind], neginf=-LARGEST[kind]).clamp(-LARGEST[kind], LARGEST[kind])
    return x.to(torch.float8_e4m3fn) if kind == "e4m3" else torch.round(x).to(torch.int8)


class _Plain:
    """Pages of codes [pages, Hkv, R, D], scales [pages, Hkv], page table, lengths and holders, in tensors."""

    def __init__(self, c, n_seqs, n_pages, max_pages):
        self.kind, self.R, self.n_pages, dev = c["kind"], c["R"], n_pages, "cuda"
        shape, t = (n_pages, c["Hkv"], c["R"], c["D"]), torch.float8_e4m3fn if c["kind"] == "e4m3" else torch.int8
        self.code = [torch.zeros(shape, dtype=t, device=dev) for _ in range(2)]
        self.scale = [torch.full(shape[:2], 2.0 ** -126, device=dev) for _ in range(2)]
        self.table = torch.zeros((n_seqs, max_pages), dtype=torch.int64, device=dev)
        self.len, self.held = (torch.zeros(n_seqs, dtype=torch.int32, device=dev) for _ in range(2))
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device=dev)
        self.place = torch.arange(max_pages, device=dev)

    def _let_go(self, rows):
        """Pages of every sequence from those that hold `rows` rows on are given back."""
        first = (rows + self.R - 1) // self.R
        gone = (self.place >= first[:, None]) & (self.place < self.held[:, None])
        self.refs -= torch.zeros_like(self.refs).index_add_(0, self.table.flatten(), gone.flatten().to(torch.int32))
        self.held = torch.minimum(self.held, first)

    def trim(self, rows):
        self._let_go(rows)
        self.len = rows

    def reserve(self, add):
        """The lowest free pages, in the order of the sequences."""
        need = ((self.len + add + self.R - 1) // self.R - self.held).clamp(min=0)
        free = torch.sort(self.refs > 0, stable=True).indices
        new = (self.place >= self.held[:, None]) & (self.place < (self.held + need)[:, None])
        rank = (torch.cumsum(need, 0) - need - self.held)[:, None] + self.place
        page = free[rank.clamp(0, self.n_pages - 1)]
        self.table = torch.where(new, page, self.table)
        self.refs = self.refs.index_add(0, page.flatten(), new.flatten().to(torch.int32))
        self.held = self.held + need

    def gather(self, which, pages, first=None):
        """Rows [sequences, Hkv, pages * R, D] of `pages` pages (from the `first` of each), in 32 bits."""
        at = self.place[:pages] if first is None else (first[:, None] + self.place[:pages]).clamp(max=len(self.place) - 1)
        ids = self.table.gather(1, at.expand(len(self.table), pages).to(torch.int64))
        x = self.code[which][ids].float() * self.scale[which][ids][..., None, None]
        return x.transpose(1, 2).flatten(2, 3), ids

    def append(self, k, v, rows):
        """The first rows[i] of k[i], v[i] go behind the rows of sequence i; a page's scale may grow, its rows follow."""
        R, n, most = self.R, len(self.len), k.shape[2]
        pages = min(len(self.place), (most + R - 1) // R + 1)
        first = (self.len // R).clamp(max=max(0, len(self.place) - pages))
        spot = (first * R)[:, None] + torch.arange(pages * R, device="cuda")
        old = (spot < self.len[:, None]).view(n, pages, R)
        fresh = ((spot >= self.len[:, None]) & (spot < (self.len + rows)[:, None])).view(n, pages, R)
        touched = fresh.any(2)
        source = (spot - self.len[:, None]).clamp(0, most - 1)[:, None, :, None]
        for which, x in enumerate((k, v)):
            held, ids = self.gather(which, pages, first)
            held = held.view(n, -1, pages, R, x.shape[-1])
            x = x.float().gather(2, source.expand(n, x.shape[1], pages * R, x.shape[3])).view_as(held)
            size = torch.where(x.isfinite(), x, 0.0).abs().mul_(fresh[:, None, :, :, None]).amax((3, 4)).transpose(1, 2)
            before = torch.where(old.any(2)[..., None], self.scale[which][ids], torch.zeros_like(size))
            scale = torch.maximum(_scale_for(size, self.kind), before)
            x = torch.where(fresh[:, None, :, :, None], x, torch.where(old[:, None, :, :, None], held, 0.0))
            code = _code(x / scale.transpose(1, 2)[..., None, None], self.kind).transpose(1, 2)
            there = ids[touched]
            self.scale[which][there] = scale[touched]
            self.code[which].view(torch.uint8)[there] = code.contiguous().view(torch.uint8)[touched]
        self.len = self.len + rows

    def read(self, pages, out, t):
        """The rows as 16-bit numbers into out; rows past a sequence's length stay as they are."""
        keep = torch.arange(out[0].shape[2], device="cuda") >= self.len[:, None]
        for which, o in enumerate(out):
            x = self.gather(which, pages)[0][:, :, :o.shape[2]]
            x = x.clamp(torch.finfo(t).min, torch.finfo(t).max).to(t)
            o.copy_(torch.where(keep[:, None, :, None], o, x))


def _plain_attend(cache, q, pages, causal):
    """Softmax attention of q [n, Hq, nq, D] over each sequence's rows, and the logarithm of its denominators."""
    n, Hq, nq, D = q.shape
    k, v = (cache.gather(w, pages)[0] for w in range(2))
    Hkv, rows = k.shape[1], k.shape[2]
    s = torch.matmul(q.float().reshape(n, Hkv, -1, D), k.transpose(-1, -2)) / math.sqrt(D)
    behind = nq - 1 - torch.arange(nq, device="cuda") if causal else torch.zeros(nq, dtype=torch.int64, device="cuda")
    seen = torch.arange(rows, device="cuda") < (cache.len[:, None] - behind)[..., None]
    s = s.view(n, Hkv, -1, nq, rows).masked_fill(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(n, Hkv, -1, rows), v).view(n, Hkv, -1, nq, D) / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total)).squeeze(-1)
    return out.reshape(n, Hq, nq, D), lse.reshape(n, Hq, nq)


# ---- the cache of the library ---------------------------------------------------------------------------------------------
class _Shown:
    """Integers inside the library's cache, for torch."""

    def __init__(self, owner, address, shape):
        self.owner = owner
        self.__cuda_array_interface__ = {"data": (address, False), "shape": shape, "typestr": "<i4", "version": 3}


class _Own:
    def __init__(self, c, n_seqs, n_pages, max_pages):
        from paper_2412_14838_b200 import binding as B
        self.B = B
        self.handle = B.dkv_cache8_create(B.make_cache8_config(
            n_pages=n_pages, page_rows=c["R"], n_seqs=n_seqs, max_pages=max_pages, n_q_heads=c["Hkv"] * c["G"],
            n_kv_heads=c["Hkv"], head_dim=c["D"], kind=B.DKV_E4M3 if c["kind"] == "e4m3" else B.DKV_INT8,
            io=B.DKV_BF16 if c["io"] == "bf16" else B.DKV_F16))
        at = B.dkv_cache8_views(self.handle)
        self.len = torch.as_tensor(_Shown(self, at["len"], (n_seqs,)), device="cuda")
        self.refs = torch.as_tensor(_Shown(self, at["refs"], (n_pages,)), device="cuda")

    def __del__(self):
        if getattr(self, "handle", None):
            self.B.dkv_cache8_destroy(self.handle)


def _rotary(c, scaling="none", factor=1.0):
    from paper_2412_14838_b200 import binding as B
    return B.dkv_rotary_init(
        head_dim=c["D"], rot_dim=c["rot"], layout=B.DKV_ROTARY_HALF if c["layout"] == "half" else B.DKV_ROTARY_PAIRS, theta=THETA,
        scaling=SCALINGS.index(scaling), factor=factor, low=LOW, high=FAST if scaling == "ramp" else HIGH, trained_len=TRAINED)


# ---- prepare and run ------------------------------------------------------------------------------------------------------
class State(dict):
    pass


def prepare(case, seed):
    c, s = case, State(_inputs(case, seed))
    s["case"] = c
    if c["use"] == "rotate":
        if c["backward"]:                        # head-major gradients in, the projection's layout out
            s["g"] = [t.contiguous() for t in _views(s, c)]
            s["grad"] = torch.zeros_like(s["x"])
            s["out"] = _views({"x": s["grad"]}, c)
        else:
            s["out"] = tuple(torch.empty_like(t, memory_format=torch.contiguous_format) for t in _views(s, c))
        if own:
            s["rotary"] = _rotary(c, c["scaling"], c["factor"])
        else:
            s["rotary"] = _frequencies(c["rot"], c["scaling"], c["factor"])
        return s
    n, room = c["n"], max(1, _pages(c, c["rows"] + (c["nq"] if c["use"] == "step" else 0)))
    forks = n if c["use"] == "evict" else 0
    pages = n * room + forks * max(1, _pages(c, c["keep"]))
    cache = s["cache"] = (_Own if own else _Plain)(c, n + forks, pages, room)
    if c["use"] == "fill":
        s["out"] = [torch.zeros_like(s[w]) for w in "kv"]
        if c["rot"]:
            s["rotary"] = _rotary(c) if own else _frequencies(c["rot"], "none", 1.0)
        return s
    lens = torch.cat([s["lens"], torch.zeros(forks, dtype=torch.int32, device="cuda")])
    if own:
        B = cache.B
        B.dkv_cache8_reserve(cache.handle, 0, n, 1, s["lens"], 0)
        B.dkv_cache8_append(cache.handle, 0, n, 1, s["k"], s["v"], s["lens"])
    else:
        cache.reserve(lens)
        fill = [torch.nn.functional.pad(s[w], (0, 0, 0, 0, 0, 0, 0, forks)) if forks else s[w] for w in "kv"]
        cache.append(*fill, lens)
    del s["k"], s["v"]
    if "q" in s:
        s["out"] = torch.zeros(s["q"].shape, dtype=torch.float32, device="cuda")
        s["lse"] = torch.zeros(s["q"].shape[:3], dtype=torch.float32, device="cuda")
    if forks:
        s["out"] = [torch.zeros((n, c["Hkv"], min(c["keep"], c["rows"]), c["D"]), dtype=IO[c["io"]], device="cuda") for _ in "kv"]
    return s


def _run_rotate(s, c):
    x = s["g"] if c["backward"] else _views(s, c)
    if own:
        from paper_2412_14838_b200 import binding as B
        B.dkv_rotate(s["rotary"], s["pos"], x[0], s["out"][0], x[1], s["out"][1], transpose=c["backward"])
    else:
        freq, amplitude = s["rotary"]
        s["out"][0].copy_(_plain_rotate(x[0], s["pos"][:, None], freq, amplitude, c["rot"], c["layout"], c["backward"]))
        s["out"][1].copy_(_plain_rotate(x[1], s["pos"][:, None], freq, amplitude, c["rot"], c["layout"], c["backward"]))
    return {"grad": s["grad"]} if c["backward"] else {"q": s["out"][0], "k": s["out"][1]}


def _run_attend(s, c):
    cache = s["cache"]
    if own:
        cache.B.dkv_cache8_attend(cache.handle, 0, c["n"], 1, s["q"], s["out"], s["lse"], causal=c["causal"])
        return {"out": s["out"], "lse": s["lse"]}
    out, lse = _plain_attend(cache, s["q"], max(1, _pages(c, c["rows"])), c["causal"])
    return {"out": out, "lse": lse}


def _run_step(s, c):
    cache, n, nq = s["cache"], c["n"], c["nq"]
    if own:
        B, h = cache.B, cache.handle
        B.dkv_cache8_reserve(h, 0, n, 1, None, nq)
        B.dkv_cache8_append(h, 0, n, 1, s["k_new"], s["v_new"])
        B.dkv_cache8_attend(h, 0, n, 1, s["q"], s["out"], s["lse"], causal=True)
        B.dkv_cache8_trim(h, 0, n, 1, None, nq)
        return {"out": s["out"], "lse": s["lse"], "len": cache.len, "refs": cache.refs}
    cache.reserve(nq)
    cache.append(s["k_new"], s["v_new"], torch.full_like(cache.len, nq))
    out, lse = _plain_attend(cache, s["q"], _pages(c, c["rows"] + nq), True)
    cache.trim(cache.len - nq)
    return {"out": out, "lse": lse, "len": cache.len, "refs": cache.refs}


def _run_fill(s, c):
    cache, n = s["cache"], c["n"]
    if own:
        B, h = cache.B, cache.handle
        B.dkv_cache8_trim(h, 0, n, 1, None, 2**31 - 1)
        B.dkv_cache8_reserve(h, 0, n, 1, s["lens"], 0)
        B.dkv_cache8_append(h, 0, n, 1, s["k"], s["v"], s["lens"], s.get("rotary"), s.get("pos0"))
        B.dkv_cache8_read(h, 0, n, 1, *s["out"])
    else:
        cache.trim(torch.zeros_like(cache.len))
        cache.reserve(s["lens"])
        k = s["k"]
        if c["rot"]:
            pos = s["pos0"][:, None] + torch.arange(c["rows"], device="cuda")
            k = _plain_rotate(k, pos[:, None], *s["rotary"], c["rot"], c["layout"])
        cache.append(k, s["v"], s["lens"])
        cache.read(max(1, _pages(c, c["rows"])), s["out"], IO[c["io"]])
    return {"k": s["out"][0], "v": s["out"][1], "len": cache.len, "refs": cache.refs}


def _run_evict(s, c):
    cache, n = s["cache"], c["n"]
    if own:
        B, h = cache.B, cache.handle
        B.dkv_cache8_fork(h, 0, n, n, 1)
        B.dkv_cache8_compact(h, n, n, 1, s["idx"], s["n_keep"])
        B.dkv_cache8_read(h, n, n, 1, *s["out"])
        return {"k": s["out"][0], "v": s["out"][1], "len": cache.len, "refs": cache.refs}
    source, made = slice(0, n), slice(n, 2 * n)
    cache.trim(torch.cat([cache.len[source], torch.zeros_like(cache.len[made])]))     # what the forks held before
    pages = max(1, _pages(c, c["rows"]))
    rows = [cache.gather(w, pages)[0][source] for w in range(2)]
    take = s["idx"].to(torch.int64)[..., None].expand(*s["idx"].shape, c["D"])
    rows = [torch.nn.functional.pad(x.gather(2, take), (0, 0, 0, 0, 0, 0, n, 0)) for x in rows]
    add = torch.cat([torch.zeros_like(s["n_keep"]), s["n_keep"]])
    cache.reserve(add)
    cache.append(*rows, add)
    both = [torch.cat([torch.empty_like(o), o]) for o in s["out"]]
    cache.read(max(1, _pages(c, c["keep"])) if c["keep"] <= c["rows"] else pages, both, IO[c["io"]])
    return {"k": both[0][made], "v": both[1][made], "len": cache.len, "refs": cache.refs}


def run(state):
    c = state["case"]
    return {"rotate": _run_rotate, "attend": _run_attend, "step": _run_step, "fill": _run_fill, "evict": _run_evict}[c["use"]](state, c)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------
def _near(x, kind):
    """The code next to x, as a number."""
    most = 448.0 if kind == "e4m3" else 127.0
    x = x.clamp(-most, most)
    if kind == "int8":
        return torch.round(x)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(x / step) * step


def _block_scale(x, kind):
    """Power of two of blocks x [.., rows, D]."""
    most = x.abs().amax((-1, -2), keepdim=True)
    e = torch.ceil(torch.log2(most / (448.0 if kind == "e4m3" else 127.0)) - 1e-12)      # (log2 of a power of two may be off its integer)
    return torch.exp2(torch.where(most > 0, e, torch.full_like(e, -126.0)).clamp(min=-126.0))


def _stored(x, c):
    """Rows x [Hkv, rows, D] in 64 bits as the cache holds them, block by block from its first row."""
    got = []
    for a in range(0, x.shape[1], c["R"]):
        block = x[:, a:a + c["R"]]
        scale = _block_scale(block, c["kind"])
        got.append(_near(block / scale, c["kind"]) * scale)
    return torch.cat(got, 1) if got else x


def _stored_and(x, new, c):
    """The same, and then rows `new` behind them: the last block's scale grows where they need it."""
    held, at = _stored(x, c), x.shape[1] // c["R"] * c["R"]
    tail, room = held[:, at:], c["R"] - (x.shape[1] - at)
    scale = _block_scale(new[:, :room], c["kind"])
    if tail.shape[1]:
        scale = torch.maximum(scale, _block_scale(x[:, at:], c["kind"]))
        tail = _near(tail / scale, c["kind"]) * scale
    first = _near(new[:, :room] / scale, c["kind"]) * scale
    return torch.cat([held[:, :at], tail, first, _stored(new[:, room:], c)], 1)


def _exact_attend(c, q, k, v):
    """One sequence: q [Hq, nq, D] over k, v [Hkv, rows, D]."""
    Hq, nq, D = q.shape
    out, lse = torch.zeros((Hq, nq, D), dtype=torch.float64, device="cuda"), torch.full((Hq, nq), -math.inf, dtype=torch.float64, device="cuda")
    for i in range(nq):
        rows = k.shape[1] - (nq - 1 - i if c["causal"] else 0)
        if rows > 0:
            z = torch.einsum("hgd,hrd->hgr", q[:, i].view(-1, c["G"], D), k[:, :rows]) * D ** -0.5
            lse[:, i] = torch.logsumexp(z, -1).flatten()
            out[:, i] = torch.einsum("hgr,hrd->hgd", torch.softmax(z, -1), v[:, :rows]).reshape(Hq, D)
    return out, lse


def _exact_frequency(i, rot, scaling, factor):
    """Radians a position of pair i."""
    wave = 2.0 * math.pi * THETA ** (2.0 * i / rot)
    if scaling == "base":
        return math.exp(-2.0 * i / rot * (math.log(THETA) + rot / (rot - 2) * math.log(factor)))
    if scaling == "linear":
        wave *= factor
    elif scaling == "wavelength" and wave > TRAINED / LOW:
        wave *= factor
    elif scaling == "wavelength" and wave >= TRAINED / HIGH:
        kept = (TRAINED / wave - LOW) / (HIGH - LOW)
        wave = 1.0 / (kept / wave + (1.0 - kept) / (factor * wave))
    elif scaling == "ramp":                      # by the place of the pairs that turn FAST and LOW times in TRAINED positions
        lo = max(math.floor(rot / 2 * math.log(TRAINED / (FAST * 2.0 * math.pi), THETA)), 0)
        hi = min(math.ceil(rot / 2 * math.log(TRAINED / (LOW * 2.0 * math.pi), THETA)), rot - 1)
        slow = min(1.0, max(0.0, (i - lo) / (hi - lo if hi > lo else 0.001)))
        wave = 1.0 / (slow / (factor * wave) + (1.0 - slow) / wave)
    return 2.0 * math.pi / wave


def _exact_frequencies(rot, scaling, factor):
    f = [_exact_frequency(i, rot, scaling, factor) for i in range(rot // 2)]
    return torch.tensor(f, dtype=torch.float64, device="cuda"), 1.0 + math.log(factor) / 10.0 if scaling == "ramp" else 1.0


def _exact_turn(x, angle, amplitude, c):
    """x [.., tokens, D] in 64 bits, its pairs as complex numbers times amplitude * exp(i angle)."""
    rot, x = c["rot"], x.clone()
    pair = (slice(0, rot // 2), slice(rot // 2, rot)) if c["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    z = torch.complex(x[..., pair[0]].contiguous(), x[..., pair[1]].contiguous()) * torch.polar(torch.full_like(angle, amplitude), angle)
    x[..., pair[0]], x[..., pair[1]] = z.real, z.imag
    return x


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["use"] == "rotate":
        freq, amplitude = _exact_frequencies(c["rot"], c["scaling"], c["factor"])
        angle = s["pos"].double()[..., None] * freq * (-1.0 if c["backward"] else 1.0)
        got = [_exact_turn(t.double(), angle[:, None], amplitude, c) for t in _views(s, c)]
        if not c["backward"]:
            return {"q": got[0], "k": got[1]}
        grad = torch.zeros_like(s["x"], dtype=torch.float64)
        for to, g in zip(_views({"x": grad}, c), got):
            to.copy_(g)
        return {"grad": grad}
    lens = _lengths(c)
    if c["use"] in ("attend", "step"):
        out, lse = [], []
        for i, rows in enumerate(lens):
            k, v = (s[w][i, :, :rows].double() for w in "kv")
            if c["use"] == "step":
                k, v = (_stored_and(x, s[w][i].double(), c) for x, w in ((k, "k_new"), (v, "v_new")))
            else:
                k, v = _stored(k, c), _stored(v, c)
            o, z = _exact_attend(c, s["q"][i].double(), k, v)
            out.append(o)
            lse.append(z)
        got = {"out": torch.stack(out), "lse": torch.stack(lse)}
        return dict(got, len=None, refs=None) if c["use"] == "step" else got
    rows = c["rows"] if c["use"] == "fill" else min(c["keep"], c["rows"])
    got = {w: torch.zeros((c["n"], c["Hkv"], rows, c["D"]), dtype=torch.float64, device="cuda") for w in "kv"}
    for i, n in enumerate(lens):
        for w in "kv":
            x = s[w][i, :, :n].double()
            if c["use"] == "evict":
                keep = min(n, c["keep"])
                take = s["idx"][i, :, :keep].long()[..., None].expand(-1, -1, c["D"])
                x, n_out = _stored(x, c).gather(1, take), keep
            else:
                n_out = n
                if w == "k" and c["rot"]:
                    pos = s["pos0"][i].double() + torch.arange(n, device="cuda", dtype=torch.float64)
                    x = _exact_turn(x, pos[:, None] * _exact_frequencies(c["rot"], "none", 1.0)[0], 1.0, c)
            got[w][i, :, :n_out] = _stored(x, c)
    return dict(got, len=None, refs=None)


def work(case):
    """Bytes: every input read once and every output written once (8 bits a number in the cache, 16 outside, 4 bytes a
    scale), operations: six a rotated pair, four a query, row and dim of attention."""
    c = case
    if c["use"] == "rotate":
        tokens, size = c["B"] * c["T"], torch.finfo(IO[c["io"]]).bits // 8
        heads = c["Hq"] + c["Hk"]
        return {"bytes": tokens * (2 * heads * c["D"] * size + 4), "flops": 3 * tokens * heads * c["rot"]}
    held, width = sum(_lengths(c)) * c["Hkv"], c["D"] * 2
    if c["use"] in ("attend", "step"):
        step = c["use"] == "step"
        rows = held + (c["n"] * c["Hkv"] * c["nq"] if step else 0)
        queries = c["n"] * c["Hkv"] * c["G"] * c["nq"]
        new = c["n"] * c["nq"] * c["Hkv"] * width * 3 if step else 0
        return {"bytes": rows * width + queries * (c["D"] * 6 + 4) + new, "flops": 4 * rows * c["G"] * c["nq"] * c["D"]}
    if c["use"] == "fill":
        return {"bytes": held * width * (2 + 1 + 1 + 2), "flops": held * c["D"] * 8}
    kept = sum(min(n, c["keep"]) for n in _lengths(c)) * c["Hkv"]
    return {"bytes": kept * width * (1 + 1 + 1 + 2) + kept * 4, "flops": kept * c["D"] * 8}
