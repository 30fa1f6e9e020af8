// csrc/ring.cuh on the host, against barriers that are counted: every wait is for the phase that a copy on its way completes, and no
// copy is on its way into memory that has been given back.  Prints how many runs were looked at; ends with 1 at the first fault.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../paper_2412_14838_b200/csrc/ring.cuh"

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); std::exit(1); } } while (0)

struct Place { int phases = 0; bool expects = false, copy = false; int holds = -1; };       // phases: completed so far

// Heads of counts[h] chunks through one ring.  The wait for the `late`-th chunk of them all runs out (-1: none); that chunk's copy is only slow, or
// (`withheld`) never started.
template <int S>
void heads(const std::vector<int>& counts, int late, bool withheld) {
  dkv::RingPlaces<S> ring;
  Place places[S];
  int asked = 0, used = 0, failed = 0, drained = 0;
  for (int count : counts) {
    const bool was_broken = ring.broken;
    int begun = 0, next = 0, from = asked;
    ring.run(
        count,
        [&](int x, int at) {
          CHECK(!was_broken && x < count && x == asked - from && at >= 0 && at < S);
          Place& p = places[at];
          CHECK(!p.expects && !p.copy && p.holds < 0);       // nobody reads from the place, nothing is on its way there
          p.expects = true;
          p.holds = x;
          p.copy = !(withheld && asked == late);
          ++asked;
          return p.copy;
        },
        [&] { ++begun; },
        [&](int at, int parity) {
          Place& p = places[at];
          CHECK(!was_broken && !failed && p.expects);
          CHECK((p.phases & 1) == parity);                   // another parity: the test is true at once, whatever is on its way
          if (used == late) { ++failed; return false; }
          CHECK(p.copy);
          p.copy = p.expects = false;
          ++p.phases;
          return true;
        },
        [&](int x, int at) {
          CHECK(!failed && x == next && places[at].holds == x && !places[at].expects);
          places[at].holds = -1;
          ++next;
          ++used;
        },
        [&](int at, int parity) {
          Place& p = places[at];
          CHECK(failed && (p.phases & 1) == parity);
          CHECK(p.copy);                                     // never waits for what was not asked for
          p.copy = p.expects = false;
          ++p.phases;
          ++drained;
        });
    CHECK(begun == 1);
    for (const Place& p : places) CHECK(!p.copy);            // whatever was started has ended when run() returns
    CHECK(ring.broken == (failed > 0));
    CHECK(failed || next == count);
    CHECK(!was_broken || next == 0);
  }
  int all = 0;
  for (int count : counts) all += count;
  CHECK(failed == (late >= 0 && late < all) && (failed || used == all));
  CHECK(!failed || withheld || drained >= 1);
}

template <int S>
int all_of() {
  int runs = 0;
  for (int a = 0; a < 9; ++a)
    for (int b = 0; b < 9; ++b)
      for (int c = 0; c < 4; ++c)
        for (int late = -1; late < a + b + c; ++late)
          for (int withheld = 0; withheld < 2; ++withheld, ++runs) heads<S>({a, b, c, 3}, late, withheld);
  return runs;
}

int main() {
  const int runs = all_of<2>() + all_of<3>() + all_of<4>();
  std::printf("%d\n", runs);
  return 0;
}
