// Which place of a ring a chunk lies in, which phase of the place's barrier its copy completes, and which copies are on their way.
// No GPU code: tests compile it for the host, with barriers of their own.
#pragma once

#ifdef __CUDACC__
#define DKV_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define DKV_HOST_DEVICE inline
#endif

namespace dkv {

// A ring of kStages places, each with a barrier whose phases complete one copy after the other.
template <int kStages>
struct RingPlaces {
  int stage = 0, phase = 0;                            // of the next chunk that is waited for
  unsigned int asked = 0;                              // bit per place: a copy into it is on its way
  bool broken = false;                                 // a wait ran out: nothing more is asked for or waited for

  DKV_HOST_DEVICE int place(int ahead) const { return (stage + ahead) % kStages; }       // of the chunk `ahead` after the next one
  DKV_HOST_DEVICE int parity(int at) const { return at < stage ? phase ^ 1 : phase; }    // of the copy on its way into place `at`
  DKV_HOST_DEVICE void take() {                        // the next chunk is there
    asked &= ~(1u << stage);
    if (++stage == kStages) { stage = 0; phase ^= 1; }
  }

  // Runs chunks 0 .. count - 1 through the ring, kStages - 1 of them ahead of the one that is worked on.  ask(x, place): asks for chunk x;
  // whether a copy was started.  wait(place, parity): false where the wait ran out.  use(x, place).  begin(): once the first chunks are asked
  // for.  Where a wait runs out the copies that were started are waited for right there, by drain(place, parity), which has a limit of its
  // own: the memory is the caller's again.  The counters stay where they were then: what they say of the phases holds for what was on its way.
  template <typename Ask, typename Begin, typename Wait, typename Use, typename Drain>
  DKV_HOST_DEVICE void run(int count, Ask ask, Begin begin, Wait wait, Use use, Drain drain) {
    auto fetch = [&](int x, int at) { if (x < count && ask(x, at)) asked |= 1u << at; };
    if (!broken) {
#ifdef __CUDACC__
#pragma unroll
#endif
      for (int x = 0; x < kStages - 1; ++x) fetch(x, place(x));
    }
    begin();
    if (broken) return;
    for (int x = 0; x < count; ++x) {
      fetch(x + kStages - 1, place(kStages - 1));
      if (!wait(stage, phase)) {
        broken = true;
        for (int at = 0; at < kStages; ++at)
          if (asked >> at & 1) drain(at, parity(at));
        asked = 0;
        return;
      }
      use(x, stage);
      take();
    }
  }
};

}  // namespace dkv
