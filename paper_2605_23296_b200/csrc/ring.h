// Which rounds of a ring of stages may have copies in flight when its producer leaves.  Plain arithmetic, for host and
// device, so that it can be checked without either.
#pragma once

#ifdef __CUDACC__
#define CPA_HD __host__ __device__
#else
#define CPA_HD
#endif

struct ring_rounds {
    int first, end;           // [first, end)
};

// Round i goes through stage i % stages, and is issued once round i - stages has been consumed.  The producer has issued
// the copies of rounds 0 .. it - 1, and leaves either because it gave up waiting for round it - stages to be consumed
// (which may then be what is in flight), or, `ended`, after announcing round `it`, the end, which copies nothing.  In that
// case round it - stages has been consumed, and its stage's barrier is in a later phase: it must not be waited for.
CPA_HD constexpr ring_rounds ring_in_flight(int it, int stages, bool ended) {
    const int first = it - stages + (ended ? 1 : 0);
    return {first > 0 ? first : 0, it};
}
