// Which tokens of a run a store copy moves, and which of a block's the rotation turns. Plain C++, so that a host compiler can check the
// arithmetic over its whole range.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define GKV_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define GKV_HOST_DEVICE inline
#endif

namespace gkv {

constexpr int kRun = 8;        // tokens of a run

struct RunRows { int lo, hi; };   // tokens lo .. hi - 1 of the run (none: lo >= hi), both in 0 .. kRun

// Tokens t0 .. t0 + kRun - 1 of a sequence that are below its count (below 0 as 0, above n_tokens as n_tokens) and whose row
// first + t is one of 0 .. capacity - 1. first and count are whatever the caller's arrays hold. A first above the capacity has no row
// just as the capacity has none, and one below -2^30 just as -2^30 (there are fewer tokens than that), so they are brought there
// first; with t0 up to 2^30 + 64 and a capacity up to 2^24 everything that follows fits 32 bits.
GKV_HOST_DEVICE RunRows run_rows(int32_t first, int32_t count, int n_tokens, int capacity, int t0) {
    const int n = count < 0 ? 0 : count < n_tokens ? count : n_tokens;
    const int row0 = (first > capacity ? capacity : first < -(1 << 30) ? -(1 << 30) : first) + t0;
    const int left = n - t0, room = capacity - row0, hi = left < room ? left : room, lo = -row0;
    return {lo < 0 ? 0 : lo > kRun ? kRun : lo, hi < 0 ? 0 : hi > kRun ? kRun : hi};
}

// How many of the tokens t0 .. t0 + per - 1 are below a sequence's count (below 0 as 0, above n_tokens as n_tokens), whatever the
// caller's array holds.
GKV_HOST_DEVICE int tokens_here(int32_t count, int n_tokens, int t0, int per) {
    const int left = (count < 0 ? 0 : count < n_tokens ? count : n_tokens) - t0;
    return left < 0 ? 0 : left < per ? left : per;
}

}  // namespace gkv
