// Which tokens of a run a store copy moves. Plain C++, so that a host compiler can check the arithmetic over its whole range.
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
// first + t is one of 0 .. capacity - 1. first and count are whatever the caller's arrays hold: all differences in 64 bits, and
// clamped there.
GKV_HOST_DEVICE RunRows run_rows(int32_t first, int32_t count, int n_tokens, int capacity, int t0) {
    const int64_t n = count < 0 ? 0 : count < n_tokens ? count : n_tokens, row0 = (int64_t)first + t0;
    const int64_t left = n - t0, room = capacity - row0, hi = left < room ? left : room, lo = -row0;
    return {(int)(lo < 0 ? 0 : lo > kRun ? kRun : lo), (int)(hi < 0 ? 0 : hi > kRun ? kRun : hi)};
}

}  // namespace gkv
