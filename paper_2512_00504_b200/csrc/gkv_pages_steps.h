// Where a warp of the paged attention is in its ring of copies, and the shape of the merge behind it. Plain C++, so that a host compiler
// can check it.
#pragma once

#include <stdint.h>

#ifndef GKV_HOST_DEVICE
#ifdef __CUDACC__
#define GKV_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define GKV_HOST_DEVICE inline
#endif
#endif

namespace gkv {

// The place of a step in a ring of S stages: step s is stage s % S, and its copies complete that barrier's phase s / S, which is waited
// for by its parity.
template <int S>
struct RingPlace {
    int stage = 0;
    uint32_t parity = 0;
    GKV_HOST_DEVICE void next() {
        if (++stage == S) { stage = 0; parity ^= 1; }
    }
};
// A warp that gives up at a step (nothing is issued after that) has the copies of that step and of some behind it under way, `copies`
// steps' in all: wait(stage, parity) for each of them, and for nothing else.
template <int S, class Wait>
GKV_HOST_DEVICE void drain_ring(RingPlace<S> at, int copies, Wait wait) {
    for (; copies > 0; --copies, at.next()) wait(at.stage, at.parity);
}

// The merge of `units` units on a device of `sms` SMs: 2^split CTAs a unit, which with few units are CTAs of 256 threads, two an SM, else
// of 128, eight an SM, as many as fit the device at once.
struct MergeShape {
    bool few;
    int split;
};
GKV_HOST_DEVICE MergeShape merge_shape(int64_t units, int sms) {
    MergeShape m = {units <= 2ll * sms, 0};
    while (m.split < (m.few ? 3 : 2) && (units << (m.split + 1)) <= (m.few ? 2ll : 8ll) * sms) ++m.split;
    return m;
}

}  // namespace gkv
