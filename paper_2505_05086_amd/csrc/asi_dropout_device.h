// Which elements dropout keeps (asi_dropout.hip, asi_residual.hip): 16 bits of Philox4x32-10 for each, eight neighbouring elements a
// call.  16 bits and not 32 halve what the generator costs (70 integer multiplications and additions a call); the share that is
// dropped is then a multiple of 2^-16 and the factor of the others is one over the share that is kept, so that the mean stays exact.
#pragma once
#include "asi_lm_device.h"

namespace asi {

struct Keep {
    uint32_t key0, key1, offset0, offset1;
    uint32_t below;            // an element is dropped if its 16 bits are below this
    float factor;
    const int64_t* seed;       // the key, if given
};

__device__ __forceinline__ void read_seed(Keep* k) {
    if (!k->seed) return;
    const uint64_t s = (uint64_t)*k->seed;
    k->key0 = (uint32_t)s;
    k->key1 = (uint32_t)(s >> 32);
}
// the bits of elements 8 group .. 8 group + 7, two to a word
__device__ __forceinline__ void drawn(const Keep& k, unsigned long long group, uint32_t w[4]) {
    philox4x32_10((uint32_t)group, (uint32_t)(group >> 32), k.offset0, k.offset1, k.key0, k.key1, w);
}
// the bits of elements first .. first + 7 for any first
__device__ __forceinline__ void drawn_from(const Keep& k, unsigned long long first, uint32_t w[4]) {
    const int shift = (int)(first & 7);
    uint32_t u[8];
    drawn(k, first >> 3, u);
    if (shift == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = u[i];
        return;
    }
    drawn(k, (first >> 3) + 1, u + 4);
    const int whole = shift >> 1;
    uint32_t t[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) t[i] = whole == 0 ? u[i] : whole == 1 ? u[i + 1] : whole == 2 ? u[i + 2] : u[i + 3];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (shift & 1) ? (t[i] >> 16) | (t[i + 1] << 16) : t[i];
}
__device__ __forceinline__ bool kept(const Keep& k, const uint32_t w[4], int e) {
    return ((e & 1) ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu) >= k.below;
}

// ---- host ----
// Fills what the device reads from p, seed and offset; false if p is none that is taken.
inline bool fill_keep(double p, int64_t seed, int64_t offset, const int64_t* on_device, Keep* k) {
    if (!(p >= 0.0 && p < 1.0)) return false;
    const double below = __builtin_rint(p * 65536.0);
    if (below >= 65536.0) return false;
    k->key0 = (uint32_t)(uint64_t)seed;
    k->key1 = (uint32_t)((uint64_t)seed >> 32);
    k->offset0 = (uint32_t)(uint64_t)offset;
    k->offset1 = (uint32_t)((uint64_t)offset >> 32);
    k->below = (uint32_t)below;
    k->factor = (float)(65536.0 / (65536.0 - below));
    k->seed = on_device;
    return true;
}

}  // namespace asi
