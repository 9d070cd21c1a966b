// Device helpers of the language-model operators (include/asi_lm.h): typed vectors of 16 bytes, rounding to
// bf16, reductions over a wave.  Host helpers for their argument checks.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/asi_lm.h"
#include "asi_device.h"

namespace asi {

constexpr int kWave = 64;

// bf16 rounding is to nearest, ties to even, NaN stays NaN (the conversion instruction of gfx950)
__device__ __forceinline__ bf16_t to_bf16(float x) {
    union { __bf16 b; uint16_t u; } c;
    c.b = (__bf16)x;
    return bf16_t{c.u};
}
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16_t from_f32<bf16_t>(float x) { return to_bf16(x); }

// 16 and 8 bytes of any type
typedef uint32_t words4 __attribute__((ext_vector_type(4), may_alias));
typedef uint32_t words2 __attribute__((ext_vector_type(2), may_alias));
__device__ __forceinline__ uint4 load_words4(const void* p) {
    const words4 w = *static_cast<const words4*>(p);
    return make_uint4(w.x, w.y, w.z, w.w);
}
__device__ __forceinline__ uint2 load_words2(const void* p) {
    const words2 w = *static_cast<const words2*>(p);
    return make_uint2(w.x, w.y);
}
__device__ __forceinline__ void store_words(void* p, uint4 v) { *static_cast<words4*>(p) = words4{v.x, v.y, v.z, v.w}; }
__device__ __forceinline__ void store_words(void* p, uint2 v) { *static_cast<words2*>(p) = words2{v.x, v.y}; }
// Accesses past the caches, of what a kernel touches once: kept in the caches it would push out what is used again (zeros into 32000
// rows of 2048 in fp32 67.8 -> 59.8 us; 4096 x 32000 logits and their gradient 105 -> 102 with the stores, 99 with the loads; AdamW on
// 308 million elements 1548 -> 1415 us).
__device__ __forceinline__ void store_past(void* p, uint4 v) { __builtin_nontemporal_store(words4{v.x, v.y, v.z, v.w}, static_cast<words4*>(p)); }
__device__ __forceinline__ void store_past(void* p, uint2 v) { __builtin_nontemporal_store(words2{v.x, v.y}, static_cast<words2*>(p)); }
__device__ __forceinline__ void load_past(const void* p, uint4* v) {
    const words4 w = __builtin_nontemporal_load(static_cast<const words4*>(p));
    *v = make_uint4(w.x, w.y, w.z, w.w);
}
__device__ __forceinline__ void load_past(const void* p, uint2* v) {
    const words2 w = __builtin_nontemporal_load(static_cast<const words2*>(p));
    *v = make_uint2(w.x, w.y);
}

// 16 bytes of a row: 4 fp32 or 8 bf16 values, kept as loaded so that many can be in flight at little cost in registers
template <typename T> struct Vec16 {
    static constexpr int N = 16 / sizeof(T);
    uint4 raw;
    __device__ __forceinline__ void load(const T* p) { raw = load_words4(p); }
    __device__ __forceinline__ void load_once(const T* p) { load_past(p, &raw); }
    __device__ __forceinline__ void store(T* p) const { store_words(p, raw); }
    __device__ __forceinline__ float get(int i) const;
    __device__ __forceinline__ void set(const float* f);
};
template <> __device__ __forceinline__ float Vec16<float>::get(int i) const {
    return __uint_as_float(i == 0 ? raw.x : i == 1 ? raw.y : i == 2 ? raw.z : raw.w);
}
template <> __device__ __forceinline__ float Vec16<bf16_t>::get(int i) const {
    const uint32_t w = (i >> 1) == 0 ? raw.x : (i >> 1) == 1 ? raw.y : (i >> 1) == 2 ? raw.z : raw.w;
    return __uint_as_float((i & 1) ? (w & 0xffff0000u) : (w << 16));
}
template <> __device__ __forceinline__ void Vec16<float>::set(const float* f) {
    raw = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) { return (uint32_t)to_bf16(lo).bits | ((uint32_t)to_bf16(hi).bits << 16); }
template <> __device__ __forceinline__ void Vec16<bf16_t>::set(const float* f) {
    raw = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}

// N values (a multiple of 4) to and from fp32, in accesses of up to 16 bytes; the address has to be a multiple of min(16, N * size)
template <int N> __device__ __forceinline__ void load_values(const float* p, float* f) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        Vec16<float> v;
        v.load(p + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) f[i + k] = v.get(k);
    }
}
template <int N> __device__ __forceinline__ void load_values(const bf16_t* p, float* f) {
    if constexpr (N % 8 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 8) {
            Vec16<bf16_t> v;
            v.load(p + i);
#pragma unroll
            for (int k = 0; k < 8; ++k) f[i + k] = v.get(k);
        }
    } else {
        static_assert(N == 4, "4 or a multiple of 8");
        const uint2 v = load_words2(p);
        f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
        f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
    }
}
template <int N> __device__ __forceinline__ void store_values(float* p, const float* f) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        Vec16<float> v;
        v.set(f + i);
        v.store(p + i);
    }
}
template <int N> __device__ __forceinline__ void store_values(bf16_t* p, const float* f) {
    if constexpr (N % 8 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 8) {
            Vec16<bf16_t> v;
            v.set(f + i);
            v.store(p + i);
        }
    } else {
        static_assert(N == 4, "4 or a multiple of 8");
        store_words(p, make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])));
    }
}

// The same past the caches: for large results that are written once and not read soon, and for what is read once.
template <int N> __device__ __forceinline__ void load_values_past(const float* p, float* f) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        Vec16<float> v;
        v.load_once(p + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) f[i + k] = v.get(k);
    }
}
template <int N> __device__ __forceinline__ void load_values_past(const bf16_t* p, float* f) {
    if constexpr (N % 8 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 8) {
            Vec16<bf16_t> v;
            v.load_once(p + i);
#pragma unroll
            for (int k = 0; k < 8; ++k) f[i + k] = v.get(k);
        }
    } else {
        static_assert(N == 4, "4 or a multiple of 8");
        uint2 v;
        load_past(p, &v);
        f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
        f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
    }
}
template <int N> __device__ __forceinline__ void store_values_past(float* p, const float* f) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        Vec16<float> v;
        v.set(f + i);
        store_past(p + i, v.raw);
    }
}
template <int N> __device__ __forceinline__ void store_values_past(bf16_t* p, const float* f) {
    if constexpr (N % 8 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 8) {
            Vec16<bf16_t> v;
            v.set(f + i);
            store_past(p + i, v.raw);
        }
    } else {
        static_assert(N == 4, "4 or a multiple of 8");
        store_past(p, make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])));
    }
}

// Reductions over `width` neighbouring lanes (a power of two); every lane gets the result, always in the same order.
template <int WIDTH = kWave> __device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
    for (int o = WIDTH / 2; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// The largest over the wave, or over each half of it, in every lane: steps within 16 lanes, then across their rows, without a way
// through LDS.
template <int CTRL> __device__ __forceinline__ uint32_t moved(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, CTRL, 0xf, 0xf, false); }
__device__ __forceinline__ uint32_t max_at_row_pairs(uint32_t x) {
    x = max(x, moved<0x111>(x));      // from 1, 2, 4 and 8 lanes before it in its row of 16
    x = max(x, moved<0x112>(x));
    x = max(x, moved<0x114>(x));
    x = max(x, moved<0x118>(x));
    return max(x, moved<0x142>(x));   // the last lane of a row to the next row
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    x = max_at_row_pairs(x);
    x = max(x, moved<0x143>(x));      // the last lane of the first half to the second half
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ __forceinline__ uint32_t half_wave_max(uint32_t x) {
    x = max_at_row_pairs(x);
    const uint32_t lower = (uint32_t)__builtin_amdgcn_readlane((int)x, 31), upper = (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
    return (threadIdx.x & 32) ? upper : lower;
}

// the larger of two, NaN if either is
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// ---- host ----
inline bool dtype_ok(int32_t d) { return d == ASI_F32 || d == ASI_BF16; }
inline size_t dtype_size(int32_t d) { return d == ASI_F32 ? 4 : 2; }
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }
// A launch has fewer than 2^32 threads in a dimension: workgroups that are sure to fit.
constexpr long long most_workgroups(int threads) { return 0xffffffffLL / threads; }
inline asi_status launched() { return hipGetLastError() == hipSuccess ? ASI_OK : ASI_ERR_HIP; }

}  // namespace asi
