// AdamW over many tensors (include/asi_lm.h).
//
// A launch takes the records of up to kTensors tensors by value; every workgroup finds its tensor from its block index and
// updates a chunk of it, each lane 16 bytes of fp32 (4 elements) or two of them (8, states in 8 bits: half a wave then has the 256
// elements that share a scale).  The update reads and writes each element once and is bound by memory.  A chunk is one piece a wave:
// many short workgroups keep the memory busier than few that loop (six blocks of 2048 in fp32, 308 million elements: chunks of 8192,
// 4096, 1024 elements 1667, 1638, 1571 us; past the caches 1383 us, 6.2 TB/s; 103 million elements in bf16 with fp32 copies and states of
// 8 bits 301 us, 5.5 TB/s).
//
// Products, sums, the quotient and the root are rounded one by one (no contraction), so that the result is that of the same
// formula in elementary fp32 operations, bit for bit: an 8-bit code then does not depend on how a compiler fused it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "asi_lm_device.h"

namespace asi {
namespace {

constexpr int kTensors = 40;
constexpr int kThreads = 256;
constexpr int kBlock = ASI_ADAMW_BLOCK;          // elements that share a scale
constexpr float kCodeMax = 448.f;                // largest value of the 8-bit format
constexpr float kLeastScale = 0x1p-126f;

struct Tensor {
    void* param;
    const void* grad;
    float* master;
    void* avg;
    void* sq;
    float* avg_scale;
    float* sq_scale;
    long long count;
    float decay, rate;       // 1 - lr * weight_decay; lr / (1 - beta1^step)
    int vec, pad;            // every pointer allows vectors
};
struct Args {
    float b1, c1, b2, c2, root_factor, eps;      // c = 1 - beta; root_factor = 1 / sqrt(1 - beta2^step)
    const float* grad_scale;
    const int32_t* skip;
    int first[kTensors + 1];                     // of each tensor's workgroups
    Tensor t[kTensors];
};

// E elements of a lane: neighbours where vectors are allowed, otherwise and at a tensor's end as far apart as the piece has lanes, so
// that neighbouring lanes have neighbours either way.
template <int E> struct Part {
    long long at, count;
    int apart;
    bool vec;
    __device__ __forceinline__ long long index(int i) const { return vec ? at + i : at + (long long)apart * i; }
    __device__ __forceinline__ bool has(int i) const { return vec || index(i) < count; }
};
template <typename T, int E> __device__ __forceinline__ void load(const T* p, const Part<E>& q, float* f) {
    if (q.vec) {
        load_values_past<E>(p + q.at, f);
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] = q.has(i) ? to_f32(p[q.index(i)]) : 0.f;
    }
}
template <typename T, int E> __device__ __forceinline__ void store(T* p, const Part<E>& q, const float* f) {
    if (q.vec) {
        store_values_past<E>(p + q.at, f);
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (q.has(i)) p[q.index(i)] = from_f32<T>(f[i]);
    }
}
// 8 codes of a lane, in two words
using Lane8 = Part<8>;
__device__ __forceinline__ uint2 load_codes(const uint8_t* p, const Lane8& q) {
    if (q.vec) {
        uint2 v;
        load_past(p + q.at, &v);
        return v;
    }
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (q.has(i)) w[i / 4] |= (uint32_t)p[q.index(i)] << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store_codes(uint8_t* p, const Lane8& q, uint2 w) {
    if (q.vec) {
        store_past(p + q.at, w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (q.has(i)) p[q.index(i)] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
}
__device__ __forceinline__ void decode(uint32_t w, float scale, float* f) {
#pragma clang fp contract(off)
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    f[0] = lo[0] * scale; f[1] = lo[1] * scale; f[2] = hi[0] * scale; f[3] = hi[1] * scale;
}
__device__ __forceinline__ float finite_magnitude(float x) {
    const float a = fabsf(x);
    return a < __builtin_inff() ? a : 0.f;
}
// Codes of the 256 values of half a wave and their scale.  POSITIVE: values are roots, of which a positive one is not held as zero.
template <bool POSITIVE> __device__ __forceinline__ uint2 encode(const float* f, float* scale) {
#pragma clang fp contract(off)
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, finite_magnitude(f[i]));
    most = __uint_as_float(half_wave_max(__float_as_uint(most)));         // magnitudes are in the order of their bits
    float s = most * (1.f / kCodeMax);
    const bool held = s >= kLeastScale;
    const float inv = held ? 1.f / s : 0.f;
    *scale = held ? s : 0.f;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = f[i] * inv;
        if (!(fabsf(f[i]) < __builtin_inff())) v[i] = __builtin_nanf("");
    }
    uint32_t w[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        w[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * k], v[4 * k + 1], 0, false);
        w[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * k + 2], v[4 * k + 3], (int)w[k], true);
        if (POSITIVE && held) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (f[4 * k + i] > 0.f && (w[k] >> (8 * i) & 0xffu) == 0) w[k] |= 1u << (8 * i);
        }
    }
    return make_uint2(w[0], w[1]);
}

template <bool EIGHT> struct Shape {
    static constexpr int E = EIGHT ? 8 : 4, lanes = kBlock / E, chunk = kThreads * E;     // lanes of a piece of 256 elements
};
template <typename PT, typename GT, bool MASTER, bool EIGHT>
__global__ __launch_bounds__(kThreads) void k_adamw(const Args a) {
#pragma clang fp contract(off)
    constexpr int E = Shape<EIGHT>::E, LANES = Shape<EIGHT>::lanes;
    if (a.skip && *a.skip != 0) return;
    int j = 0;
#pragma unroll
    for (int k = 1; k < kTensors; ++k) j += (int)blockIdx.x >= a.first[k];
    const Tensor& t = a.t[j];
    const float gs = a.grad_scale ? *a.grad_scale : 1.f;
    const int lane = threadIdx.x & (LANES - 1);
    const long long block = (long long)((int)blockIdx.x - a.first[j]) * (kThreads / LANES) + threadIdx.x / LANES, base = block * kBlock;
    Part<E> q;
    q.count = t.count;
    q.apart = LANES;
    q.vec = t.vec && base + kBlock <= t.count;
    q.at = base + (q.vec ? E * lane : lane);
    float p[E], g[E], m[E], v[E], root[E];
    if (MASTER) load(t.master, q, p);
    else load(static_cast<const PT*>(t.param), q, p);
    load(static_cast<const GT*>(t.grad), q, g);
    if constexpr (EIGHT) {
        const bool any = base < t.count;
        const uint2 wm = load_codes(static_cast<const uint8_t*>(t.avg), q), wv = load_codes(static_cast<const uint8_t*>(t.sq), q);
        const float sm = any ? t.avg_scale[block] : 0.f, sv = any ? t.sq_scale[block] : 0.f;
        decode(wm.x, sm, m); decode(wm.y, sm, m + 4);
        decode(wv.x, sv, root); decode(wv.y, sv, root + 4);
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = root[i] * root[i];
    } else {
        load(static_cast<const float*>(t.avg), q, m);
        load(static_cast<const float*>(t.sq), q, v);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const float gi = g[i] * gs;
        m[i] = m[i] * a.b1 + gi * a.c1;
        v[i] = v[i] * a.b2 + (gi * gi) * a.c2;
        root[i] = sqrtf(v[i]);
        const float u = m[i] / (root[i] * a.root_factor + a.eps);
        p[i] = p[i] * t.decay - u * t.rate;
    }
    if (MASTER) store(t.master, q, p);
    store(static_cast<PT*>(t.param), q, p);
    if constexpr (EIGHT) {
        float sm, sv;
        const uint2 wm = encode<false>(m, &sm), wv = encode<true>(root, &sv);
        store_codes(static_cast<uint8_t*>(t.avg), q, wm);
        store_codes(static_cast<uint8_t*>(t.sq), q, wv);
        if (lane == 0 && base < t.count) {
            t.avg_scale[block] = sm;
            t.sq_scale[block] = sv;
        }
    } else {
        store(static_cast<float*>(t.avg), q, m);
        store(static_cast<float*>(t.sq), q, v);
    }
}

template <typename PT, typename GT, bool MASTER> void launch(const Args& a, bool eight, hipStream_t st) {
    const dim3 grid((unsigned)a.first[kTensors]);
    if (eight) hipLaunchKernelGGL((k_adamw<PT, GT, MASTER, true>), grid, kThreads, 0, st, a);
    else hipLaunchKernelGGL((k_adamw<PT, GT, MASTER, false>), grid, kThreads, 0, st, a);
}
// Kinds of tensor, each with an instantiation: parameter and gradient types, with or without an fp32 copy.
int kind_of(const asi_adamw_tensor& t) { return (t.param_dtype == ASI_BF16 ? 1 : 0) + (t.grad_dtype == ASI_BF16 ? 2 : 0) + (t.master ? 4 : 0); }
void launch_kind(int kind, const Args& a, bool eight, hipStream_t st) {
    switch (kind) {
        case 0: launch<float, float, false>(a, eight, st); break;
        case 1: launch<bf16_t, float, false>(a, eight, st); break;
        case 2: launch<float, bf16_t, false>(a, eight, st); break;
        case 3: launch<bf16_t, bf16_t, false>(a, eight, st); break;
        case 4: launch<float, float, true>(a, eight, st); break;
        case 5: launch<bf16_t, float, true>(a, eight, st); break;
        case 6: launch<float, bf16_t, true>(a, eight, st); break;
        default: launch<bf16_t, bf16_t, true>(a, eight, st); break;
    }
}
bool valid(const asi_adamw_tensor& t, bool eight) {
    if (!dtype_ok(t.param_dtype) || !dtype_ok(t.grad_dtype) || t.count < 0 || t.count > (1LL << 40)) return false;
    if (!std::isfinite(t.lr) || !std::isfinite(t.weight_decay)) return false;
    if (t.count == 0) return true;
    if (!t.param || !t.grad || !t.exp_avg || !t.exp_avg_sq || (eight && (!t.exp_avg_scale || !t.exp_avg_sq_scale))) return false;
    const bool fit = aligned(t.param, dtype_size(t.param_dtype)) && aligned(t.grad, dtype_size(t.grad_dtype)) && aligned(t.master, 4);
    return fit && (eight ? aligned(t.exp_avg_scale, 4) && aligned(t.exp_avg_sq_scale, 4) : aligned(t.exp_avg, 4) && aligned(t.exp_avg_sq, 4));
}

}  // namespace
}  // namespace asi

using namespace asi;

extern "C" asi_status asi_adamw(int32_t count, const asi_adamw_tensor* tensors, int32_t state_bits, double beta1, double beta2,
                                double eps, int64_t step, const float* grad_scale, const int32_t* skip, asi_stream_t stream) {
    if (count < 0 || (count > 0 && !tensors) || step < 1) return ASI_ERR_INVALID_ARG;
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !std::isfinite(eps)) return ASI_ERR_INVALID_ARG;
    if (state_bits != 32 && state_bits != 8) return ASI_ERR_UNSUPPORTED;
    if (!aligned(grad_scale, 4) || !aligned(skip, 4)) return ASI_ERR_INVALID_ARG;
    const bool eight = state_bits == 8;
    for (int32_t i = 0; i < count; ++i)
        if (!valid(tensors[i], eight)) return ASI_ERR_INVALID_ARG;
    Args a{};
    a.b1 = (float)beta1; a.c1 = (float)(1.0 - beta1);
    a.b2 = (float)beta2; a.c2 = (float)(1.0 - beta2);
    a.root_factor = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    a.eps = (float)eps;
    a.grad_scale = grad_scale;
    a.skip = skip;
    const int chunk = eight ? Shape<true>::chunk : Shape<false>::chunk;
    constexpr long long most = most_workgroups(kThreads);
    bool any = false;
    const double correction = 1.0 - std::pow(beta1, (double)step);
    for (int kind = 0; kind < 8; ++kind) {
        int n = 0;
        long long blocks = 0;
        auto flush = [&]() {
            for (int k = n; k <= kTensors; ++k) a.first[k] = (int)blocks;
            if (n) launch_kind(kind, a, eight, static_cast<hipStream_t>(stream));
            any |= n > 0;
            n = 0;
            blocks = 0;
        };
        for (int32_t i = 0; i < count; ++i) {
            const asi_adamw_tensor& s = tensors[i];
            if (s.count == 0 || kind_of(s) != kind) continue;
            const size_t ps = dtype_size(s.param_dtype), gs = dtype_size(s.grad_dtype), ss = eight ? 1 : 4;
            // accesses of up to 16 bytes
            const size_t state = eight ? 8 : 16, e = eight ? 8 : 4;
            const bool vec = aligned(s.param, std::min<size_t>(16, e * ps)) && aligned(s.grad, std::min<size_t>(16, e * gs)) && aligned(s.master, 16) &&
                             aligned(s.exp_avg, state) && aligned(s.exp_avg_sq, state);
            // a tensor that is more than a launch takes is several
            for (long long at = 0; at < s.count; at += most * chunk) {
                const long long n_here = std::min<long long>(s.count - at, most * chunk), need = (n_here + chunk - 1) / chunk;
                if (n == kTensors || blocks + need > most) flush();
                Tensor& t = a.t[n];
                t.param = static_cast<char*>(s.param) + at * ps;
                t.grad = static_cast<const char*>(s.grad) + at * gs;
                t.master = s.master ? s.master + at : nullptr;
                t.avg = static_cast<char*>(s.exp_avg) + at * ss;
                t.sq = static_cast<char*>(s.exp_avg_sq) + at * ss;
                t.avg_scale = eight ? s.exp_avg_scale + at / kBlock : nullptr;
                t.sq_scale = eight ? s.exp_avg_sq_scale + at / kBlock : nullptr;
                t.count = n_here;
                t.decay = (float)(1.0 - s.lr * s.weight_decay);
                t.rate = (float)(s.lr / correction);
                t.vec = vec;
                a.first[n] = (int)blocks;
                blocks += need;
                ++n;
            }
        }
        flush();
    }
    return any ? launched() : ASI_OK;
}
