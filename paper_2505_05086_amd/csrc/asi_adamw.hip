// AdamW over many tensors (include/asi_lm.h).
//
// A launch takes the records of up to kTensors tensors by value; every workgroup finds its tensor from its block index and
// updates 4096 consecutive elements of it, each wave in pieces of 256, which is also the block that shares a scale of the
// 8-bit states.  The update reads and writes each element once and is bound by memory.
//
// Products, sums, the quotient and the root are rounded one by one (no contraction), so that the result is that of the same
// formula in elementary fp32 operations, bit for bit: an 8-bit code then does not depend on how a compiler fused it.
#include <hip/hip_runtime.h>

#include <cmath>

#include "asi_lm_device.h"

namespace asi {
namespace {

constexpr int kTensors = 40;
constexpr int kThreads = 256;
constexpr int kPiece = ASI_ADAMW_BLOCK;          // elements a wave takes at a time: 4 a lane
constexpr int kChunk = 4096;                     // elements of a workgroup
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
    int vec, pad;            // every pointer allows loads of four elements
};
struct Args {
    float b1, c1, b2, c2, root_factor, eps;      // c = 1 - beta; root_factor = 1 / sqrt(1 - beta2^step)
    const float* grad_scale;
    const int32_t* skip;
    int first[kTensors + 1];                     // of each tensor's workgroups
    Tensor t[kTensors];
};

// Four elements of a lane: neighbours where loads of four are allowed, 64 apart otherwise and at a tensor's end.
struct Quad {
    long long at;
    long long count;
    bool vec;
    __device__ __forceinline__ long long index(int i) const { return vec ? at + i : at + 64LL * i; }
    __device__ __forceinline__ bool has(int i) const { return vec || index(i) < count; }
};
__device__ __forceinline__ void load4(const float* p, const Quad& q, float* f) {
    if (q.vec) {
        const float4 v = *reinterpret_cast<const float4*>(p + q.at);
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = q.has(i) ? p[q.index(i)] : 0.f;
    }
}
__device__ __forceinline__ void load4(const bf16_t* p, const Quad& q, float* f) {
    if (q.vec) {
        const uint2 v = *reinterpret_cast<const uint2*>(p + q.at);
        f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
        f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = q.has(i) ? to_f32(p[q.index(i)]) : 0.f;
    }
}
__device__ __forceinline__ void store4(float* p, const Quad& q, const float* f) {
    if (q.vec) {
        *reinterpret_cast<float4*>(p + q.at) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (q.has(i)) p[q.index(i)] = f[i];
    }
}
__device__ __forceinline__ void store4(bf16_t* p, const Quad& q, const float* f) {
    if (q.vec) {
        *reinterpret_cast<uint2*>(p + q.at) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (q.has(i)) p[q.index(i)] = to_bf16(f[i]);
    }
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, const Quad& q) {
    if (q.vec) return *reinterpret_cast<const uint32_t*>(p + q.at);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (q.has(i)) w |= (uint32_t)p[q.index(i)] << (8 * i);
    return w;
}
__device__ __forceinline__ void store_codes(uint8_t* p, const Quad& q, uint32_t w) {
    if (q.vec) {
        *reinterpret_cast<uint32_t*>(p + q.at) = w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (q.has(i)) p[q.index(i)] = (uint8_t)(w >> (8 * i));
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
// Codes of a wave's 256 values and their scale.  POSITIVE: values are roots, of which a positive one is not held as zero.
template <bool POSITIVE> __device__ __forceinline__ uint32_t encode(const float* f, float* scale) {
#pragma clang fp contract(off)
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = fmaxf(most, finite_magnitude(f[i]));
    most = lanes_max(most);
    float s = most * (1.f / kCodeMax);
    const bool held = s >= kLeastScale;
    const float inv = held ? 1.f / s : 0.f;
    *scale = held ? s : 0.f;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = f[i] * inv;
        if (!(fabsf(f[i]) < __builtin_inff())) v[i] = __builtin_nanf("");
    }
    uint32_t w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], (int)w, true);
    if (POSITIVE && held) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (f[i] > 0.f && (w >> (8 * i) & 0xffu) == 0) w |= 1u << (8 * i);
    }
    return w;
}

template <typename PT, typename GT, bool MASTER, bool EIGHT>
__global__ __launch_bounds__(kThreads) void k_adamw(const Args a) {
#pragma clang fp contract(off)
    if (a.skip && *a.skip != 0) return;
    int j = 0;
#pragma unroll
    for (int k = 1; k < kTensors; ++k) j += (int)blockIdx.x >= a.first[k];
    const Tensor& t = a.t[j];
    const float gs = a.grad_scale ? *a.grad_scale : 1.f;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long begin = (long long)((int)blockIdx.x - a.first[j]) * kChunk;
#pragma unroll 2
    for (int k = 0; k < kChunk / kPiece / (kThreads / 64); ++k) {
        const long long base = begin + (long long)(k * (kThreads / 64) + wave) * kPiece;
        if (base >= t.count) break;
        Quad q;
        q.count = t.count;
        q.vec = t.vec && base + kPiece <= t.count;
        q.at = base + (q.vec ? 4 * lane : lane);
        float p[4], g[4], m[4], v[4], root[4];
        if (MASTER) load4(t.master, q, p);
        else load4(static_cast<const PT*>(t.param), q, p);
        load4(static_cast<const GT*>(t.grad), q, g);
        if (EIGHT) {
            const uint32_t wm = load_codes(static_cast<const uint8_t*>(t.avg), q), wv = load_codes(static_cast<const uint8_t*>(t.sq), q);
            decode(wm, t.avg_scale[base / kPiece], m);
            decode(wv, t.sq_scale[base / kPiece], root);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = root[i] * root[i];
        } else {
            load4(static_cast<const float*>(t.avg), q, m);
            load4(static_cast<const float*>(t.sq), q, v);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float gi = g[i] * gs;
            m[i] = m[i] * a.b1 + gi * a.c1;
            v[i] = v[i] * a.b2 + (gi * gi) * a.c2;
            root[i] = sqrtf(v[i]);
            const float u = m[i] / (root[i] * a.root_factor + a.eps);
            p[i] = p[i] * t.decay - u * t.rate;
        }
        if (MASTER) store4(t.master, q, p);
        store4(static_cast<PT*>(t.param), q, p);
        if (EIGHT) {
            float sm, sv;
            const uint32_t wm = encode<false>(m, &sm), wv = encode<true>(root, &sv);
            store_codes(static_cast<uint8_t*>(t.avg), q, wm);
            store_codes(static_cast<uint8_t*>(t.sq), q, wv);
            if (lane == 0) {
                t.avg_scale[base / kPiece] = sm;
                t.sq_scale[base / kPiece] = sv;
            }
        } else {
            store4(static_cast<float*>(t.avg), q, m);
            store4(static_cast<float*>(t.sq), q, v);
        }
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
    if (!dtype_ok(t.param_dtype) || !dtype_ok(t.grad_dtype) || t.count < 0 || t.count > (1LL << 42)) return false;
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
            const long long need = (s.count + kChunk - 1) / kChunk;
            if (n == kTensors || blocks + need > 0x7fffffffLL) flush();
            Tensor& t = a.t[n];
            t.param = s.param; t.grad = s.grad; t.master = s.master; t.avg = s.exp_avg; t.sq = s.exp_avg_sq;
            t.avg_scale = s.exp_avg_scale; t.sq_scale = s.exp_avg_sq_scale; t.count = s.count;
            t.decay = (float)(1.0 - s.lr * s.weight_decay);
            t.rate = (float)(s.lr / correction);
            const size_t state = eight ? 4 : 16;
            t.vec = aligned(s.param, 4 * dtype_size(s.param_dtype)) && aligned(s.grad, 4 * dtype_size(s.grad_dtype)) &&
                    aligned(s.master, 16) && aligned(s.exp_avg, state) && aligned(s.exp_avg_sq, state);
            a.first[n] = (int)blocks;
            blocks += need;
            ++n;
        }
        flush();
    }
    return any ? launched() : ASI_OK;
}
