// Norms of queries and keys for each head with the position rotation in the same pass, and the backward pass
// (include/asi_lm.h).
//
// A head is read once, into registers, as pairs of 16-byte vectors: vector i of the first half of the rotated part with vector i of
// its second half, which are turned into each other; of what is not turned, and where neighbours are turned into each other, the
// vectors of one half with those of the other.  A lane holds one such pair, a group of 2^k neighbouring lanes a head, so
// that the partners of a rotation are in one lane, neighbouring lanes load and store neighbouring vectors, and only the sum of
// squares crosses lanes.  Heads whose length or addresses do not allow vectors take the kernel that goes element by element, a
// wave a head.
//
// Backward: with u = x r, n = u gain, w = gain dn:  dn = rotation of dy by the negative angle,
//     dx = r (w - u mean(w u)),   dgain = sum dn u.
// Each lane keeps the dgain of its columns over all heads that it takes; the sums of a workgroup's lanes go to scratch
// and a second kernel adds them up, in an order that depends on the sizes alone.
//
// Bound by memory: 4096 tokens of 36 heads of 64 in bf16 10.0 us (3.9 TB/s, a launch's ramp and tail among it), the gradient of 12003 tokens
// of 24 heads of 128 in fp32 80 us (5.6 TB/s); 8 tokens by the launch, 3.5 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "asi_lm_device.h"

namespace asi {
namespace {

constexpr int kThreads = 256;

// n / d of 0 <= n < 2^31 by a product: m = floor(2^(31 + l) / d) + 1 with 2^l >= d is off by less than n can show
struct Divider {
    uint64_t m;
    int shift, d;
    void set(int divisor) {
        d = divisor;
        int l = 0;
        while ((1LL << l) < d) ++l;
        shift = 31 + l;
        m = (1ull << shift) / (uint64_t)d + 1;
    }
    __device__ __forceinline__ int quotient(int n) const { return (int)((uint64_t)(uint32_t)n * m >> shift); }
};

struct Side {                      // queries or keys
    const void* x;
    const void* gain;
    void* y;                       // forward: output; backward: dx
    const void* dy;                // backward: gradient of the output
    long long xs[3], ys[3], ds[3]; // strides of x, of the output (or dy), of dx
    int heads;
    Divider by_heads;              // backward
};
struct Args {
    Side side[2];
    const int64_t* positions;
    const float* cos;
    const float* sin;
    float* part;                   // backward: [side][workgroup][head_dim]
    long long rows;                // batch * tokens
    long long first;               // forward: what the launch begins with
    long long position_stride, max_position;
    Divider by_tokens, by_parts;   // parts: what the heads of a token are taken in, forward
    int q_parts, parts;
    int tokens, head_dim, rot_dim, interleaved;
    float eps, inv_dim;
};

// Position of token t of batch entry b; -1 where there are no angles for it.
__device__ __forceinline__ long long position_of(const Args& a, int b, int t) {
    if (a.rot_dim == 0) return 0;
    const long long p = a.positions ? a.positions[b * a.position_stride + t] : t;
    return p >= 0 && p < a.max_position ? p : -1;
}

// The two vectors of a lane's pair `slot`: their first elements, and whether they are turned.
struct Pair {
    int ia, ib;
    bool ta, tb;
};
template <typename T, bool INTER> __device__ __forceinline__ Pair pair_of(int slot, int dim, int rot) {
    constexpr int N = Vec16<T>::N;
    if (INTER) {
        const int ia = slot * N, ib = dim / 2 + slot * N;
        return {ia, ib, ia < rot, ib < rot};
    }
    const int behind = slot * N - rot / 2;        // elements behind the rotated part's first half
    if (behind < 0) return {slot * N, rot / 2 + slot * N, true, true};
    return {rot + behind, rot + (dim - rot) / 2 + behind, false, false};
}
// (f, g) turned by the lane's angles; `sign` -1 turns back.  INTER: neighbours within the vectors are partners, the first half of the
// angles belongs to f.
template <typename T, bool INTER> __device__ __forceinline__ void turn(float* f, float* g, const float* c, const float* s, float sign) {
    constexpr int N = Vec16<T>::N;
    if (INTER) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float s0 = sign * s[i / 2], s1 = sign * s[N / 2 + i / 2], c0 = c[i / 2], c1 = c[N / 2 + i / 2];
            const float a = f[i], b = f[i + 1], d = g[i], e = g[i + 1];
            f[i] = a * c0 - b * s0; f[i + 1] = b * c0 + a * s0;
            g[i] = d * c1 - e * s1; g[i + 1] = e * c1 + d * s1;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float si = sign * s[i], a = f[i], b = g[i];
            f[i] = a * c[i] - b * si;
            g[i] = b * c[i] + a * si;
        }
    }
}
template <int M> __device__ __forceinline__ void load_angles(const Args& a, long long at, bool in_range, bool turned, float* c, float* s) {
    if (turned && in_range) {
        if constexpr (M % 4 == 0) {
            load_values<M>(a.cos + at, c);
            load_values<M>(a.sin + at, s);
        } else {
            const uint2 vc = load_words2(a.cos + at), vs = load_words2(a.sin + at);
            c[0] = __uint_as_float(vc.x); c[1] = __uint_as_float(vc.y);
            s[0] = __uint_as_float(vs.x); s[1] = __uint_as_float(vs.y);
        }
    } else {
#pragma unroll
        for (int i = 0; i < M; ++i) {
            c[i] = turned ? __builtin_nanf("") : 1.f;
            s[i] = 0.f;
        }
    }
}
// cos and sin of a lane's pair, 1 and 0 where it is not turned, NaN where there is no such position
template <typename T, bool INTER> __device__ __forceinline__ void load_angles(const Args& a, const Pair& p, long long pos, float* c, float* s) {
    constexpr int N = Vec16<T>::N;
    const long long row = pos * (a.rot_dim / 2);
    if (INTER) {
        load_angles<N / 2>(a, row + p.ia / 2, pos >= 0, p.ta, c, s);
        load_angles<N / 2>(a, row + p.ib / 2, pos >= 0, p.tb, c + N / 2, s + N / 2);
    } else {
        load_angles<N>(a, row + p.ia, pos >= 0, p.ta, c, s);
    }
}
// gains: N values, their address a multiple of 16 bytes or of the N values' size
template <typename T, typename G> __device__ __forceinline__ void load_gain(const void* gain, int at, float* w) {
    constexpr int N = Vec16<T>::N;
    if (gain) {
        load_values<N>(static_cast<const G*>(gain) + at, w);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = 1.f;
    }
}

// Forward: a group of GROUP lanes takes HEADS neighbouring heads of a token, which share its angles and the gains.
template <typename T, typename G, int GROUP, int HEADS, bool INTER> __global__ __launch_bounds__(kThreads) void k_rotate(const Args a) {
    constexpr int N = Vec16<T>::N;
    const int lane = threadIdx.x & (GROUP - 1);
    const long long id = a.first + (long long)blockIdx.x * (kThreads / GROUP) + threadIdx.x / GROUP;
    const bool have = id < a.rows * a.parts;
    const int row = have ? a.by_parts.quotient((int)id) : 0;
    int part = have ? (int)id - row * a.parts : 0;
    const int b = a.by_tokens.quotient(row), t = row - b * a.tokens;
    const bool is_k = part >= a.q_parts;
    if (is_k) part -= a.q_parts;
    const Side& s = a.side[is_k];
    const Pair p = pair_of<T, INTER>(lane, a.head_dim, a.rot_dim);
    const bool mine = have && lane * 2 * N < a.head_dim;
    const int h0 = part * HEADS;
    const T* x = static_cast<const T*>(s.x) + b * s.xs[0] + t * s.xs[1] + h0 * s.xs[2];
    Vec16<T> va[HEADS], vb[HEADS];
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
        va[h].raw = vb[h].raw = make_uint4(0, 0, 0, 0);
        if (mine && h0 + h < s.heads) { va[h].load(x + h * s.xs[2] + p.ia); vb[h].load(x + h * s.xs[2] + p.ib); }
    }
    float wa[N], wb[N], c[N], sn[N];
    if (mine) {
        load_gain<T, G>(s.gain, p.ia, wa);
        load_gain<T, G>(s.gain, p.ib, wb);
        load_angles<T, INTER>(a, p, position_of(a, b, t), c, sn);
    }
    T* y = static_cast<T*>(s.y) + b * s.ys[0] + t * s.ys[1] + h0 * s.ys[2];
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
        float f[N], g[N], sum = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            f[i] = va[h].get(i); g[i] = vb[h].get(i);
            sum += f[i] * f[i] + g[i] * g[i];
        }
        sum = lanes_sum<GROUP>(sum);
        if (!mine || h0 + h >= s.heads) continue;
        const float r = 1.f / sqrtf(sum * a.inv_dim + a.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) { f[i] *= r * wa[i]; g[i] *= r * wb[i]; }
        turn<T, INTER>(f, g, c, sn, 1.f);
        store_values<N>(y + h * s.ys[2] + p.ia, f);
        store_values<N>(y + h * s.ys[2] + p.ib, g);
    }
}

// Backward: the groups of the grid take the heads of one side after another, a grid apart.  PAST: heads are accessed past the caches.
template <typename T, typename G, int GROUP, bool INTER, bool PAST> __global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 4 : 3) void k_rotate_grad(const Args a) {
    constexpr int N = Vec16<T>::N;
    constexpr int GROUPS = kThreads / GROUP;
    const int lane = threadIdx.x & (GROUP - 1), group = threadIdx.x / GROUP;
    const Pair p = pair_of<T, INTER>(lane, a.head_dim, a.rot_dim);
    const bool column = lane * 2 * N < a.head_dim;
    __shared__ float sums[kThreads / 64][2 * N * GROUP];
    for (int side = 0; side < 2; ++side) {
        const Side& s = a.side[side];
        if (!s.heads) continue;
        float wa[N], wb[N], ga[N], gb[N];
#pragma unroll
        for (int i = 0; i < N; ++i) { wa[i] = wb[i] = 1.f; ga[i] = gb[i] = 0.f; }
        if (column) { load_gain<T, G>(s.gain, p.ia, wa); load_gain<T, G>(s.gain, p.ib, wb); }
        const long long n = a.rows * s.heads;
        // every group of a wave makes the same number of rounds: the sums across lanes need all of them
        for (long long id0 = (long long)blockIdx.x * GROUPS; id0 < n; id0 += (long long)gridDim.x * GROUPS) {
            const long long id = id0 + group;
            const bool have = id < n, mine = have && column;
            const int row = have ? s.by_heads.quotient((int)id) : 0;
            const int h = have ? (int)id - row * s.heads : 0;
            const int b = a.by_tokens.quotient(row), t = row - b * a.tokens;
            Vec16<T> va{}, vb{}, da{}, db{};
            float c[N], sn[N];
            if (mine) {
                const T* x = static_cast<const T*>(s.x) + b * s.xs[0] + t * s.xs[1] + h * s.xs[2];
                const T* dy = static_cast<const T*>(s.dy) + b * s.ys[0] + t * s.ys[1] + h * s.ys[2];
                if (PAST) {
                    va.load_once(x + p.ia); vb.load_once(x + p.ib);
                    da.load_once(dy + p.ia); db.load_once(dy + p.ib);
                } else {
                    va.load(x + p.ia); vb.load(x + p.ib);
                    da.load(dy + p.ia); db.load(dy + p.ib);
                }
                load_angles<T, INTER>(a, p, position_of(a, b, t), c, sn);
            }
            float f[N], g[N], df[N], dg[N], sq = 0.f, dot = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                f[i] = va.get(i); g[i] = vb.get(i);
                df[i] = da.get(i); dg[i] = db.get(i);
                sq += f[i] * f[i] + g[i] * g[i];
            }
            if (mine) turn<T, INTER>(df, dg, c, sn, -1.f);
#pragma unroll
            for (int i = 0; i < N; ++i) dot += wa[i] * df[i] * f[i] + wb[i] * dg[i] * g[i];
            sq = lanes_sum<GROUP>(sq);
            dot = lanes_sum<GROUP>(dot);
            const float r = 1.f / sqrtf(sq * a.inv_dim + a.eps);
            const float k = dot * a.inv_dim * r * r;         // mean(w u) / r times r^2
            if (mine) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    ga[i] += df[i] * (f[i] * r);
                    gb[i] += dg[i] * (g[i] * r);
                    f[i] = r * (wa[i] * df[i] - f[i] * k);
                    g[i] = r * (wb[i] * dg[i] - g[i] * k);
                }
                T* dx = static_cast<T*>(s.y) + b * s.ds[0] + t * s.ds[1] + h * s.ds[2];
                if (PAST) {
                    store_values_past<N>(dx + p.ia, f);
                    store_values_past<N>(dx + p.ib, g);
                } else {
                    store_values<N>(dx + p.ia, f);
                    store_values<N>(dx + p.ib, g);
                }
            }
        }
        if (!a.part) continue;
#pragma unroll
        for (int i = 0; i < N; ++i) {
#pragma unroll
            for (int o = 32; o >= GROUP; o >>= 1) { ga[i] += __shfl_xor(ga[i], o); gb[i] += __shfl_xor(gb[i], o); }
        }
        __syncthreads();
        if ((threadIdx.x & 63) < GROUP && column) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                sums[threadIdx.x >> 6][p.ia + i] = ga[i];
                sums[threadIdx.x >> 6][p.ib + i] = gb[i];
            }
        }
        __syncthreads();
        float* out = a.part + ((long long)side * gridDim.x + blockIdx.x) * a.head_dim;
        for (int d = threadIdx.x; d < a.head_dim; d += kThreads) {
            float v = 0.f;
            for (int w = 0; w < kThreads / 64; ++w) v += sums[w][d];
            out[d] = v;
        }
    }
}

// ---- element by element: a wave a head -----------------------------------------------------------------
__device__ __forceinline__ void partners(const Args& a, int e, int* i, int* j) {
    *i = a.interleaved ? 2 * e : e;
    *j = a.interleaved ? 2 * e + 1 : e + a.rot_dim / 2;
}
template <typename T, typename G> __global__ __launch_bounds__(kThreads) void k_rotate_any(const Args a) {
    const int lane = threadIdx.x & 63;
    const long long id = a.first + (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    const int heads = a.side[0].heads + a.side[1].heads;
    if (id >= a.rows * heads) return;
    const unsigned row = (unsigned)id / (unsigned)heads;
    int h = (int)((unsigned)id - row * (unsigned)heads);
    const int b = (int)(row / (unsigned)a.tokens), t = (int)(row - (unsigned)b * (unsigned)a.tokens);
    const bool is_k = h >= a.side[0].heads;
    if (is_k) h -= a.side[0].heads;
    const Side& s = a.side[is_k];
    const T* x = static_cast<const T*>(s.x) + b * s.xs[0] + t * s.xs[1] + h * s.xs[2];
    T* y = static_cast<T*>(s.y) + b * s.ys[0] + t * s.ys[1] + h * s.ys[2];
    const G* gain = static_cast<const G*>(s.gain);
    float sum = 0.f;
    for (int d = lane; d < a.head_dim; d += 64) { const float v = to_f32(x[d]); sum += v * v; }
    const float r = 1.f / sqrtf(lanes_sum(sum) * a.inv_dim + a.eps);
    const long long pos = position_of(a, b, t);
    const int half = a.rot_dim / 2;
    for (int e = lane; e < half; e += 64) {
        int i, j;
        partners(a, e, &i, &j);
        const float c = pos < 0 ? __builtin_nanf("") : a.cos[pos * half + e], sn = pos < 0 ? 0.f : a.sin[pos * half + e];
        const float f = to_f32(x[i]) * r * (gain ? to_f32(gain[i]) : 1.f), g = to_f32(x[j]) * r * (gain ? to_f32(gain[j]) : 1.f);
        y[i] = from_f32<T>(f * c - g * sn);
        y[j] = from_f32<T>(g * c + f * sn);
    }
    for (int d = a.rot_dim + lane; d < a.head_dim; d += 64) y[d] = from_f32<T>(to_f32(x[d]) * r * (gain ? to_f32(gain[d]) : 1.f));
}
constexpr int kMaxDim = 1024;
template <typename T, typename G> __global__ __launch_bounds__(64) void k_rotate_grad_any(const Args a) {
    const int lane = threadIdx.x;
    __shared__ float dgain[kMaxDim];               // every element is one lane's
    const int half = a.rot_dim / 2, units = half + (a.head_dim - a.rot_dim);
    for (int side = 0; side < 2; ++side) {
        const Side& s = a.side[side];
        if (!s.heads) continue;
        const G* gain = static_cast<const G*>(s.gain);
        // unit e < half: a pair; unit half + k: element rot_dim + k
        for (int e = lane; e < units; e += 64) {
            int i = a.rot_dim + e - half, j = i;
            if (e < half) partners(a, e, &i, &j);
            dgain[i] = 0.f;
            dgain[j] = 0.f;
        }
        const long long n = a.rows * s.heads;
        for (long long id = blockIdx.x; id < n; id += gridDim.x) {
            const unsigned row = (unsigned)id / (unsigned)s.heads;
            const int h = (int)((unsigned)id - row * (unsigned)s.heads);
            const int b = (int)(row / (unsigned)a.tokens), t = (int)(row - (unsigned)b * (unsigned)a.tokens);
            const long long xo = b * s.xs[0] + t * s.xs[1] + h * s.xs[2], yo = b * s.ys[0] + t * s.ys[1] + h * s.ys[2];
            const long long po = b * s.ds[0] + t * s.ds[1] + h * s.ds[2];
            const T* x = static_cast<const T*>(s.x) + xo;
            const T* dy = static_cast<const T*>(s.dy) + yo;
            T* dx = static_cast<T*>(s.y) + po;
            const long long pos = position_of(a, b, t);
            float sq = 0.f, dot = 0.f;
            for (int pass = 0; pass < 2; ++pass) {
                float r = 0.f, k = 0.f;
                if (pass) {
                    r = 1.f / sqrtf(lanes_sum(sq) * a.inv_dim + a.eps);
                    k = lanes_sum(dot) * a.inv_dim * r * r;
                }
                for (int e = lane; e < units; e += 64) {
                    const bool turned = e < half;
                    int i = a.rot_dim + e - half, j = i;
                    if (turned) partners(a, e, &i, &j);
                    float f = to_f32(x[i]), df = to_f32(dy[i]), g = 0.f, dg = 0.f;
                    const float wi = gain ? to_f32(gain[i]) : 1.f, wj = gain ? to_f32(gain[j]) : 1.f;
                    if (turned) {
                        g = to_f32(x[j]); dg = to_f32(dy[j]);
                        const float c = pos < 0 ? __builtin_nanf("") : a.cos[pos * half + e], sn = pos < 0 ? 0.f : a.sin[pos * half + e];
                        const float u = df, v = dg;
                        df = u * c + v * sn;
                        dg = v * c - u * sn;
                    }
                    if (!pass) {
                        sq += f * f + g * g;
                        dot += wi * df * f + wj * dg * g;
                        continue;
                    }
                    dgain[i] += df * (f * r);
                    dx[i] = from_f32<T>(r * (wi * df - f * k));
                    if (turned) {
                        dgain[j] += dg * (g * r);
                        dx[j] = from_f32<T>(r * (wj * dg - g * k));
                    }
                }
            }
        }
        if (!a.part) continue;
        float* out = a.part + ((long long)side * gridDim.x + blockIdx.x) * a.head_dim;
        for (int e = lane; e < units; e += 64) {
            int i = a.rot_dim + e - half, j = i;
            if (e < half) partners(a, e, &i, &j);
            out[i] = dgain[i];
            if (j != i) out[j] = dgain[j];
        }
    }
}

// dgain[side][d] = sum over workgroups of part[side][.][d]: a workgroup takes 16 columns of a side, a sixty-fourth of the parts a
// thread, several of them on their way at a time.  A side without heads has no parts: its gradient is zero.
constexpr int kSumColumns = 16, kSumShares = 64;
__global__ __launch_bounds__(kSumColumns * kSumShares) void k_gain_sum(const float* part, int parts, int q_parts, int k_parts, int dim, float* dq, float* dk) {
    const int side = blockIdx.y, column = threadIdx.x % kSumColumns, share = threadIdx.x / kSumColumns, d = blockIdx.x * kSumColumns + column;
    float* out = side ? dk : dq;
    if (!out) return;
    __shared__ float sums[kSumShares][kSumColumns + 1];
    float v = 0.f;
    const int n = side ? k_parts : q_parts;
    if (d < dim) {
#pragma unroll 8
        for (int w = share; w < n; w += kSumShares) v += part[((long long)side * parts + w) * dim + d];
    }
    sums[share][column] = v;
    __syncthreads();
    for (int half = kSumShares / 2; half; half /= 2) {
        if (share < half) sums[share][column] += sums[share + half][column];
        __syncthreads();
    }
    if (share == 0 && d < dim) out[d] = sums[0][column];
}

// ---- host ----
asi_status check(const asi_qk_desc* d) {
    if (!d) return ASI_ERR_INVALID_ARG;
    if (!dtype_ok(d->dtype) || !dtype_ok(d->gain_dtype)) return ASI_ERR_UNSUPPORTED;
    if (d->batch < 0 || d->tokens < 0 || d->q_heads < 0 || d->k_heads < 0 || d->head_dim < 1) return ASI_ERR_INVALID_ARG;
    if (d->rot_dim < 0 || d->rot_dim % 2 || d->rot_dim > d->head_dim || (d->interleaved != 0 && d->interleaved != 1)) return ASI_ERR_INVALID_ARG;
    if (!(d->eps >= 0.f) || !std::isfinite(d->eps) || d->max_position < 0 || d->position_stride < 0) return ASI_ERR_INVALID_ARG;
    if (d->head_dim > kMaxDim || d->batch > 0x7fffffffLL || d->tokens > 0x7fffffffLL || d->q_heads > 65536 || d->k_heads > 65536) return ASI_ERR_UNSUPPORTED;
    const long long heads = (long long)d->q_heads + d->k_heads;
    if (heads > 0 && d->batch > 0 && d->tokens > 0x7fffffffLL / d->batch / heads) return ASI_ERR_UNSUPPORTED;
    return ASI_OK;
}
bool nothing(const asi_qk_desc* d) { return d->batch == 0 || d->tokens == 0 || d->q_heads + d->k_heads == 0; }

// Lanes of a head, 0 where vectors are not allowed.
int group_of(const asi_qk_desc* d, const Args& a, bool back) {
    const size_t es = dtype_size(d->dtype);
    const int n = (int)(16 / es);
    if (d->head_dim % (2 * n) || d->rot_dim % (2 * n) || d->head_dim / (2 * n) > 64) return 0;
    if (d->rot_dim && (!aligned(a.cos, 16) || !aligned(a.sin, 16))) return 0;
    for (const Side& s : a.side) {
        if (!s.heads) continue;
        if (!aligned(s.x, 16) || !aligned(s.y, 16) || !aligned(s.gain, 16) || (back && !aligned(s.dy, 16))) return 0;
        for (int k = 0; k < 3; ++k)
            if (s.xs[k] % n || s.ys[k] % n || (back && s.ds[k] % n)) return 0;
    }
    int g = 2;
    while (g < d->head_dim / (2 * n)) g *= 2;
    return g;
}
void fill(const asi_qk_desc* d, Args* a) {
    for (int k = 0; k < 3; ++k) {
        a->side[0].xs[k] = d->q_stride[k]; a->side[0].ys[k] = d->q_out_stride[k];
        a->side[1].xs[k] = d->k_stride[k]; a->side[1].ys[k] = d->k_out_stride[k];
        a->side[0].ds[k] = d->dq_stride[k]; a->side[1].ds[k] = d->dk_stride[k];
    }
    a->side[0].heads = d->q_heads;
    a->side[1].heads = d->k_heads;
    a->rows = d->batch * d->tokens;
    a->tokens = (int)d->tokens;
    a->head_dim = d->head_dim;
    a->rot_dim = d->rot_dim;
    a->interleaved = d->interleaved;
    a->position_stride = d->position_stride;
    a->max_position = d->max_position;
    a->eps = d->eps;
    a->inv_dim = 1.f / (float)d->head_dim;
    a->by_tokens.set(std::max(1, a->tokens));
    for (Side& s : a->side) s.by_heads.set(std::max(1, s.heads));
}
// Forward: how the heads of a token are taken
void set_parts(Args* a, int heads) {
    a->q_parts = (a->side[0].heads + heads - 1) / heads;
    a->parts = a->q_parts + (a->side[1].heads + heads - 1) / heads;
    a->by_parts.set(std::max(1, a->parts));
}
bool fits(const asi_qk_desc* d, const Args& a, bool back) {
    const size_t es = dtype_size(d->dtype);
    for (const Side& s : a.side) {
        if (!s.heads) continue;
        if (!s.x || !s.y || (back && !s.dy) || !aligned(s.x, es) || !aligned(s.y, es) || !aligned(s.dy, es)) return false;
        if (!aligned(s.gain, dtype_size(d->gain_dtype))) return false;
    }
    if (d->rot_dim && (!a.cos || !a.sin || !aligned(a.cos, 4) || !aligned(a.sin, 4))) return false;
    return aligned(a.positions, 8);
}
// Whether a group's loads and stores are whole lines of 128 bytes each.  Past the caches they are faster then (12003 tokens of 24 heads of
// 128 in fp32 91.0 -> 80.6 us, 16384 of 20 in bf16 60.4 -> 58.3) and slower otherwise, where the other part of a line comes later (20
// heads of 160 79.3 -> 83.0, of 64 in fp32 half turned 56.2 -> 60.4).
bool whole_lines(const Args& a, size_t size) {
    const int per = 2 * 128 / (int)size;
    return a.interleaved ? a.head_dim % per == 0 : a.rot_dim % per == 0 && (a.head_dim - a.rot_dim) % per == 0;
}
// Workgroups of the backward pass: as many as are resident at once, which is what registers leave room for (bf16, 16384 tokens of
// 18 heads of 128: 768 51 us, 1024, which the compiler has to spill for, 54; fp32, half of that: 1024 46 us, 768 48), fewer where
// that gives every group of lanes a head.  Scratch is planned for a head a group of 64 lanes.
int most_blocks(const asi_qk_desc* d) {
    const long long heads = d->batch * d->tokens * std::max(d->q_heads, d->k_heads);
    return (int)std::max(1LL, std::min(d->dtype == ASI_F32 ? 1024LL : 768LL, (heads + 3) / 4));
}
int grad_blocks(const asi_qk_desc* d, int group) {
    if (!group) return most_blocks(d);
    const long long heads = d->batch * d->tokens * std::max(d->q_heads, d->k_heads), groups = kThreads / group;
    return (int)std::max(1LL, std::min<long long>(most_blocks(d), (heads + groups - 1) / groups));
}

// Forward: f(grid) for as many of n at a time, `each` a workgroup, as a launch takes
template <typename F> void in_launches(long long n, int each, Args* a, F f) {
    const long long most = most_workgroups(kThreads) * each;
    for (a->first = 0; a->first < n; a->first += most) f(dim3((unsigned)((std::min(most, n - a->first) + each - 1) / each)));
}
template <typename T, typename G, int GROUP, int HEADS> void forward(Args a, hipStream_t st) {
    set_parts(&a, HEADS);
    in_launches(a.rows * a.parts, kThreads / GROUP, &a, [&](dim3 grid) {
        if (a.interleaved) hipLaunchKernelGGL((k_rotate<T, G, GROUP, HEADS, true>), grid, kThreads, 0, st, a);
        else hipLaunchKernelGGL((k_rotate<T, G, GROUP, HEADS, false>), grid, kThreads, 0, st, a);
    });
}
template <typename T, typename G, int GROUP, bool INTER> void backward(const Args& a, int blocks, hipStream_t st) {
    constexpr bool lines = GROUP * 16 >= 128;         // a vector of each lane of a group fills a line
    if (lines && whole_lines(a, sizeof(T))) hipLaunchKernelGGL((k_rotate_grad<T, G, GROUP, INTER, lines>), dim3(blocks), kThreads, 0, st, a);
    else hipLaunchKernelGGL((k_rotate_grad<T, G, GROUP, INTER, false>), dim3(blocks), kThreads, 0, st, a);
}
template <typename T, typename G, int GROUP> void go(const Args& a, bool back, int blocks, hipStream_t st) {
    // two heads a lane share the angles and gains (8 x 512 tokens of 36 heads of 64 9.9 us, one head 11.0, four 10.8); where one
    // head a lane does not fill the chip the shorter chain counts (8 tokens of these heads 3.4 us, two 3.8)
    const long long waves = a.rows * (a.side[0].heads + a.side[1].heads) * GROUP / 64;
    if (!back && waves > 4096) forward<T, G, GROUP, 2>(a, st);
    else if (!back) forward<T, G, GROUP, 1>(a, st);
    else if (a.interleaved) backward<T, G, GROUP, true>(a, blocks, st);
    else backward<T, G, GROUP, false>(a, blocks, st);
}
template <typename T, typename G> void go(int group, const Args& a, bool back, int blocks, hipStream_t st) {
    switch (group) {
        case 2: go<T, G, 2>(a, back, blocks, st); break;
        case 4: go<T, G, 4>(a, back, blocks, st); break;
        case 8: go<T, G, 8>(a, back, blocks, st); break;
        case 16: go<T, G, 16>(a, back, blocks, st); break;
        case 32: go<T, G, 32>(a, back, blocks, st); break;
        case 64: go<T, G, 64>(a, back, blocks, st); break;
        default:
            if (back) {
                hipLaunchKernelGGL((k_rotate_grad_any<T, G>), dim3(blocks), 64, 0, st, a);
            } else {
                Args b = a;
                in_launches(a.rows * (a.side[0].heads + a.side[1].heads), kThreads / 64, &b,
                            [&](dim3 grid) { hipLaunchKernelGGL((k_rotate_any<T, G>), grid, kThreads, 0, st, b); });
            }
    }
}
void go(const asi_qk_desc* d, const Args& a, int group, bool back, int blocks, hipStream_t st) {
    if (d->dtype == ASI_F32) {
        if (d->gain_dtype == ASI_F32) go<float, float>(group, a, back, blocks, st);
        else go<float, bf16_t>(group, a, back, blocks, st);
    } else {
        if (d->gain_dtype == ASI_F32) go<bf16_t, float>(group, a, back, blocks, st);
        else go<bf16_t, bf16_t>(group, a, back, blocks, st);
    }
}

}  // namespace
}  // namespace asi

using namespace asi;

extern "C" {

asi_status asi_qk_norm_rotate(const asi_qk_desc* desc, const void* q, const void* k, const void* q_gain, const void* k_gain,
                              const int64_t* positions, const float* cos, const float* sin, void* q_out, void* k_out,
                              asi_stream_t stream) {
    if (asi_status why = check(desc); why != ASI_OK) return why;
    if (nothing(desc)) return ASI_OK;
    Args a{};
    fill(desc, &a);
    a.side[0].x = q; a.side[0].gain = q_gain; a.side[0].y = q_out;
    a.side[1].x = k; a.side[1].gain = k_gain; a.side[1].y = k_out;
    a.positions = positions; a.cos = cos; a.sin = sin;
    if (!fits(desc, a, false)) return ASI_ERR_INVALID_ARG;
    go(desc, a, group_of(desc, a, false), false, 0, static_cast<hipStream_t>(stream));
    return launched();
}

size_t asi_qk_norm_rotate_grad_workspace_bytes(const asi_qk_desc* desc) {
    if (check(desc) != ASI_OK || nothing(desc)) return 0;
    return round256((size_t)2 * most_blocks(desc) * desc->head_dim * sizeof(float));
}

asi_status asi_qk_norm_rotate_grad(const asi_qk_desc* desc, const void* q, const void* k, const void* q_gain,
                                   const void* k_gain, const int64_t* positions, const float* cos, const float* sin,
                                   const void* grad_q, const void* grad_k, void* dq, void* dk, float* dq_gain,
                                   float* dk_gain, void* ws, size_t ws_bytes, asi_stream_t stream) {
    if (asi_status why = check(desc); why != ASI_OK) return why;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (!aligned(dq_gain, 4) || !aligned(dk_gain, 4)) return ASI_ERR_INVALID_ARG;
    Args a{};
    fill(desc, &a);
    a.side[0].x = q; a.side[0].gain = q_gain; a.side[0].y = dq; a.side[0].dy = grad_q;
    a.side[1].x = k; a.side[1].gain = k_gain; a.side[1].y = dk; a.side[1].dy = grad_k;
    a.positions = positions; a.cos = cos; a.sin = sin;
    const bool empty = nothing(desc);
    if (!empty && !fits(desc, a, true)) return ASI_ERR_INVALID_ARG;
    const int group = empty ? 0 : group_of(desc, a, true);
    const int blocks = empty ? 0 : grad_blocks(desc, group);
    const bool gains = dq_gain || dk_gain;
    if (!empty) {
        if (gains) {
            if (!ws || !aligned(ws, 256) || ws_bytes < asi_qk_norm_rotate_grad_workspace_bytes(desc)) return ASI_ERR_WORKSPACE;
            a.part = static_cast<float*>(ws);
        }
        go(desc, a, group, true, blocks, st);
    }
    if (!gains) return empty ? ASI_OK : launched();
    // also of a side without heads, or a call without tokens: the sum of nothing
    const dim3 grid((unsigned)((desc->head_dim + kSumColumns - 1) / kSumColumns), 2);
    hipLaunchKernelGGL(k_gain_sum, grid, kSumColumns * kSumShares, 0, st, a.part, blocks, desc->q_heads ? blocks : 0, desc->k_heads ? blocks : 0, desc->head_dim, dq_gain, dk_gain);
    return launched();
}

}  // extern "C"
