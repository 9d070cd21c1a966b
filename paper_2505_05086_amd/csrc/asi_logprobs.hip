// Log probabilities of given tokens with entropy and the top alternatives, and their gradient (include/asi_lm.h).
//
// With m the largest logit of a row, d_i = x_i - m and e_i = exp(scale d_i):
//     s = sum e_i,  w = sum d_i e_i;   logprob = scale d_target - log s;   entropy = log s - scale w / s
// Differences from the row's largest logit keep the digits that z - lse would lose where logits are large.
//
// Forward: a workgroup takes a row in one pass, several vectors a thread at a time; every thread keeps a running largest logit
// and the sums relative to it.
// Top alternatives: each wave takes the c largest of its threads' largest logits, c = ceil(top / waves) + 1; the `top`-th of all of
// those is a bound that at least `top` logits reach.  Only the vectors of threads whose largest may reach it are looked at again, shared by all threads,
// and hand over the logits that reach it, a few more than wanted; of these each finds its place by counting the ones before
// it.  Rows where too many reach the bound (many equal logits) are searched `top` times instead.
//
// Few long rows are cut into parts, a workgroup each, which leave their sums and alternatives in scratch for a second kernel to join in
// the order of the parts.
//
// Gradient: a row is kept in registers between the pass that sums and the one that writes, so that it is read once and written once;
// of rows too long for that the rest is read again.
//
// Bound by memory: 1023 x 50001 in fp32 with 5 alternatives 39.5 us (5.2 TB/s), 4096 x 32000 in bf16 with its gradient 94 us (5.6 TB/s);
// few rows by the chain of one workgroup: 8 x 32000 in bf16 5.6 us, with 20 alternatives 10.4.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "asi_lm_device.h"

namespace asi {
namespace {

constexpr float kLowest = -3.402823466e+38f;     // stands for a thread that has seen no logit above -infinity
// The scale as the kernels use it.
struct Scale {
    float c;             // exp(scale d) = 2^(c d)
    float far;           // differences are not let below this, where 2^(c d) is 0 and its products with d and c d are, not NaN
};
constexpr float kLeastScale = 1e-20f, kMostScale = 1e20f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A row as 16-byte vectors from its first aligned address on, with up to N - 1 elements before them and behind.
template <typename T> struct RowView {
    const T* x;
    int head, nvec, tail_at, n;
    __device__ __forceinline__ RowView(const T* row, int vocab) {
        constexpr int N = Vec16<T>::N;
        x = row;
        n = vocab;
        head = min((int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(T), vocab);
        nvec = (vocab - head) / N;
        tail_at = head + nvec * N;
    }
    // the element of this thread that no vector holds: index, or -1
    __device__ __forceinline__ int loose(int tid) const {
        if (tid < head) return tid;
        const int i = tail_at + tid - head;
        return tid >= head && i < n ? i : -1;
    }
    __device__ __forceinline__ const T* vec(int v) const { return x + head + v * Vec16<T>::N; }
    __device__ __forceinline__ int index(int v) const { return head + v * Vec16<T>::N; }
};

struct Sums {
    float m, s, w;
};
// Sums of another part joined to these: both relative to the larger of the two largest logits.  Products are rounded by themselves, so
// that a and b may change places and all threads of a row get the same sums.
__device__ __forceinline__ Sums joined(const Sums& a, const Sums& b, const Scale& k) {
#pragma clang fp contract(off)
    Sums r;
    r.m = fmaxf(a.m, b.m);
    const float da = max_nan(a.m - r.m, k.far), db = max_nan(b.m - r.m, k.far);
    const float fa = exp2_fast(da * k.c), fb = exp2_fast(db * k.c);
    r.s = a.s * fa + b.s * fb;
    r.w = fa * (a.w + da * a.s) + fb * (b.w + db * b.s);
    return r;
}
template <int WIDTH> __device__ __forceinline__ Sums over_lanes(Sums a, const Scale& k) {
#pragma unroll
    for (int o = WIDTH / 2; o; o >>= 1) {
        Sums b;
        b.m = __shfl_xor(a.m, o); b.s = __shfl_xor(a.s, o); b.w = __shfl_xor(a.w, o);
        a = joined(a, b, k);
    }
    return a;
}
// Over the workgroup; every thread gets the result.
template <int THREADS> __device__ __forceinline__ Sums over_workgroup(Sums a, const Scale& k, Sums* scratch) {
    constexpr int W = THREADS / 64;
    a = over_lanes<64>(a, k);
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = a;
    __syncthreads();
    return over_lanes<W>(scratch[threadIdx.x & (W - 1)], k);
}
// Keeps the instructions of one vector together: interleaving several costs more registers than it saves time.
__device__ __forceinline__ void one_at_a_time() { __builtin_amdgcn_sched_barrier(0); }
// Has the bf16 values of a vector taken apart anew from here on, rather than kept as twice the registers
__device__ __forceinline__ void taken_apart_anew(Vec16<float>*) {}
__device__ __forceinline__ void taken_apart_anew(Vec16<bf16_t>* v) {
    asm volatile("" : "+v"(v->raw.x), "+v"(v->raw.y), "+v"(v->raw.z), "+v"(v->raw.w));
}
// One more logit of a thread
__device__ __forceinline__ void take_one(Sums* a, float x, const Scale& k) {
    Sums b{x > kLowest ? x : kLowest, 0.f, 0.f};
    const float d = max_nan(x - b.m, k.far);
    b.s = exp2_fast(d * k.c);
    b.w = d * b.s;
    *a = joined(*a, b, k);
}
template <typename T> __device__ __forceinline__ float largest(const Vec16<T>& v) {
    float m = v.get(0);
#pragma unroll
    for (int i = 1; i < Vec16<T>::N; ++i) m = fmaxf(m, v.get(i));
    return m;
}
// a vector of nothing but -infinity
template <typename T> __device__ __forceinline__ void set_nothing(Vec16<T>* v) {
    const uint32_t w = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    v->raw = make_uint4(w, w, w, w);
}
// Vectors v[0 .. U) of which the first `have` are the thread's own or nothing; `have` is the same in all threads
template <typename T, int U> __device__ __forceinline__ void take(Sums* a, Vec16<T>* v, int have, const Scale& k) {
    float m = a->m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (u < have) m = fmaxf(m, largest(v[u]));
        if (U > 2) one_at_a_time();
    }
    const float shift = max_nan(a->m - m, k.far), f = exp2_fast(shift * k.c);
    a->w = f * (a->w + shift * a->s);
    a->s *= f;
    a->m = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (u < have) {
            if (U > 4) taken_apart_anew(&v[u]);       // up to 4 vectors leave room for their values
#pragma unroll
            for (int i = 0; i < Vec16<T>::N; ++i) {
                const float d = max_nan(v[u].get(i) - m, k.far), e = exp2_fast(d * k.c);
                a->s += e;
                a->w += d * e;
            }
        }
        if (U > 2) one_at_a_time();
    }
}
// Vectors first, first + threads, ... of the thread, U of them; behind the row's end nothing.  Returns how many some thread has.
// AGAIN: they will be read again.
template <typename T, int U, bool AGAIN = false> __device__ __forceinline__ int load(const RowView<T>& r, int first, int threads, Vec16<T>* v) {
    auto one = [&](int u) {
        if (AGAIN) v[u].load(r.vec(first + u * threads));
        else v[u].load_once(r.vec(first + u * threads));
    };
    const int base = first - (int)threadIdx.x;
    if (base + threads * U <= r.nvec) {
#pragma unroll
        for (int u = 0; u < U; ++u) one(u);
        return U;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (first + u * threads < r.nvec) one(u);
        else set_nothing(&v[u]);
    }
    return (max(0, r.nvec - base) + threads - 1) / threads;
}

struct Values {
    float lse, logprob, entropy, m, ls;       // m: the largest logit; ls: log s, -infinity without a logit above -infinity
};
// z - lse of a logit x
__device__ __forceinline__ float logprob_of(float x, float m, float ls, float scale) {
    if (x == -__builtin_inff() && ls == ls) return x;         // also where ls is -infinity
    const float d = x - m;
    // finite logits farther apart than fp32 reaches: both scaled first
    return d == -__builtin_inff() ? fmaf(x, scale, -m * scale) - ls : fmaf(d, scale, -ls);
}
// target < 0: none
template <typename T> __device__ __forceinline__ Values values_of(const Sums& a, const T* row, long long target, int vocab, long long ignore, float scale) {
    Values v;
    const float inf = __builtin_inff(), nan = __builtin_nanf("");
    const bool empty = a.s == 0.f;                // no logit above -infinity
    const float ls = logf(a.s);
    v.m = a.m;
    v.ls = ls;
    v.lse = empty ? -inf : a.m * scale + ls;
    v.entropy = empty ? 0.f : ls - scale * (a.w / a.s);
    if (target == ignore) v.logprob = 0.f;
    else if (target < 0 || target >= vocab) v.logprob = nan;
    else v.logprob = logprob_of(to_f32(row[target]), a.m, ls, scale);
    return v;
}

struct Args {
    const void* x;
    const int64_t* targets;
    float* logprob;
    float* entropy;
    float* lse;
    float* top_logprob;
    int64_t* top_index;
    long long stride, ignore;
    int vocab, top;
    float scale;
    Scale k;
    // rows in parts of `part` logits: [row][part] sums, [row][part][top] keys of alternatives, 0 where there are fewer
    int parts, part;
    Sums* sums;
    unsigned long long* keys;
};

// ---- top alternatives -----------------------------------------------------------------------------------------
// Logits as whole numbers in their order: NaN above everything, -0 equal to 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// An alternative: larger is earlier.  Equal logits: the lower index is.
__device__ __forceinline__ unsigned long long rank_key(float x, int index) { return (unsigned long long)order_of(x) << 32 | (uint32_t)~index; }
__device__ __forceinline__ unsigned long long lanes_max64(unsigned long long k) {
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        const unsigned long long other = __shfl_xor(k, o);
        k = other > k ? other : k;
    }
    return k;
}
__device__ __forceinline__ float logit_of(unsigned long long key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return o == 0xffffffffu ? __builtin_nanf("") : __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
constexpr int kCandidates = 1024;
constexpr int kBounds = 128;          // at least waves * (ceil(ASI_LOGPROB_MAX_TOP / waves) + 1)
template <int THREADS> struct TopScratch {
    unsigned long long key[kCandidates];
    unsigned long long wave[THREADS / 64];
    uint32_t largest[kBounds];        // of the threads of each wave
    int who[THREADS];                 // threads whose vectors are looked at again
    int count, many;
};
__device__ __forceinline__ void write_alternative(const Args& a, long long row, const Values& v, int place, unsigned long long key) {
    a.top_logprob[row * a.top + place] = logprob_of(logit_of(key), v.m, v.ls, a.scale);
    a.top_index[row * a.top + place] = (int)~(uint32_t)key;
}
// The order of the largest of a thread's vectors, 0 without any: `least` is one that is there, none is above `upto`.
struct Most {
    uint32_t least, upto;
};
// write(place, key) for the `top` largest of the row's logits, top <= the row's length.  `index0`: of the row's first logit.
template <typename T, int THREADS, typename F>
__device__ __forceinline__ void find_top(const RowView<T>& r, const Most& most, int top, int index0, TopScratch<THREADS>* sc, F write) {
    constexpr int W = THREADS / 64, N = Vec16<T>::N;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // Waves whose threads do not all have a vector bound nothing; where there is no other, everything is handed over (less than
    // kCandidates then).
    const int full = min(W, r.nvec / 64);
    const int c = full ? min(64, (top + full - 1) / full + 1) : 0;
    static_assert(W <= 16 && W * (ASI_LOGPROB_MAX_TOP / W + 2) <= kBounds, "room for the waves' largest");
    if (wave < full) {
        uint32_t left = most.least;
        for (int got = 0; got < c;) {
            const uint32_t m = wave_max(left);
            const unsigned long long with = __ballot(left == m);
            if (left == m) {
                const int at = got + __builtin_amdgcn_mbcnt_hi((uint32_t)(with >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)with, 0u));
                if (at < c) sc->largest[wave * c + at] = m;
                left = 0;
            }
            got += __popcll(with);
        }
    }
    if (threadIdx.x == 0) sc->count = sc->many = 0;
    __syncthreads();
    uint32_t bound = 0;
    if (full) {
        // every wave finds the `top`-th of them: the one that fewer than `top` are above and at least `top` reach
        const int n = full * c;                   // at least `top`
        uint32_t found = 0;
        for (int half = 0; half < n; half += 64) {
            const uint32_t mine = half + lane < n ? sc->largest[half + lane] : 0u;
            int above = 0, reach = 0;
#pragma unroll 8
            for (int k = 0; k < n; ++k) {
                const uint32_t o = sc->largest[k];
                above += o > mine;
                reach += o >= mine;
            }
            if (half + lane < n && above < top && reach >= top) found = mine;
        }
        bound = wave_max(found);
    }
    auto hand_over = [&](float x, int i) {
        if (order_of(x) >= bound) {
            const int at = atomicAdd(&sc->count, 1);
            if (at < kCandidates) sc->key[at] = rank_key(x, index0 + i);
        }
    };
    if (most.upto >= bound && most.upto) sc->who[atomicAdd(&sc->many, 1)] = threadIdx.x;
    if (const int l = r.loose(threadIdx.x); l >= 0) hand_over(to_f32(r.x[l]), l);
    __syncthreads();
    {
        const int each = (r.nvec + THREADS - 1) / THREADS, all = sc->many * each;
#pragma unroll 1
        for (int item = threadIdx.x; item < all; item += THREADS) {
            const int k = item / each, v = sc->who[k] + (item - k * each) * THREADS;
            if (v < r.nvec) {
                Vec16<T> raw;
                raw.load(r.vec(v));
#pragma unroll
                for (int i = 0; i < N; ++i) hand_over(raw.get(i), r.index(v) + i);
            }
        }
    }
    __syncthreads();
    const int n = sc->count;
    if (n <= kCandidates) {
        for (int i = threadIdx.x; i < n; i += THREADS) {
            const unsigned long long key = sc->key[i];
            int before = 0;
#pragma unroll 8
            for (int k = 0; k < n; ++k) before += sc->key[k] > key;
            if (before < top) write(before, key);
        }
        return;
    }
    unsigned long long last = 0;                  // of the place before
    for (int place = 0; place < top; ++place) {
        unsigned long long best = 0;
        auto look = [&](float x, int i) {
            const unsigned long long key = rank_key(x, index0 + i);
            if ((place == 0 || key < last) && key > best) best = key;      // NaN at index 0 has the largest key there is
        };
        if (const int l = r.loose(threadIdx.x); l >= 0) look(to_f32(r.x[l]), l);
#pragma unroll 1
        for (int v = threadIdx.x; v < r.nvec; v += THREADS) {
            Vec16<T> raw;
            raw.load(r.vec(v));
#pragma unroll
            for (int i = 0; i < N; ++i) look(raw.get(i), r.index(v) + i);
        }
        best = lanes_max64(best);
        __syncthreads();
        if (lane == 0) sc->wave[wave] = best;
        __syncthreads();
        best = sc->wave[0];
        for (int k = 1; k < W; ++k) best = sc->wave[k] > best ? sc->wave[k] : best;
        last = best;
        if (threadIdx.x == 0) write(place, best);
    }
}

// ---- forward ----------------------------------------------------------------------------------------------------
// The largest of a thread's vectors where their sums are `a`
__device__ __forceinline__ Most most_of(const Sums& a) {
    const float inf = __builtin_inff();
    if (a.s != a.s) return {a.m == inf ? order_of(inf) : 0xffffffffu, 0xffffffffu};      // +infinity makes the sum NaN, beside NaN or without
    const uint32_t o = order_of(a.s == 0.f ? -inf : a.m);
    return {o, o};
}
__device__ __forceinline__ void write_values(const Args& a, long long row, const Values& v) {
    if (a.logprob) a.logprob[row] = v.logprob;
    if (a.entropy) a.entropy[row] = v.entropy;
    if (a.lse) a.lse[row] = v.lse;
}
// U: vectors that a thread loads at a time.  SPLIT: a part of the row.
template <typename T, int THREADS, int U, bool TOP, bool SPLIT> __global__ __launch_bounds__(THREADS) void k_logprobs(const Args a) {
    __shared__ Sums scratch[THREADS / 64];
    const long long row = SPLIT ? blockIdx.x / a.parts : blockIdx.x;
    const int part = SPLIT ? (int)(blockIdx.x - row * a.parts) : 0, index0 = SPLIT ? part * a.part : 0;
    const T* x = static_cast<const T*>(a.x) + row * a.stride;
    const int n = SPLIT ? min(a.part, a.vocab - index0) : a.vocab;
    const RowView<T> r(x + index0, n);
    const Scale k = a.k;
    Sums acc{kLowest, 0.f, 0.f};
    Vec16<T> v[U];
    for (int base = 0; base < r.nvec; base += THREADS * U) {
        const int have = load<T, U>(r, base + threadIdx.x, THREADS, v);
        take<T, U>(&acc, v, have, k);
    }
    const Most most = TOP && (int)threadIdx.x < r.nvec ? most_of(acc) : Most{0u, 0u};
    if (const int l = r.loose(threadIdx.x); l >= 0) take_one(&acc, to_f32(r.x[l]), k);
    const Sums all = over_workgroup<THREADS>(acc, k, scratch);
    Values val{};
    if constexpr (SPLIT) {
        if (threadIdx.x == 0) a.sums[blockIdx.x] = all;
    } else {
        const long long target = a.targets ? a.targets[row] : a.ignore;
        val = values_of(all, x, target, a.vocab, a.ignore, a.scale);
        if (threadIdx.x == 0) write_values(a, row, val);
    }
    if constexpr (TOP) {
        __shared__ TopScratch<THREADS> top;
        if constexpr (SPLIT) {
            unsigned long long* keys = a.keys + (long long)blockIdx.x * a.top;
            const int want = min(a.top, n);
            find_top<T, THREADS>(r, most, want, index0, &top, [&](int place, unsigned long long key) { keys[place] = key; });
            for (int i = want + threadIdx.x; i < a.top; i += THREADS) keys[i] = 0;
        } else {
            find_top<T, THREADS>(r, most, a.top, 0, &top, [&](int place, unsigned long long key) { write_alternative(a, row, val, place, key); });
        }
    }
}
// The parts of a row, a workgroup a row
constexpr int kMaxParts = 16, kJoinThreads = 256;
template <typename T> __global__ __launch_bounds__(kJoinThreads) void k_join_parts(const Args a) {
    __shared__ unsigned long long key[kMaxParts * ASI_LOGPROB_MAX_TOP];
    const long long row = blockIdx.x;
    const int n = a.parts * a.top;
    for (int i = threadIdx.x; i < n; i += kJoinThreads) key[i] = a.keys[row * n + i];
    const int p = threadIdx.x & (kMaxParts - 1);
    Sums all{kLowest, 0.f, 0.f};
    if (p < a.parts) all = a.sums[row * a.parts + p];
    all = over_lanes<kMaxParts>(all, a.k);
    const long long target = a.targets ? a.targets[row] : a.ignore;
    const Values val = values_of(all, static_cast<const T*>(a.x) + row * a.stride, target, a.vocab, a.ignore, a.scale);
    if (threadIdx.x == 0) write_values(a, row, val);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kJoinThreads) {
        const unsigned long long mine = key[i];
        int before = 0;
#pragma unroll 8
        for (int k = 0; k < n; ++k) before += key[k] > mine;
        if (mine && before < a.top) write_alternative(a, row, val, before, mine);
    }
}

// ---- gradient ---------------------------------------------------------------------------------------------------
struct GradArgs {
    const void* x;
    void* dx;
    const int64_t* targets;
    const float* a;
    const float* b;
    float* logprob;
    float* entropy;
    long long stride, grad_stride, ignore;
    int vocab;
    float scale;
    Scale k;
};
// KEEP: vectors that a thread keeps in registers.  REST: the row is longer, its rest is read again.
template <typename T, int THREADS, int KEEP, bool REST> __global__ __launch_bounds__(THREADS) void k_logprobs_grad(const GradArgs g) {
    constexpr int N = Vec16<T>::N;
    __shared__ Sums scratch[THREADS / 64];
    const long long row = blockIdx.x;
    const T* x = static_cast<const T*>(g.x) + row * g.stride;
    T* dx = static_cast<T*>(g.dx) + row * g.grad_stride;
    const RowView<T> r(x, g.vocab);
    const Scale s = g.k;
    const int l = r.loose(threadIdx.x);
    const float loose = l >= 0 ? to_f32(x[l]) : 0.f;
    const long long target = g.targets ? g.targets[row] : g.ignore;
    Sums acc{kLowest, 0.f, 0.f};
    Vec16<T> kept[KEEP], again[2];
    const int have = load<T, KEEP>(r, threadIdx.x, THREADS, kept);
    take<T, KEEP>(&acc, kept, have, s);
    if constexpr (REST) {
        for (int base = KEEP * THREADS; base < r.nvec; base += 2 * THREADS) {
            const int more = load<T, 2, true>(r, base + threadIdx.x, THREADS, again);
            take<T, 2>(&acc, again, more, s);
        }
    }
    if (l >= 0) take_one(&acc, loose, s);
    const Sums all = over_workgroup<THREADS>(acc, s, scratch);
    const Values val = values_of(all, x, target, g.vocab, g.ignore, g.scale);
    if (threadIdx.x == 0) {
        if (g.logprob) g.logprob[row] = val.logprob;
        if (g.entropy) g.entropy[row] = val.entropy;
    }
    const bool given = target != g.ignore, in_range = target >= 0 && target < g.vocab;
    const float wa = given && g.a ? g.a[row] : 0.f, wb = g.b ? g.b[row] : 0.f;
    const bool empty = all.s == 0.f;
    // dx_i = scale (a delta_i - p_i (a + b (log p_i + entropy))),  log p_i = scale d_i - log s:  e_i (k0 + k1 c d_i) with these.  The scale
    // times d_i is within what has a probability, the scale's square need not be within fp32.
    const float inv = empty ? 0.f : 1.f / all.s, ls = empty ? 0.f : logf(all.s);
    const float bad = given && !in_range ? __builtin_nanf("") : 0.f;
    const float k0 = -g.scale * inv * (wa + wb * (val.entropy - ls)) + bad, k1 = -g.scale * inv * wb * kLn2;
    const float hot = empty ? 0.f : g.scale * wa;
    auto grad = [&](float v) {
        const float d = max_nan(v - all.m, s.far) * s.c;
        return exp2_fast(d) * (k0 + k1 * d);
    };
    // dx's rows need not lie as x's do
    const bool vec = ((reinterpret_cast<uintptr_t>(dx + r.head)) & 15) == 0;
    auto write = [&](const Vec16<T>& raw, int v) {
        float f[N];
        const int i0 = r.index(v);
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = grad(raw.get(i));
        if (vec) {
            store_values_past<N>(dx + i0, f);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) dx[i0 + i] = from_f32<T>(f[i]);
        }
    };
    // Of the target there is more to say: its thread writes it once more, behind its vector.
    const int at = given && in_range ? (int)target : -1;
    const float of_target = at >= 0 ? to_f32(x[at]) : 0.f;
    __syncthreads();                              // before dx, which may be x, is written every thread has read its target
    if (l >= 0) dx[l] = from_f32<T>(grad(loose));
#pragma unroll
    for (int k = 0; k < KEEP; ++k) {
        const int v = threadIdx.x + k * THREADS;
        if (v < r.nvec) write(kept[k], v);
        one_at_a_time();
    }
    if constexpr (REST) {
        for (int base = KEEP * THREADS; base < r.nvec; base += 2 * THREADS) {
            load<T, 2>(r, base + threadIdx.x, THREADS, again);
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (const int v = base + k * THREADS + (int)threadIdx.x; v < r.nvec) write(again[k], v);
        }
    }
    const bool in_vector = at >= r.head && at < r.tail_at;
    if (at >= 0 && (in_vector ? (at - r.head) / N % THREADS == (int)threadIdx.x : at == l)) dx[at] = from_f32<T>(grad(of_target) + hot);
}

// ---- host ----
Scale scale_of(const asi_logprob_desc* d) {
    const float c = d->scale * kLog2e;
    return {c, -300.f / c};                       // 2^-300 is below the least number of fp32
}
asi_status check(const asi_logprob_desc* d) {
    if (!d) return ASI_ERR_INVALID_ARG;
    if (!dtype_ok(d->dtype)) return ASI_ERR_UNSUPPORTED;
    if (d->rows < 0 || d->vocab < 1 || d->row_stride < d->vocab || d->reserved) return ASI_ERR_INVALID_ARG;
    if (!(d->scale > 0.f) || !std::isfinite(d->scale)) return ASI_ERR_INVALID_ARG;
    if (d->scale < kLeastScale || d->scale > kMostScale) return ASI_ERR_UNSUPPORTED;
    if (d->rows > 0x7fffffffLL || d->vocab > (1LL << 28)) return ASI_ERR_UNSUPPORTED;
    return ASI_OK;
}
// Parts of a row: 1, or of long rows too few to fill the chip as many as leave each 1024 vectors, and the joining kernel no more than
// about 160 alternatives to compare with each other.  Measured: 8 rows of 128000 in bf16 without alternatives 11.3 us in one part, 6.0
// in 15, with 20 alternatives 16.1 in one, 18.3 in 15, 12.6 in 7; 5 rows of 195072 in fp32 17.9 and 8.3; 64 of
// 33000 in fp32 with 20 alternatives 11.0 and 13.1, without them 66000 in bf16 8.2 and 6.0.
int parts_of(const asi_logprob_desc* d) {
    const long long nvec = d->vocab / (int)(16 / dtype_size(d->dtype));
    if (nvec < (d->top ? 12288 : 8192) || d->rows > 64) return 1;
    const long long joined = d->top ? std::max(2, 160 / d->top) : kMaxParts;
    return (int)std::max(1LL, std::min<long long>({kMaxParts, joined, nvec / 1024, 512 / std::max<int64_t>(1, d->rows)}));
}
// f(first row, rows) for as many rows at a time as a launch of 1024 threads each takes
template <typename F> void in_launches(long long rows, F f) {
    constexpr long long most = most_workgroups(1024);
    for (long long first = 0; first < rows; first += most) f(first, (unsigned)std::min(most, rows - first));
}
template <typename P> P* behind(P* p, long long n) { return p ? p + n : nullptr; }
size_t sums_bytes(const asi_logprob_desc* d, int parts) { return round256((size_t)d->rows * parts * sizeof(Sums)); }

template <typename T, int THREADS, int U, bool SPLIT> void forward(const Args& a, unsigned blocks, hipStream_t st) {
    if (a.top) hipLaunchKernelGGL((k_logprobs<T, THREADS, U, true, SPLIT>), dim3(blocks), THREADS, 0, st, a);
    else hipLaunchKernelGGL((k_logprobs<T, THREADS, U, false, SPLIT>), dim3(blocks), THREADS, 0, st, a);
}
// Threads of a row: all that one compute unit has where there are few rows, fewer where rows overlap or are short (2902 x 31898 in fp32
// with 5 alternatives: 1024 threads 103.7 us, 512 70.3, 256 71.4; 247 x 10748 in bf16 with 20: 1024 10.3, 256 8.5)
template <typename T> void forward(const Args& a, unsigned rows, hipStream_t st) {
    const int nvec = a.vocab / Vec16<T>::N;
    if (a.parts > 1) {
        forward<T, 512, 4, true>(a, rows * a.parts, st);
        hipLaunchKernelGGL(k_join_parts<T>, dim3(rows), kJoinThreads, 0, st, a);
    } else if (nvec <= 256 || (nvec <= 1024 && rows > 2048)) {
        // a wave a row needs no barrier; of longer rows enough waves (8081 x 6302 in bf16 27.5 us by four waves a row, 22.0 by one)
        forward<T, 64, 4, false>(a, rows, st);
    } else if (nvec <= 2048) {
        forward<T, 256, 4, false>(a, rows, st);
    } else if (rows > 256) {
        forward<T, 512, 4, false>(a, rows, st);
    } else {
        forward<T, 1024, 4, false>(a, rows, st);
    }
}
// Threads of a row, and vectors that each keeps: as few as leave a compute unit several workgroups, of which some load while others write
// (4096 x 32000 in bf16: 256 threads that keep 16 114.5 us, 512 that keep 8 105.2, 1024 that keep 4 113.1; 1324 x 41616 in fp32: 512 that keep 24
// 107.1, 1024 that keep 16 110.7; 1142 x 76156 in fp32: 1024 that keep 24 167.7, 16 and the rest read again 171.3, all of it 209)
template <typename T> void backward(const GradArgs& g, unsigned rows, hipStream_t st) {
    const int nvec = g.vocab / Vec16<T>::N;
#define ASI_GRAD(THREADS, KEEP, REST) hipLaunchKernelGGL((k_logprobs_grad<T, THREADS, KEEP, REST>), dim3(rows), THREADS, 0, st, g)
    if (nvec <= 256) ASI_GRAD(64, 4, false);
    else if (sizeof(T) == 2 && nvec <= 1024 && rows > 2048) ASI_GRAD(64, 16, false);      // 7176 x 7051 46.2 -> 42.8 us, in fp32 slower
    else if (nvec <= 1024) ASI_GRAD(256, 4, false);
    else if (nvec <= 4096) ASI_GRAD(512, 8, false);
    else if (nvec <= 8192) ASI_GRAD(512, 16, false);
    else if (nvec <= 12288) ASI_GRAD(512, 24, false);
    else ASI_GRAD(1024, 24, true);
#undef ASI_GRAD
}

}  // namespace
}  // namespace asi

using namespace asi;

extern "C" {

size_t asi_token_logprobs_workspace_bytes(const asi_logprob_desc* desc) {
    if (check(desc) != ASI_OK || desc->top < 0 || desc->top > desc->vocab || desc->top > ASI_LOGPROB_MAX_TOP) return 0;
    const int parts = parts_of(desc);
    return parts == 1 ? 0 : sums_bytes(desc, parts) + round256((size_t)desc->rows * parts * desc->top * 8);
}

asi_status asi_token_logprobs(const asi_logprob_desc* desc, const void* logits, const int64_t* targets, float* logprob,
                              float* entropy, float* lse, float* top_logprob, int64_t* top_index, void* ws,
                              size_t ws_bytes, asi_stream_t stream) {
    if (asi_status why = check(desc); why != ASI_OK) return why;
    if (desc->top < 0 || desc->top > desc->vocab || desc->top > ASI_LOGPROB_MAX_TOP) return ASI_ERR_INVALID_ARG;
    if (desc->rows == 0) return ASI_OK;
    const size_t es = dtype_size(desc->dtype);
    if (!logits || !aligned(logits, es) || (logprob && !targets) || !aligned(targets, 8) || !aligned(logprob, 4) || !aligned(entropy, 4) ||
        !aligned(lse, 4) || (desc->top && (!top_logprob || !top_index || !aligned(top_logprob, 4) || !aligned(top_index, 8))))
        return ASI_ERR_INVALID_ARG;
    Args a{logits, targets, logprob, entropy, lse, top_logprob, top_index, desc->row_stride, desc->ignore_index, (int)desc->vocab,
           desc->top, desc->scale, scale_of(desc), parts_of(desc), 0, nullptr, nullptr};
    if (a.parts > 1) {
        if (!ws || !aligned(ws, 256) || ws_bytes < asi_token_logprobs_workspace_bytes(desc)) return ASI_ERR_WORKSPACE;
        a.part = (a.vocab + a.parts - 1) / a.parts;
        a.part = (a.part + 63) / 64 * 64;         // parts begin where 128 bytes of an aligned row do
        a.sums = static_cast<Sums*>(ws);
        a.keys = reinterpret_cast<unsigned long long*>(static_cast<char*>(ws) + sums_bytes(desc, a.parts));
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    in_launches(desc->rows, [&](long long first, unsigned rows) {
        Args b = a;
        b.x = static_cast<const char*>(logits) + first * desc->row_stride * (long long)es;
        b.targets = behind(targets, first); b.logprob = behind(logprob, first); b.entropy = behind(entropy, first); b.lse = behind(lse, first);
        b.top_logprob = behind(top_logprob, first * desc->top); b.top_index = behind(top_index, first * desc->top);
        if (desc->dtype == ASI_F32) forward<float>(b, rows, st);
        else forward<bf16_t>(b, rows, st);
    });
    return launched();
}

asi_status asi_token_logprobs_grad(const asi_logprob_desc* desc, const void* logits, const int64_t* targets,
                                   const float* grad_logprob, const float* grad_entropy, void* dlogits, float* logprob,
                                   float* entropy, asi_stream_t stream) {
    if (asi_status why = check(desc); why != ASI_OK) return why;
    if (desc->grad_stride < desc->vocab || (dlogits == logits && desc->grad_stride != desc->row_stride)) return ASI_ERR_INVALID_ARG;
    if (desc->rows == 0) return ASI_OK;
    const size_t es = dtype_size(desc->dtype);
    if (!logits || !dlogits || !aligned(logits, es) || !aligned(dlogits, es) || ((logprob || grad_logprob) && !targets) || !aligned(targets, 8) ||
        !aligned(grad_logprob, 4) || !aligned(grad_entropy, 4) || !aligned(logprob, 4) || !aligned(entropy, 4))
        return ASI_ERR_INVALID_ARG;
    const GradArgs g{logits, dlogits, targets, grad_logprob, grad_entropy, logprob, entropy, desc->row_stride, desc->grad_stride,
                     desc->ignore_index, (int)desc->vocab, desc->scale, scale_of(desc)};
    hipStream_t st = static_cast<hipStream_t>(stream);
    in_launches(desc->rows, [&](long long first, unsigned rows) {
        GradArgs h = g;
        h.x = static_cast<const char*>(logits) + first * desc->row_stride * (long long)es;
        h.dx = static_cast<char*>(dlogits) + first * desc->grad_stride * (long long)es;
        h.targets = behind(targets, first); h.a = behind(grad_logprob, first); h.b = behind(grad_entropy, first);
        h.logprob = behind(logprob, first); h.entropy = behind(entropy, first);
        if (desc->dtype == ASI_F32) backward<float>(h, rows, st);
        else backward<bf16_t>(h, rows, st);
    });
    return launched();
}

}  // extern "C"
