// Embedding lookup with scaling, and its gradient by sorted tokens (include/asi_lm.h).
//
// Lookup: a wave copies up to 256 vectors of one row; bound by memory.
//
// Gradient: the positions are sorted by token (equal tokens by position), the sorted list is cut into runs of `run` entries, and a
// group of lanes adds up the rows of one run, each lane a vector of columns, writing a row of the table's gradient wherever the
// token changes.  A token whose entries cross the end of a run leaves partial rows in scratch, which a second kernel adds in the
// order of the runs.  So a token that makes up most of a batch costs what any other share of it costs, no sum depends on the order
// in which workgroups run, and every row of the result is written once: the workgroups behind those of the runs fill
// the rows without a token with zeros.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "asi_lm_device.h"

namespace asi {
namespace {

constexpr int kThreads = 256;
constexpr int kFillRows = 32;         // table rows of a workgroup that writes zeros

// ---- lookup ------------------------------------------------------------------------------------------------
struct LookupArgs {
    const int64_t* tokens;
    const void* table;
    void* out;
    long long n, vocab, table_stride, out_stride;
    int dim, parts;                   // parts: waves of a row
    float scale;
};
template <typename T, typename O> __global__ __launch_bounds__(kThreads) void k_lookup(const LookupArgs a) {
    // values of a lane's vector: 16 bytes of the wider type
    constexpr int N = sizeof(T) > sizeof(O) ? Vec16<T>::N : Vec16<O>::N;
    const int lane = threadIdx.x & 63;
    const long long id = (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (id >= a.n * a.parts) return;
    const long long t = id / a.parts;
    const int part = (int)(id - t * a.parts);
    const long long tok = a.tokens[t];
    const bool ok = tok >= 0 && tok < a.vocab;
    const T* src = static_cast<const T*>(a.table) + (ok ? tok : 0) * a.table_stride;
    O* dst = static_cast<O*>(a.out) + t * a.out_stride;
    const float nan = __builtin_nanf("");
    const int end = min(a.dim, (part + 1) * 256 * N);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int d = part * 256 * N + (k * 64 + lane) * N;
        if (d + N <= end) {
            float f[N];
            load_values<N>(src + d, f);
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = ok ? f[i] * a.scale : nan;
            store_values<N>(dst + d, f);
        }
    }
}
template <typename T, typename O> __global__ __launch_bounds__(kThreads) void k_lookup_any(const LookupArgs a) {
    const int lane = threadIdx.x & 63;
    const long long id = (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (id >= a.n * a.parts) return;
    const long long t = id / a.parts;
    const int part = (int)(id - t * a.parts);
    const long long tok = a.tokens[t];
    const bool ok = tok >= 0 && tok < a.vocab;
    const T* src = static_cast<const T*>(a.table) + (ok ? tok : 0) * a.table_stride;
    O* dst = static_cast<O*>(a.out) + t * a.out_stride;
    const int end = min(a.dim, (part + 1) * 1024);
#pragma unroll 4
    for (int d = part * 1024 + lane; d < end; d += 64) dst[d] = from_f32<O>(ok ? to_f32(src[d]) * a.scale : __builtin_nanf(""));
}

// ---- gradient: sorting ----------------------------------------------------------------------------------------
// A token that counts for nothing sorts behind all others, as `vocab`.
struct SortArgs {
    const int64_t* tokens;
    uint32_t* key;                    // sorted tokens
    uint32_t* pos;                    // their positions
    long long padding;
    uint32_t vocab;
    int n;
};
__device__ __forceinline__ uint32_t key_of(const SortArgs& a, int i) {
    const long long t = a.tokens[i];
    return t >= 0 && t < (long long)a.vocab && t != a.padding ? (uint32_t)t : a.vocab;
}
// Every entry's place is the number of entries before it: those with a smaller token and those with the same one at an earlier position.
constexpr int kRankKeys = 16, kRankTile = 4096;
__global__ __launch_bounds__(kThreads) void k_rank(const SortArgs a) {
    __shared__ uint32_t tile[kRankTile];
    __shared__ int count[kThreads / kRankKeys][kRankKeys];
    const int which = threadIdx.x & (kRankKeys - 1), share = threadIdx.x / kRankKeys;
    const int i = blockIdx.x * kRankKeys + which;
    const uint32_t mine = i < a.n ? key_of(a, i) : 0;
    int before = 0;
    for (int base = 0; base < a.n; base += kRankTile) {
        const int m = min(kRankTile, a.n - base);
        __syncthreads();
        for (int j = threadIdx.x; j < m; j += kThreads) tile[j] = key_of(a, base + j);
        __syncthreads();
        for (int j = share; j < m; j += kThreads / kRankKeys) {
            const uint32_t k = tile[j];
            before += k < mine || (k == mine && base + j < i);
        }
    }
    count[share][which] = before;
    __syncthreads();
    if (threadIdx.x < kRankKeys && i < a.n) {
        int place = 0;
        for (int s = 0; s < kThreads / kRankKeys; ++s) place += count[s][which];
        a.key[place] = mine;
        a.pos[place] = (uint32_t)i;
    }
}

// ---- gradient: sums -------------------------------------------------------------------------------------------
struct SumArgs {
    const uint32_t* key;
    const uint32_t* pos;
    const void* dout;
    void* dtable;
    float* part;                      // [run][2][dim]: what a run has of the token it shares with the run before it, and with the one after
    long long out_stride, table_stride;
    uint32_t vocab;
    int n, run, runs, dim;
    int columns, lanes, column_tiles; // lanes: of a group (a power of two); columns: that a group covers
    int run_blocks;                   // workgroups of runs, before those that write zeros
    int accumulate, vec;
    float scale;
};
template <typename D, int N> __device__ __forceinline__ void write_row(const SumArgs& a, uint32_t token, int d, const float* acc) {
    D* dst = static_cast<D*>(a.dtable) + (long long)token * a.table_stride + d;
    float v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = acc[i] * a.scale;
    if constexpr (N > 1) {
        if (a.vec) {
            if (a.accumulate) {
                float old[N];
                load_values<N>(dst, old);
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] += old[i];
            }
            store_values<N>(dst, v);
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) dst[i] = from_f32<D>(a.accumulate ? to_f32(dst[i]) + v[i] : v[i]);
}
// N: columns of a lane
template <typename O, typename D, int N> __device__ __forceinline__ void sum_run(const SumArgs& a) {
    const int groups = kThreads / a.lanes, lane = threadIdx.x & (a.lanes - 1);
    const int id = blockIdx.x / a.column_tiles, tile = blockIdx.x - id * a.column_tiles;
    const int r = id * groups + threadIdx.x / a.lanes;
    const int d = tile * a.columns + lane * N;
    if (r >= a.runs || d >= a.dim) return;
    const int begin = r * a.run, end = min(a.n, begin + a.run);
    const O* dout = static_cast<const O*>(a.dout) + d;
    uint32_t token = a.key[begin];
    bool before = begin > 0 && a.key[begin - 1] == token;
    float acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.f;
    for (int e = begin; e < end; ++e) {
        const uint32_t next = e + 1 < a.n ? a.key[e + 1] : 0xffffffffu;
        if (token < a.vocab) {
            const O* row = dout + (long long)a.pos[e] * a.out_stride;
            if constexpr (N == Vec16<O>::N) {
                Vec16<O> v;
                v.load(row);
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] += v.get(i);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] += to_f32(row[i]);
            }
        }
        if (next != token || e + 1 == end) {
            const bool after = next == token;
            if (token < a.vocab) {
                if (!before && !after) {
                    write_row<D, N>(a, token, d, acc);
                } else {
                    float* p = a.part + ((long long)r * 2 + (before ? 0 : 1)) * a.dim + d;
#pragma unroll
                    for (int i = 0; i < N; ++i) p[i] = acc[i];
                }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] = 0.f;
            before = false;
            token = next;
        }
    }
}
// First place in the sorted keys with a key of at least `bound`: 64 places are looked at in a step.  All lanes of a wave take part.
__device__ __forceinline__ int lower_bound(const uint32_t* key, int n, uint32_t bound) {
    int lo = 0, hi = n;               // the answer is in [lo, hi]
    const int lane = threadIdx.x & 63;
    while (hi > lo) {
        const int step = (hi - lo + 63) / 64;
        const int at = lo + lane * step;
        const bool less = at < hi && key[at] < bound;
        const int c = __popcll(__ballot(less));     // the lanes that see a smaller key are the first ones
        if (c == 0) return lo;
        const int last = lo + (c - 1) * step;       // key[last] < bound
        hi = min(hi, last + step);
        lo = last + 1;
    }
    return lo;
}
template <typename D> __device__ __forceinline__ void write_zeros(const SumArgs& a) {
    __shared__ uint32_t present[kFillRows];
    __shared__ int range[2];
    const uint32_t v0 = (uint32_t)(blockIdx.x - a.run_blocks) * kFillRows;
    const int rows = (int)min((uint32_t)kFillRows, a.vocab - v0);
    const int wave = threadIdx.x >> 6;
    if (threadIdx.x < kFillRows) present[threadIdx.x] = 0;
    if (wave < 2) {
        const int at = lower_bound(a.key, a.n, wave ? v0 + rows : v0);
        if ((threadIdx.x & 63) == 0) range[wave] = at;
    }
    __syncthreads();
    for (int e = range[0] + threadIdx.x; e < range[1]; e += kThreads) present[a.key[e] - v0] = 1;   // every writer writes the same
    __syncthreads();
    constexpr int N = Vec16<D>::N;
    for (int r = 0; r < rows; ++r) {
        if (present[r]) continue;
        D* dst = static_cast<D*>(a.dtable) + (long long)(v0 + r) * a.table_stride;
        if (a.vec) {
            for (int d = threadIdx.x * N; d < a.dim; d += kThreads * N) *reinterpret_cast<uint4*>(dst + d) = make_uint4(0, 0, 0, 0);
        } else {
            for (int d = threadIdx.x; d < a.dim; d += kThreads) dst[d] = from_f32<D>(0.f);
        }
    }
}
template <typename O, typename D, int N> __global__ __launch_bounds__(kThreads) void k_sum(const SumArgs a) {
    if ((int)blockIdx.x >= a.run_blocks) write_zeros<D>(a);
    else sum_run<O, D, N>(a);
}
// Adds up the partial rows of the token that run `blockIdx.x / tiles` shares with the next one and none before it.
template <typename D> __global__ __launch_bounds__(kThreads) void k_join(const SumArgs a, int tiles) {
    const int r = blockIdx.x / tiles, tile = blockIdx.x - r * tiles;
    const int last = (r + 1) * a.run - 1;                         // r is not the last run
    const uint32_t token = a.key[last];
    if (token >= a.vocab || a.key[last + 1] != token) return;
    if (a.key[r * a.run] == token && r > 0 && a.key[r * a.run - 1] == token) return;    // it began in an earlier run
    // runs r + 1 .. r + more begin with it
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int more = 0;
    for (;;) {
        const int at = r + 1 + more + lane;
        const unsigned long long same = __ballot(at < a.runs && a.key[(long long)at * a.run] == token);
        const int c = same == ~0ull ? 64 : __ffsll((long long)~same) - 1;
        more += c;
        if (c < 64) break;
    }
    __shared__ float sums[kThreads / 64][64];
    const int d = tile * 64 + lane;
    float v = 0.f;
    if (d < a.dim) {
        if (wave == 0) v = a.part[((long long)r * 2 + 1) * a.dim + d];
        const int share = (more + kThreads / 64 - 1) / (kThreads / 64);
        const int from = wave * share, to = min(more, from + share);
#pragma unroll 8
        for (int k = from; k < to; ++k) v += a.part[(long long)(r + 1 + k) * 2 * a.dim + d];
    }
    sums[wave][lane] = v;
    __syncthreads();
    if (wave == 0 && d < a.dim) {
        for (int w = 1; w < kThreads / 64; ++w) v += sums[w][lane];
        write_row<D, 1>(a, token, d, &v);
    }
}

// ---- host ----
asi_status check(const asi_embedding_desc* d) {
    if (!d) return ASI_ERR_INVALID_ARG;
    if (!dtype_ok(d->table_dtype) || !dtype_ok(d->out_dtype)) return ASI_ERR_UNSUPPORTED;
    if (d->tokens < 0 || d->vocab < 1 || d->dim < 1 || d->table_stride < d->dim || d->out_stride < d->dim || d->reserved) return ASI_ERR_INVALID_ARG;
    if (!std::isfinite(d->scale)) return ASI_ERR_INVALID_ARG;
    if (d->tokens >= (1LL << 30) || d->vocab >= (1LL << 30) || d->dim > (1LL << 24)) return ASI_ERR_UNSUPPORTED;
    return ASI_OK;
}
// Entries of a run: 32, more where the table's rows are many so that partial rows stay few
int run_length(const asi_embedding_desc* d) {
    int run = 32;
    while (d->tokens / run > 1024 && run < 1024) run *= 2;
    return run;
}
struct GradPlan {
    size_t key, pos, part, bytes;     // offsets
    int run, runs;
};
GradPlan plan(const asi_embedding_desc* d) {
    GradPlan p;
    p.run = run_length(d);
    p.runs = (int)((d->tokens + p.run - 1) / p.run);
    p.key = 0;
    p.pos = round256((size_t)d->tokens * 4);
    p.part = p.pos + round256((size_t)d->tokens * 4);
    p.bytes = p.part + round256((size_t)p.runs * 2 * d->dim * 4);
    return p;
}
template <typename T, typename O> void lookup(const LookupArgs& a, bool vec, dim3 grid, hipStream_t st) {
    if (vec) hipLaunchKernelGGL((k_lookup<T, O>), grid, kThreads, 0, st, a);
    else hipLaunchKernelGGL((k_lookup_any<T, O>), grid, kThreads, 0, st, a);
}
template <typename O, typename D> void sum(const SumArgs& a, int n, unsigned blocks, hipStream_t st) {
    if (n == Vec16<O>::N) hipLaunchKernelGGL((k_sum<O, D, Vec16<O>::N>), dim3(blocks), kThreads, 0, st, a);
    else hipLaunchKernelGGL((k_sum<O, D, 1>), dim3(blocks), kThreads, 0, st, a);
}

}  // namespace
}  // namespace asi

using namespace asi;

extern "C" {

asi_status asi_embedding(const asi_embedding_desc* desc, const int64_t* tokens, const void* table, void* out, asi_stream_t stream) {
    if (asi_status why = check(desc); why != ASI_OK) return why;
    if (desc->tokens == 0) return ASI_OK;
    const size_t ts = dtype_size(desc->table_dtype), os = dtype_size(desc->out_dtype);
    if (!tokens || !table || !out || !aligned(tokens, 8) || !aligned(table, ts) || !aligned(out, os)) return ASI_ERR_INVALID_ARG;
    const int n = (int)(16 / std::max(ts, os));
    const bool vec = desc->dim % n == 0 && desc->table_stride % n == 0 && desc->out_stride % n == 0 && aligned(table, n * ts) && aligned(out, n * os);
    LookupArgs a{tokens, table, out, desc->tokens, desc->vocab, desc->table_stride, desc->out_stride, (int)desc->dim, 0, desc->scale};
    const int per_wave = vec ? 256 * n : 1024;
    a.parts = (int)((desc->dim + per_wave - 1) / per_wave);
    const long long waves = a.n * a.parts;
    if (waves > 0x7fffffffLL) return ASI_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)((waves + 3) / 4));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (desc->table_dtype == ASI_F32) {
        if (desc->out_dtype == ASI_F32) lookup<float, float>(a, vec, grid, st);
        else lookup<float, bf16_t>(a, vec, grid, st);
    } else {
        if (desc->out_dtype == ASI_F32) lookup<bf16_t, float>(a, vec, grid, st);
        else lookup<bf16_t, bf16_t>(a, vec, grid, st);
    }
    return launched();
}

size_t asi_embedding_grad_workspace_bytes(const asi_embedding_desc* desc) {
    if (check(desc) != ASI_OK || desc->tokens == 0) return 0;
    return plan(desc).bytes;
}

asi_status asi_embedding_grad(const asi_embedding_desc* desc, const int64_t* tokens, const void* grad_out, void* dtable,
                              int accumulate, void* ws, size_t ws_bytes, asi_stream_t stream) {
    if (asi_status why = check(desc); why != ASI_OK) return why;
    const size_t ds = dtype_size(desc->table_dtype), os = dtype_size(desc->out_dtype);
    if (!dtable || !aligned(dtable, ds)) return ASI_ERR_INVALID_ARG;
    if (desc->tokens && (!tokens || !grad_out || !aligned(tokens, 8) || !aligned(grad_out, os))) return ASI_ERR_INVALID_ARG;
    const GradPlan p = plan(desc);
    if (desc->tokens && (!ws || !aligned(ws, 256) || ws_bytes < p.bytes)) return ASI_ERR_WORKSPACE;
    if (desc->tokens == 0 && accumulate) return ASI_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* w = static_cast<char*>(ws);
    SumArgs a{};
    a.key = reinterpret_cast<uint32_t*>(w + p.key);
    a.pos = reinterpret_cast<uint32_t*>(w + p.pos);
    a.part = reinterpret_cast<float*>(w + p.part);
    a.dout = grad_out; a.dtable = dtable;
    a.out_stride = desc->out_stride; a.table_stride = desc->table_stride;
    a.vocab = (uint32_t)desc->vocab;
    a.n = (int)desc->tokens; a.run = p.run; a.runs = p.runs; a.dim = (int)desc->dim;
    a.accumulate = accumulate != 0;
    a.scale = desc->scale;
    a.vec = aligned(dtable, 16) && desc->table_stride % (16 / ds) == 0 && desc->dim % (16 / ds) == 0;
    const int wide = (int)(16 / os);
    const int n = desc->dim % wide == 0 && desc->out_stride % wide == 0 && aligned(grad_out, 16) ? wide : 1;
    a.lanes = 1;
    while (a.lanes < kThreads && a.lanes * n < a.dim) a.lanes *= 2;
    a.columns = a.lanes * n;
    a.column_tiles = (a.dim + a.columns - 1) / a.columns;
    const int groups = kThreads / a.lanes;
    const long long run_blocks = (long long)((p.runs + groups - 1) / groups) * a.column_tiles;
    const long long fill_blocks = accumulate ? 0 : (desc->vocab + kFillRows - 1) / kFillRows;
    const int tiles = (a.dim + 63) / 64;
    if (run_blocks + fill_blocks > 0x7fffffffLL || (long long)p.runs * tiles > 0x7fffffffLL) return ASI_ERR_UNSUPPORTED;
    a.run_blocks = (int)run_blocks;
    if (desc->tokens) {
        const SortArgs s{tokens, reinterpret_cast<uint32_t*>(w + p.key), reinterpret_cast<uint32_t*>(w + p.pos), desc->padding_index, a.vocab, a.n};
        hipLaunchKernelGGL(k_rank, dim3((unsigned)((a.n + kRankKeys - 1) / kRankKeys)), kThreads, 0, st, s);
    }
    const unsigned blocks = (unsigned)(run_blocks + fill_blocks);
    if (desc->out_dtype == ASI_F32) {
        if (desc->table_dtype == ASI_F32) sum<float, float>(a, n, blocks, st);
        else sum<float, bf16_t>(a, n, blocks, st);
    } else {
        if (desc->table_dtype == ASI_F32) sum<bf16_t, float>(a, n, blocks, st);
        else sum<bf16_t, bf16_t>(a, n, blocks, st);
    }
    if (p.runs > 1) {
        const dim3 grid((unsigned)((p.runs - 1) * tiles));
        if (desc->table_dtype == ASI_F32) hipLaunchKernelGGL(k_join<float>, grid, kThreads, 0, st, a, tiles);
        else hipLaunchKernelGGL(k_join<bf16_t>, grid, kThreads, 0, st, a, tiles);
    }
    return launched();
}

}  // extern "C"
