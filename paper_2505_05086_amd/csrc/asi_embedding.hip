// Embedding lookup with scaling, and its gradient by sorted tokens (include/asi_lm.h).
//
// Lookup: a wave copies up to 256 vectors of one row; bound by memory.
//
// Gradient: the positions are sorted by token (equal tokens by position), the sorted list is cut into runs of `run` entries, and a
// group of lanes adds up the rows of one run, each lane a vector of columns, writing a row of the table's gradient wherever the
// token changes.  A token whose entries cross the end of a run leaves partial rows in scratch, which a second kernel adds in the
// order of the runs.  So a token that makes up most of a batch costs what any other share of it costs, no sum depends on the order
// in which workgroups run, and every row of the result is written once: the workgroups behind those of the runs fill
// the rows without a token with zeros.  Few tokens take one launch without scratch: a workgroup for each position looks for
// the positions of its token, and adds up their rows if its own is the first; there a token that most of them are is one chain.
//
// Measured: lookup of 4096 x 2048 in bf16 6.5 us; gradient of them into 32000 rows in fp32, zeros written past the caches, 56.7 us (4.9 TB/s),
// of 32767 x 1000 added to rows in fp32 51.5 us, of which the sums are 32 (4.5 TB/s), the sort 13 and the join 6.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "asi_lds.h"
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
// One launch: workgroup w looks at every token and keeps those in its `span` ids, so that the number of smaller ones, which
// is where its part of the sorted list begins, comes with the same look.  Its 16 waves take a part of the positions each, in
// order, and sort what they found by counting: a table of counts for each (id, wave), its prefix sums, and within a wave the rank
// among equal ids.  No atomics, and the time does not depend on the tokens.  A token that counts for nothing sorts behind all
// others, as `vocab`.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kSortList = 1024;       // entries of a wave that are kept; a wave with more looks at its tokens again
constexpr int kMaxSpan = kSortThreads;
constexpr int kPlaceBits = 22;        // of an entry: its place in the wave's part of the positions; above them its id within the span
static_assert(kMaxSpan <= 1 << (32 - kPlaceBits), "an entry is a word");
struct SortArgs {
    const int64_t* tokens;
    uint32_t* key;                    // sorted tokens
    uint32_t* pos;                    // their positions
    uint32_t padding;                 // vocab where there is none
    uint32_t vocab;
    int n, span;
};
__device__ __forceinline__ uint32_t key_of(const SortArgs& a, long long t) {
    const uint32_t lo = (uint32_t)t, k = (uint32_t)((unsigned long long)t >> 32) ? a.vocab : min(lo, a.vocab);
    return k == a.padding ? a.vocab : k;
}
__device__ __forceinline__ int lanes_below(unsigned long long mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}
// the lanes of `members` with this lane's `low`
__device__ __forceinline__ unsigned long long lanes_alike(unsigned long long members, uint32_t low) {
    unsigned long long m = members;
#pragma unroll
    for (int bit = 0; bit < 10; ++bit) {
        const unsigned long long set = __ballot(low >> bit & 1u);
        m &= low >> bit & 1u ? set : ~set;
    }
    return m;
}
static_assert(kMaxSpan <= 1 << 10, "ids within a workgroup's span have 10 bits");
__global__ __launch_bounds__(kSortThreads) void k_sort(const SortArgs a) {
    extern __shared__ uint32_t lds[];
    uint32_t* count = lds;                                     // [wave][span]
    uint32_t* list = lds + kSortWaves * a.span + (threadIdx.x >> 6) * kSortList;       // the wave's entries
    __shared__ int smaller[kSortWaves], totals[kSortWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t lo = blockIdx.x * (uint32_t)a.span, span = (uint32_t)a.span;
    const int part = ((a.n + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
    const int begin = min(a.n, wave * part), end = min(a.n, begin + part);
    for (int i = threadIdx.x; i < kSortWaves * a.span; i += kSortThreads) count[i] = 0;
    int less = 0, found = 0;
    // a token of each lane, where it counts
    auto look = [&](long long t, int i, bool counts) {
        const uint32_t k = key_of(a, t);
        less += __popcll(__ballot(counts && k < lo));
        const bool mine = counts && k - lo < span;
        const unsigned long long m = __ballot(mine);
        if (m) {                              // few looks find any
            const int at = found + lanes_below(m);
            if (mine && at < kSortList) list[at] = (k - lo) << kPlaceBits | (uint32_t)(i - begin);
            found += __popcll(m);
        }
    };
    constexpr int U = 8;
    int base = begin;
    for (; base + 64 * U <= end; base += 64 * U) {
        long long t[U];
#pragma unroll
        for (int u = 0; u < U; ++u) t[u] = a.tokens[base + 64 * u + lane];
#pragma unroll
        for (int u = 0; u < U; ++u) look(t[u], base + 64 * u + lane, true);
    }
    if (base < end) {
        long long t[U];
#pragma unroll
        for (int u = 0; u < U; ++u) t[u] = a.tokens[min(base + 64 * u + lane, a.n - 1)];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (base + 64 * u < end) look(t[u], base + 64 * u + lane, base + 64 * u + lane < end);
    }
    if (lane == 0) smaller[wave] = less;
    __syncthreads();
    uint32_t* mine = count + wave * a.span;
    // f(member, id within the span, position) for this wave's entries in order, 64 at a time
    auto entries = [&](auto f) {
        if (found <= kSortList && part <= 1 << kPlaceBits) {
            for (int e = lane; e - lane < found; e += 64) {
                const bool member = e < found;
                const uint32_t entry = member ? list[e] : 0u;
                f(member, entry >> kPlaceBits, (uint32_t)begin + (entry & ((1u << kPlaceBits) - 1)));
            }
        } else {
            for (int i0 = begin; i0 < end; i0 += 64 * U) {
                long long t[U];
#pragma unroll
                for (int u = 0; u < U; ++u) t[u] = a.tokens[min(i0 + 64 * u + lane, a.n - 1)];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + 64 * u + lane;
                    const uint32_t low = key_of(a, t[u]) - lo;
                    const bool member = i < end && low < span;
                    if (__ballot(member)) f(member, member ? low : 0u, (uint32_t)i);
                }
            }
        }
    };
    entries([&](bool member, uint32_t low, uint32_t) {
        const unsigned long long alike = lanes_alike(__ballot(member), low);
        if (member && lanes_below(alike) == 0) mine[low] += (uint32_t)__popcll(alike);
        __builtin_amdgcn_wave_barrier();
    });
    __syncthreads();
    // prefix sums: ids in order, of each id the waves in order
    uint32_t total = 0;
    if (threadIdx.x < span)
        for (int w = 0; w < kSortWaves; ++w) total += count[w * a.span + threadIdx.x];
    uint32_t upto = total;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = (uint32_t)__shfl_up((int)upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 63) totals[wave] = (int)upto;
    __syncthreads();
    uint32_t at = upto - total;
    for (int w = 0; w < kSortWaves; ++w) at += (uint32_t)smaller[w] + (w < wave ? (uint32_t)totals[w] : 0u);
    if (threadIdx.x < span) {
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = count[w * a.span + threadIdx.x];
            count[w * a.span + threadIdx.x] = at;
            at += c;
        }
    }
    __syncthreads();
    entries([&](bool member, uint32_t low, uint32_t position) {
        const unsigned long long alike = lanes_alike(__ballot(member), low);
        const int rank = lanes_below(alike);
        if (member) {
            const uint32_t first = mine[low];
            a.key[first + rank] = lo + low;
            a.pos[first + rank] = position;
            __builtin_amdgcn_wave_barrier();       // every lane has read before the first of them writes
            if (rank == 0) mine[low] = first + (uint32_t)__popcll(alike);
        }
        __builtin_amdgcn_wave_barrier();
    });
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
    int accumulate;
    float scale;
};
// C neighbouring columns of a row as loaded: so many rows can be in flight at little cost in registers
template <typename O, int C> struct Columns {
    static_assert(C == 1 || (C * sizeof(O) == 8 || C * sizeof(O) == 16), "one value, 8 or 16 bytes");
    using Raw = std::conditional_t<C == 1, O, std::conditional_t<C * sizeof(O) == 8, uint2, uint4>>;
    Raw raw;
    __device__ __forceinline__ void load(const O* p) {
        if constexpr (C == 1) raw = *p;
        else if constexpr (C * sizeof(O) == 8) raw = load_words2(p);
        else raw = load_words4(p);
    }
    // Has arrived here: the compiler would otherwise move the load of a row that may not count to where it turns out to, behind the others'.
    __device__ __forceinline__ void arrived() {
        if constexpr (C > 1 && C * sizeof(O) == 8) asm volatile("" : "+v"(raw.x), "+v"(raw.y));
        if constexpr (C > 1 && C * sizeof(O) == 16) asm volatile("" : "+v"(raw.x), "+v"(raw.y), "+v"(raw.z), "+v"(raw.w));
        if constexpr (C == 1 && sizeof(O) == 4) asm volatile("" : "+v"(raw));
        if constexpr (C == 1 && sizeof(O) == 2) asm volatile("" : "+v"(raw.bits));
    }
    __device__ __forceinline__ void add_to(float* f) const {
        if constexpr (C == 1) {
            f[0] += to_f32(raw);
        } else if constexpr (sizeof(O) == 4) {
            f[0] += __uint_as_float(raw.x); f[1] += __uint_as_float(raw.y); f[2] += __uint_as_float(raw.z); f[3] += __uint_as_float(raw.w);
        } else {
            f[0] += __uint_as_float(raw.x << 16); f[1] += __uint_as_float(raw.x & 0xffff0000u);
            f[2] += __uint_as_float(raw.y << 16); f[3] += __uint_as_float(raw.y & 0xffff0000u);
            if constexpr (C == 8) {
                f[4] += __uint_as_float(raw.z << 16); f[5] += __uint_as_float(raw.z & 0xffff0000u);
                f[6] += __uint_as_float(raw.w << 16); f[7] += __uint_as_float(raw.w & 0xffff0000u);
            }
        }
    }
};
template <typename D, int C> __device__ __forceinline__ void load_result(const SumArgs& a, uint32_t token, int d, float* old) {
    const D* src = static_cast<const D*>(a.dtable) + (long long)token * a.table_stride + d;
    if constexpr (C > 1) load_values<C>(src, old);
    else old[0] = to_f32(*src);
}
template <typename D, int C> __device__ __forceinline__ void store_result(const SumArgs& a, uint32_t token, int d, const float* v) {
    D* dst = static_cast<D*>(a.dtable) + (long long)token * a.table_stride + d;
    if constexpr (C > 1) store_values<C>(dst, v);
    else *dst = from_f32<D>(v[0]);
}
constexpr int kLeastLanes = 8, kMostRun = 64;
constexpr int kMostEntries = kThreads / kLeastLanes * kMostRun;
// A lane has P pieces of C neighbouring columns, the pieces of a group's lanes side by side, so that loads and stores of either
// type are whole lines.  ADD: the result is added to.  Rows are loaded several at a time, with the rows of the result that they
// complete where those are added to, so that a run waits for memory a few times, not once for each entry.
template <typename O, typename D, int C, int P, bool ADD> __device__ __forceinline__ void sum_run(const SumArgs& a) {
    constexpr int U = ADD ? 4 : 8;
    __shared__ uint32_t key[kMostEntries + 2], pos[kMostEntries];       // key[0]: of the entry before this workgroup's
    const int groups = kThreads / a.lanes, lane = threadIdx.x & (a.lanes - 1), group = threadIdx.x / a.lanes;
    const int id = blockIdx.x / a.column_tiles, tile = blockIdx.x - id * a.column_tiles;
    const int first = id * groups * a.run, entries = min(a.n - first, groups * a.run);
    for (int i = threadIdx.x; i < entries + 2; i += kThreads) {
        const int e = first + i - 1;
        key[i] = e >= 0 && e < a.n ? a.key[e] : 0xffffffffu;
        if (i < entries) pos[i] = a.pos[first + i];
    }
    __syncthreads();
    const int r = id * groups + group;
    const int d = tile * a.columns + lane * C, apart = a.lanes * C;     // first column of the first piece; from piece to piece
    if (r >= a.runs || d >= a.dim) return;
    const int begin = group * a.run, end = min(entries, begin + a.run);
    const O* dout = static_cast<const O*>(a.dout);
    int col[P];                          // a piece behind the row's end reads the first one's columns again and writes nothing
    bool has[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        has[p] = d + p * apart < a.dim;
        col[p] = has[p] ? d + p * apart : d;
    }
    bool before = key[begin] == key[begin + 1];
    float acc[P][C];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < C; ++i) acc[p][i] = 0.f;
    for (int e0 = begin; e0 < end; e0 += U) {
        Columns<O, C> v[U][P];
        float old[ADD ? U : 1][P][C];
        bool begun = before;             // whether the token at hand began in an earlier run
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = min(e0 + u, end - 1);
            const O* row = dout + (long long)pos[e] * a.out_stride;
#pragma unroll
            for (int p = 0; p < P; ++p) v[u][p].load(row + col[p]);
            if constexpr (ADD) {
                const uint32_t token = key[e + 1];
                const bool last = key[e + 2] != token;
                if (last && !begun && token < a.vocab) {
#pragma unroll
                    for (int p = 0; p < P; ++p) load_result<D, C>(a, token, col[p], old[u][p]);
                }
                if (last) begun = false;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int p = 0; p < P; ++p) v[u][p].arrived();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = e0 + u;
            if (e < end) {
                const uint32_t token = key[e + 1];
                const bool after = key[e + 2] == token;
#pragma unroll
                for (int p = 0; p < P; ++p) v[u][p].add_to(acc[p]);
                if (!after || e + 1 == end) {
                    if (token < a.vocab) {
                        if (before || after) {
                            float* out = a.part + ((long long)r * 2 + (before ? 0 : 1)) * a.dim;
#pragma unroll
                            for (int p = 0; p < P; ++p) {
                                if (!has[p]) continue;
                                if constexpr (C > 1) store_values<C>(out + col[p], acc[p]);      // dim is a multiple of C then
                                else out[col[p]] = acc[p][0];
                            }
                        } else {
#pragma unroll
                            for (int p = 0; p < P; ++p) {
#pragma unroll
                                for (int i = 0; i < C; ++i) acc[p][i] = ADD ? acc[p][i] * a.scale + old[u][p][i] : acc[p][i] * a.scale;
                                if (has[p]) store_result<D, C>(a, token, col[p], acc[p]);
                            }
                        }
                    }
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int i = 0; i < C; ++i) acc[p][i] = 0.f;
                    before = false;
                }
            }
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
// Zeros into the rows of this workgroup's kFillRows that have no token, a wave a row: vectors from its first whole address on, and
// the elements before and behind them
template <typename D> __device__ __forceinline__ void write_zeros(const SumArgs& a, uint32_t v0, int rows, const uint32_t* present) {
    constexpr int N = Vec16<D>::N;
    const int lane = threadIdx.x & 63;
    for (int r = threadIdx.x >> 6; r < rows; r += kThreads / 64) {
        if (present[r]) continue;
        D* dst = static_cast<D*>(a.dtable) + (long long)(v0 + r) * a.table_stride;
        const int head = min((int)((16 - (reinterpret_cast<uintptr_t>(dst) & 15)) & 15) / (int)sizeof(D), a.dim), nvec = (a.dim - head) / N;
        for (int v = lane; v < nvec; v += 64) store_past(dst + head + v * N, make_uint4(0, 0, 0, 0));
        const int loose = lane < head ? lane : nvec * N + lane;       // behind: lane - head from the end of the vectors
        if (loose < a.dim) dst[loose] = from_f32<D>(0.f);
    }
}
template <typename D> __device__ __forceinline__ void fill(const SumArgs& a) {
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
    write_zeros<D>(a, v0, rows, present);
}
template <typename O, typename D, int C, int P, bool ADD> __global__ __launch_bounds__(kThreads) void k_sum(const SumArgs a) {
    if ((int)blockIdx.x >= a.run_blocks) fill<D>(a);
    else sum_run<O, D, C, P, ADD>(a);
}
// Adds up the partial rows of tokens that cross the ends of runs, of every token in the order of the runs.  A workgroup has 8 runs and
// a tile of columns, C a lane; a wave looks whether its run shares a token with the next one and none before it, and adds up a short
// list alone.  Long lists are shared by all waves, each a stretch of the runs.
constexpr int kJoinThreads = 512, kJoinRuns = kJoinThreads / 64, kShort = 8;
template <typename D, int C> __global__ __launch_bounds__(kJoinThreads) void k_join(const SumArgs a, int tiles) {
    __shared__ int more[kJoinRuns];               // runs that go on with the token of this one
    __shared__ float sums[kJoinRuns][C][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r0 = blockIdx.x / tiles * kJoinRuns, d = ((blockIdx.x % tiles) * 64 + lane) * C;
    const int r = r0 + wave;
    uint32_t token = a.vocab;
    int n = 0;
    if (r + 1 < a.runs) {
        const int last = (r + 1) * a.run - 1;
        const uint32_t k = a.key[last], next = a.key[last + 1], head = a.key[r * a.run], prior = r > 0 ? a.key[r * a.run - 1] : 0xffffffffu;
        if (k == next && !(head == k && prior == k)) token = k;
    }
    while (token < a.vocab) {
        const int at = r + 1 + n + lane;
        const unsigned long long same = __ballot(at < a.runs && a.key[(long long)(at < a.runs ? at : 0) * a.run] == token);
        const int c = same == ~0ull ? 64 : __ffsll((long long)~same) - 1;
        n += c;
        if (c < 64) break;
    }
    if (lane == 0) more[wave] = n;
    struct Values { float v[C]; };
    // slot 1 of its first run, slot 0 of the others
    auto partial = [&](int run, int slot) {
        Values p;
        const float* src = a.part + ((long long)run * 2 + slot) * a.dim + d;
        if constexpr (C > 1) load_values<C>(src, p.v);
        else p.v[0] = *src;
        return p;
    };
    auto finish = [&](uint32_t t, Values v) {
#pragma unroll
        for (int i = 0; i < C; ++i) v.v[i] *= a.scale;
        if (a.accumulate) {
            float old[C];
            load_result<D, C>(a, t, d, old);
#pragma unroll
            for (int i = 0; i < C; ++i) v.v[i] += old[i];
        }
        store_result<D, C>(a, t, d, v.v);
    };
    if (n > 0 && n <= kShort && d < a.dim) {
        Values v = partial(r, 1), p[kShort];
#pragma unroll
        for (int k = 0; k < kShort; ++k) p[k] = k < n ? partial(r + 1 + k, 0) : Values{};
#pragma unroll
        for (int k = 0; k < kShort; ++k)
#pragma unroll
            for (int i = 0; i < C; ++i) v.v[i] += p[k].v[i];
        finish(token, v);
    }
    __syncthreads();
    for (int w = 0; w < kJoinRuns; ++w) {
        const int m = more[w];
        if (m <= kShort) continue;
        const int share = (m + kJoinRuns - 1) / kJoinRuns, from = wave * share, to = min(m, from + share);
        Values v{};
        if (d < a.dim) {
            if (wave == 0) v = partial(r0 + w, 1);
#pragma unroll 8
            for (int k = from; k < to; ++k) {
                const Values p = partial(r0 + w + 1 + k, 0);
#pragma unroll
                for (int i = 0; i < C; ++i) v.v[i] += p.v[i];
            }
        }
#pragma unroll
        for (int i = 0; i < C; ++i) sums[wave][i][lane] = v.v[i];
        __syncthreads();
        if (wave == w && d < a.dim) {
#pragma unroll
            for (int i = 0; i < C; ++i) {
                v.v[i] = sums[0][i][lane];
                for (int k = 1; k < kJoinRuns; ++k) v.v[i] += sums[k][i][lane];
            }
            finish(token, v);
        }
        __syncthreads();
    }
}

// ---- gradient of few tokens ------------------------------------------------------------------------------------
// Workgroups of positions, each with a tile of columns, before those that write zeros.  The four waves share the positions of the token.
// Up to kFew: every workgroup looks at all tokens, and a token that most of them are is one workgroup's chain.  Sorted and in one launch,
// varied tokens: 172 x 772 14.7 and 4.4 us, 1000 x 256 14.6 and 7.9, 1000 x 2048 15.6 and 14.6, 2000 x 256 15.3 and 14.2.  The rule
// knows sizes, not tokens, and loses where one token is the whole batch: 512, 700 and 1000 x 256 of one 18, 24 and 34 us, 1000 sorted
// 15.  Batches vary, and padding that is named counts for nothing.
constexpr int kFew = 1024, kFewWaves = kThreads / 64;
template <typename O, typename D, int C, int P, bool ADD> __global__ __launch_bounds__(kThreads) void k_few(const SumArgs a, const SortArgs s) {
    __shared__ uint32_t key[kFew];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int j = threadIdx.x; j < s.n; j += kThreads) key[j] = key_of(s, s.tokens[j]);
    if ((int)blockIdx.x >= a.run_blocks) {
        __shared__ uint32_t present[kFillRows];
        const uint32_t v0 = (uint32_t)(blockIdx.x - a.run_blocks) * kFillRows;
        const int rows = (int)min((uint32_t)kFillRows, a.vocab - v0);
        if (threadIdx.x < kFillRows) present[threadIdx.x] = 0;
        __syncthreads();
        for (int j = threadIdx.x; j < s.n; j += kThreads)
            if (const uint32_t k = key[j] - v0; k < (uint32_t)rows) present[k] = 1;
        __syncthreads();
        write_zeros<D>(a, v0, rows, present);
        return;
    }
    __shared__ int list[kFew];
    __shared__ float sums[kFewWaves][P * C][64];
    const int i = blockIdx.x / a.column_tiles, tile = blockIdx.x - i * a.column_tiles;
    __syncthreads();
    const uint32_t token = key[i];
    int n = 0;
    bool first = token < a.vocab;
    for (int base = 0; base < s.n && first; base += 64) {
        const int j = base + lane;
        const bool same = j < s.n && key[j] == token;
        const unsigned long long with = __ballot(same);
        if (__ballot(same && j < i)) first = false;
        if (same && wave == 0) list[n + lanes_below(with)] = j;
        n += __popcll(with);
    }
    if (!first) return;                  // the same in all waves
    __syncthreads();
    const int d = tile * a.columns + lane * C, apart = 64 * C;
    int col[P];                          // a piece behind the row's end reads the row's first columns and writes nothing
    bool has[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        has[p] = d + p * apart < a.dim;
        col[p] = has[p] ? d + p * apart : 0;
    }
    float acc[P][C], old[P][C];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (ADD && wave == 0) load_result<D, C>(a, token, col[p], old[p]);
#pragma unroll
        for (int k = 0; k < C; ++k) acc[p][k] = 0.f;
    }
    const int share = (n + kFewWaves - 1) / kFewWaves, begin = wave * share, end = min(n, begin + share);
    const O* dout = static_cast<const O*>(a.dout);
    constexpr int U = 8;
    for (int e0 = begin; e0 < end; e0 += U) {
        Columns<O, C> v[U][P];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const O* row = dout + (long long)list[min(e0 + u, end - 1)] * a.out_stride;
#pragma unroll
            for (int p = 0; p < P; ++p) v[u][p].load(row + col[p]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (e0 + u < end) {
#pragma unroll
                for (int p = 0; p < P; ++p) v[u][p].add_to(acc[p]);
            }
    }
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int k = 0; k < C; ++k) sums[wave][p * C + k][lane] = acc[p][k];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int p = 0; p < P; ++p) {
#pragma unroll
        for (int k = 0; k < C; ++k) {
            for (int w = 1; w < kFewWaves; ++w) acc[p][k] += sums[w][p * C + k][lane];
            acc[p][k] = ADD ? acc[p][k] * a.scale + old[p][k] : acc[p][k] * a.scale;
        }
        if (has[p]) store_result<D, C>(a, token, col[p], acc[p]);
    }
}

// ---- host ----
asi_status check(const asi_embedding_desc* d) {
    if (!d) return ASI_ERR_INVALID_ARG;
    if (!dtype_ok(d->table_dtype) || !dtype_ok(d->out_dtype)) return ASI_ERR_UNSUPPORTED;
    if (d->tokens < 0 || d->vocab < 1 || d->dim < 1 || d->table_stride < d->dim || d->out_stride < d->dim || d->reserved) return ASI_ERR_INVALID_ARG;
    if (!std::isfinite(d->scale)) return ASI_ERR_INVALID_ARG;
    if (d->tokens >= (1LL << 30) || d->vocab > (1LL << 24) || d->dim > (1LL << 24)) return ASI_ERR_UNSUPPORTED;
    return ASI_OK;
}
// Entries of a run: short ones of few entries, where a run is a chain that nothing overlaps (954 x 1437 with 8, 16, 32 entries 19.0, 22.0,
// 29.2 us, 377 x 2501 16.4, 20.0, 27.2); longer ones, with fewer partial rows, where the chip is filled all the same (4096 x 2048
// 56.6, 53.0, 56.0; 25807 x 136 30.6, 28.0, 31.7; 32767 x 1000 72.7, 63.3, 57.7, with 64 62.4).
int run_length(const asi_embedding_desc* d) {
    if (d->tokens <= 2048) return 8;
    const long long row = (d->dim + 255) / 256;
    int run = 16;
    while (run < kMostRun && d->tokens / run * row > 4500) run *= 2;
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
// Columns of a piece and pieces of a lane: 16 bytes of the wider type, twice where the rows that are read are the narrower ones
template <typename O, typename D> struct Shape {
    static constexpr int C = sizeof(D) == 2 && sizeof(O) == 2 ? 8 : 4, P = sizeof(O) < sizeof(D) ? 2 : 1;
    static_assert(C * P == (sizeof(O) == 2 ? 8 : 4), "columns of a lane");
};
constexpr int kLoose = 4;             // pieces of a lane where they are single columns
// How the lanes of a workgroup share runs and columns, each lane `each` columns; false if that takes more workgroups than a launch has.
bool share_out(SumArgs* a, int each, int fill_blocks) {
    const bool few = a->n <= kFew;
    a->lanes = few ? 64 : kLeastLanes;
    while (!few && a->lanes < kThreads && a->lanes * each < a->dim) a->lanes *= 2;
    a->columns = a->lanes * each;
    a->column_tiles = (a->dim + a->columns - 1) / a->columns;
    const int groups = kThreads / a->lanes;
    const long long blocks = (long long)(few ? a->n : (a->runs + groups - 1) / groups) * a->column_tiles;
    if (blocks + fill_blocks > most_workgroups(kThreads)) return false;
    a->run_blocks = (int)blocks;
    return true;
}
template <typename O, typename D, int C, int P> void sum(const SumArgs& a, const SortArgs& s, int fill_blocks, hipStream_t st) {
    const dim3 grid((unsigned)(a.run_blocks + fill_blocks));
    if (a.n <= kFew) {
        if (a.accumulate) hipLaunchKernelGGL((k_few<O, D, C, P, true>), grid, kThreads, 0, st, a, s);
        else hipLaunchKernelGGL((k_few<O, D, C, P, false>), grid, kThreads, 0, st, a, s);
    } else {
        if (a.accumulate) hipLaunchKernelGGL((k_sum<O, D, C, P, true>), grid, kThreads, 0, st, a);
        else hipLaunchKernelGGL((k_sum<O, D, C, P, false>), grid, kThreads, 0, st, a);
    }
}
int join_tiles(const SumArgs& a, bool vec) { return (a.dim + (vec ? 256 : 64) - 1) / (vec ? 256 : 64); }
long long join_blocks(const SumArgs& a, int tiles) { return (long long)((a.runs - 1 + kJoinRuns - 1) / kJoinRuns) * tiles; }
template <typename D> void join(const SumArgs& a, bool vec, hipStream_t st) {
    const int tiles = join_tiles(a, vec);
    const dim3 grid((unsigned)join_blocks(a, tiles));
    if (vec) hipLaunchKernelGGL((k_join<D, 4>), grid, kJoinThreads, 0, st, a, tiles);
    else hipLaunchKernelGGL((k_join<D, 1>), grid, kJoinThreads, 0, st, a, tiles);
}
template <typename O, typename D> void sum(const SumArgs& a, const SortArgs& s, bool vec, int fill_blocks, hipStream_t st) {
    if (vec) sum<O, D, Shape<O, D>::C, Shape<O, D>::P>(a, s, fill_blocks, st);
    else sum<O, D, 1, kLoose>(a, s, fill_blocks, st);
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
    // a launch's worth of tokens at a time
    const long long most = most_workgroups(kThreads) * (kThreads / 64) / a.parts;
    hipStream_t st = static_cast<hipStream_t>(stream);
    for (long long t = 0; t < desc->tokens; t += most) {
        a.n = std::min<long long>(most, desc->tokens - t);
        a.tokens = tokens + t;
        a.out = static_cast<char*>(out) + t * desc->out_stride * (long long)os;
        const dim3 grid((unsigned)((a.n * a.parts + 3) / 4));
        if (desc->table_dtype == ASI_F32) {
            if (desc->out_dtype == ASI_F32) lookup<float, float>(a, vec, grid, st);
            else lookup<float, bf16_t>(a, vec, grid, st);
        } else {
            if (desc->out_dtype == ASI_F32) lookup<bf16_t, float>(a, vec, grid, st);
            else lookup<bf16_t, bf16_t>(a, vec, grid, st);
        }
    }
    return launched();
}

size_t asi_embedding_grad_workspace_bytes(const asi_embedding_desc* desc) {
    if (check(desc) != ASI_OK || desc->tokens <= kFew) return 0;
    return plan(desc).bytes;
}

asi_status asi_embedding_grad(const asi_embedding_desc* desc, const int64_t* tokens, const void* grad_out, void* dtable,
                              int accumulate, void* ws, size_t ws_bytes, asi_stream_t stream) {
    if (asi_status why = check(desc); why != ASI_OK) return why;
    const size_t ds = dtype_size(desc->table_dtype), os = dtype_size(desc->out_dtype);
    if (!dtable || !aligned(dtable, ds)) return ASI_ERR_INVALID_ARG;
    if (desc->tokens && (!tokens || !grad_out || !aligned(tokens, 8) || !aligned(grad_out, os))) return ASI_ERR_INVALID_ARG;
    const GradPlan p = plan(desc);
    const bool few = desc->tokens <= kFew;
    if (!few && (!ws || !aligned(ws, 256) || ws_bytes < p.bytes)) return ASI_ERR_WORKSPACE;
    if (desc->tokens == 0 && accumulate) return ASI_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* w = static_cast<char*>(ws);
    SumArgs a{};
    if (!few) {
        a.key = reinterpret_cast<uint32_t*>(w + p.key);
        a.pos = reinterpret_cast<uint32_t*>(w + p.pos);
        a.part = reinterpret_cast<float*>(w + p.part);
    }
    a.dout = grad_out; a.dtable = dtable;
    a.out_stride = desc->out_stride; a.table_stride = desc->table_stride;
    a.vocab = (uint32_t)desc->vocab;
    a.n = (int)desc->tokens; a.run = p.run; a.runs = p.runs; a.dim = (int)desc->dim;
    a.accumulate = accumulate != 0;
    a.scale = desc->scale;
    // whole pieces: 4 columns, 8 where both types are bf16
    const int piece = ds == 2 && os == 2 ? 8 : 4;
    const bool vec = desc->dim % piece == 0 && desc->out_stride % piece == 0 && desc->table_stride % piece == 0 && aligned(grad_out, piece * os) && aligned(dtable, piece * ds);
    const int fill_blocks = accumulate ? 0 : (int)((desc->vocab + kFillRows - 1) / kFillRows);
    const int each = !vec ? kLoose : os == 2 ? 8 : 4;        // C * P
    if (!share_out(&a, each, fill_blocks) || join_blocks(a, join_tiles(a, vec)) > most_workgroups(kJoinThreads)) return ASI_ERR_UNSUPPORTED;
    const bool padded = desc->padding_index >= 0 && desc->padding_index < desc->vocab;
    SortArgs s{tokens, nullptr, nullptr, padded ? (uint32_t)desc->padding_index : a.vocab, a.vocab, a.n, 0};
    if (!few) {
        // about one workgroup a CU; the id `vocab` is one more
        const long long ids = desc->vocab + 1;
        s.key = reinterpret_cast<uint32_t*>(w + p.key);
        s.pos = reinterpret_cast<uint32_t*>(w + p.pos);
        s.span = (int)std::min<long long>(kMaxSpan, (ids + 255) / 256);
        constexpr size_t lists = (size_t)kSortWaves * kSortList * 4;
        static LdsAllowed allowed;
        if (allow_lds(reinterpret_cast<const void*>(k_sort), (size_t)kSortWaves * kMaxSpan * 4 + lists, allowed) != hipSuccess) return ASI_ERR_HIP;
        hipLaunchKernelGGL(k_sort, dim3((unsigned)((ids + s.span - 1) / s.span)), kSortThreads, (size_t)kSortWaves * s.span * 4 + lists, st, s);
    }
    if (desc->out_dtype == ASI_F32) {
        if (desc->table_dtype == ASI_F32) sum<float, float>(a, s, vec, fill_blocks, st);
        else sum<float, bf16_t>(a, s, vec, fill_blocks, st);
    } else {
        if (desc->table_dtype == ASI_F32) sum<bf16_t, float>(a, s, vec, fill_blocks, st);
        else sum<bf16_t, bf16_t>(a, s, vec, fill_blocks, st);
    }
    if (!few && p.runs > 1) {
        if (desc->table_dtype == ASI_F32) join<float>(a, vec, st);
        else join<bf16_t>(a, vec, st);
    }
    return launched();
}

}  // extern "C"
