// Token log probabilities from hidden states and the output layer's weights, and their gradients, without the logits
// (include/asi_lm.h, asi_linear_logprobs).
//
//   k_live        the rows that have a target, in order, and how many: every kernel behind it reads that number, the host does not
//   k_pack        their hidden states next to each other, k filled up with zeros to whole steps; fp32 as three planes of bf16.  The
//                 same for a piece of the weights where they cannot be read as they lie (fp32, rows that are no whole vectors)
//   k_logits      a tile of logits, vocabulary along the registers of a lane and tokens along the lanes, so that a token's maximum
//                 and sums over 128 (64) of the vocabulary stay in a lane but for one exchange.  Values: (x_max, sum e, sum e d) of
//                 each token, d = x - x_max, e = exp(scale d), and the target's logit.  Gradient: dz, rounded to bf16
//   k_few         the same values for up to 16 rows, the weights from memory straight into the matrix instructions
//   k_join        joins the tiles' values
//   k_products    the products of dz with weights (dH) and hidden states (dW), read across as they lie (asi_tiles.h)
//   k_hidden      the sums of dH, in fp32 over the pieces of the vocabulary and the parts of a piece, to their rows
//
// What bounds it: the matrix products, 2 rows dim vocab for the values and 8 with the gradients (6 if the logits were kept); the
// weights' memory for few rows.
#include <math.h>

#include "asi_lds.h"
#include "asi_tiles.h"

namespace asi {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLow = -1e30f;                       // stands for -infinity where that is multiplied by 0
constexpr int kFew = 16;                             // rows of k_few
constexpr size_t kPieceBytes = size_t(96) << 20;     // dz of a piece, in bf16

// Tiles of 256 x 256 by 8 waves where they fill the chip (8190 x 2048 logits of 100003: 2.76 ms, with tiles of 128 3.26), of 128 x 128 by
// 4 waves, two workgroups a CU, where they would not.
template <int B> struct Shape {
    static constexpr int WN = B == 256 ? 4 : 2, kThreads = 128 * WN, kSlots = B == 256 ? 256 : 512;
    template <bool A, bool X> using Of = Tile<B, B, A, X, WN>;
    static constexpr size_t kLds = 4 * B * kStep * 2 > B * (2 * B + 16) ? 4 * B * kStep * 2 : B * (2 * B + 16);      // two buffers, or a tile in bf16
};

// What the gradient needs of a row: p = exp2(scale' (x - top) - log2sum); dz = [target] a - p (a + b (log p + entropy))
struct RowInfo {
    float top, log2sum, a, b, entropy;
    int target, pad[2];
};

// ---- rows ---------------------------------------------------------------------------------------------------
// What follows from the number of live rows, which the GPU alone knows.
struct Split {
    int rows, piece, splits, pad;                    // live rows; tokens of a piece; parts that the vocabulary of a piece is cut in for dH
};
struct SplitArgs {
    long long vocab, dim, elements, piece, most_sums, most_splits;      // elements of dz and rows of sums that there is memory for
    int tile, pairs;
    bool grad, flexible, dhidden, dweight;           // flexible: pieces may be larger than `piece` where rows are fewer
};
// The number of parts that ends a launch of dH's tiles, then dW's, soonest, `slots` workgroups at a time: lengths in steps of 64 k, to which
// writing a tile adds about 6.  A lane of the wave for each number of parts.  (2731 x 2048 x 32000: 1434 us with two parts, 1508 with one.)
__device__ int best_splits(const SplitArgs& a, long long rows, long long piece) {
    const int s = (int)(threadIdx.x & 63) + 1;
    const float slots = a.tile == 256 ? 256.f : 512.f, row_tiles = (float)((rows + a.tile - 1) / a.tile), dim_tiles = (float)((a.dim + a.tile - 1) / a.tile);
    const long long v = a.vocab < piece ? a.vocab : piece;
    const float steps = (float)((v + kStep - 1) / kStep), w_units = a.dweight ? (float)((v + a.tile - 1) / a.tile) * dim_tiles : 0.f;
    const float w = (float)((rows + kStep - 1) / kStep) * a.pairs + 6.f, h = ceilf(steps / s) * a.pairs + 6.f;
    const float units = row_tiles * dim_tiles * s, whole = floorf(units / slots), late = units - whole * slots, start = whole * h;
    float end = fmaxf(start + (late > 0.f ? h : 0.f), (units * h + w_units * w) / slots);
    for (int i = 0; i < 64; ++i) {                   // until the slots that are free after `whole` tiles of dH and after one more can take dW's
        const float room = (slots - late) * floorf((end - start) / w) + late * floorf(fmaxf(end - start - h, 0.f) / w);
        if (room >= w_units) break;
        end += 0.125f * w;
    }
    const bool may = s <= a.most_splits && s * rows <= a.most_sums && (s == 1 || steps >= 8.f * s);
    // positive numbers order as their bits do; the lane in the last bits, so that of equal ends the fewest parts are taken
    uint32_t key = may ? (__float_as_uint(end) & ~63u) | (uint32_t)(s - 1) : 0xffffffffu;
    return (int)((~wave_max(~key)) & 63u) + 1;
}
// By a whole wave.
__device__ void split_rows(const SplitArgs& a, long long rows, Split* to) {
    Split p{(int)rows, (int)a.piece, 1, 0};
    if (a.grad && rows > 0) {
        if (a.flexible) {
            const long long up = (rows + a.tile - 1) / a.tile * a.tile, all = (a.vocab + 255) / 256 * 256;
            long long size = a.elements / up / 256 * 256;
            if (size > 2 * a.piece) size = 2 * a.piece;
            if (size > all) size = all;
            const long long pieces = (a.vocab + size - 1) / size;
            p.piece = (int)((a.vocab + pieces * 256 - 1) / (pieces * 256) * 256);
        }
        p.splits = best_splits(a, rows, p.piece);
    }
    if ((threadIdx.x & 63) == 0) *to = p;
}
struct LiveArgs {
    const int64_t* targets;
    long long rows, ignore;
    Split* split;
    int *live, *place;                               // place[row]: its place among the live ones, -1 if it is left out
    float *logprob, *entropy, *stats;                // 0 for a row that is left out; nullable
    SplitArgs how;
};
__global__ __launch_bounds__(1024) void k_live(const LiveArgs a) {
    __shared__ int waves[16];
    const long long each = (a.rows + 1023) / 1024, from = threadIdx.x * each, to = from + each < a.rows ? from + each : a.rows;
    int mine = 0;
    for (long long r = from; r < to; ++r) mine += a.targets[r] != a.ignore;
    int before = mine;                               // of this lane and those before it in the wave
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(before, o);
        if (lane >= o) before += x;
    }
    if (lane == 63) waves[threadIdx.x >> 6] = before;
    __syncthreads();
    int at = before - mine, all = 0;
    for (int w = 0; w < 16; ++w) {
        if (w < (int)(threadIdx.x >> 6)) at += waves[w];
        all += waves[w];
    }
    for (long long r = from; r < to; ++r) {
        const bool lives = a.targets[r] != a.ignore;
        a.place[r] = lives ? at : -1;
        if (lives) a.live[at++] = (int)r;
        else {
            if (a.logprob) a.logprob[r] = 0.f;
            if (a.entropy) a.entropy[r] = 0.f;
            if (a.stats) a.stats[2 * r] = a.stats[2 * r + 1] = 0.f;
        }
    }
    if (threadIdx.x < 64) split_rows(a.how, all, a.split);
}
__global__ __launch_bounds__(256) void k_all_live(const LiveArgs a) {
    const long long r = (long long)blockIdx.x * 256 + threadIdx.x;
    if (r < a.rows) a.live[r] = a.place[r] = (int)r;
    if (r < 64) split_rows(a.how, a.rows, a.split);
}

// ---- operands -----------------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ void planes_of(float x, uint16_t* h) {
    h[0] = to_bf16(x).bits;
    if constexpr (sizeof(T) == 4) {
        // what bf16 leaves out is exact in fp32; of an infinity or NaN the first plane says all
        const float r = x - to_f32(bf16_t{h[0]}), q = r - to_f32(to_bf16(r));
        const bool fine = fabsf(to_f32(bf16_t{h[0]})) <= 3.4e38f;
        h[1] = fine ? to_bf16(r).bits : 0;
        h[2] = fine ? to_bf16(q).bits : 0;
    }
}
struct PackArgs {
    const void* x;
    long long stride, rows;                          // rows are at least those that are packed
    const Split* split;                              // nullable, with live: all rows
    const int* live;
    int dim, pieces;                                 // pieces of 8 of a packed row
    uint16_t* out;
    long long ld, plane;
    bool whole;                                      // rows are whole vectors
};
template <typename T> __global__ __launch_bounds__(256) void k_pack(const PackArgs a) {
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, row = at / a.pieces;
    const int col = (int)(at - row * a.pieces) * 8;
    if (row >= (a.split ? a.split->rows : a.rows)) return;
    const T* x = static_cast<const T*>(a.x) + (a.live ? a.live[row] : row) * a.stride + col;
    float f[8];
    if (a.whole && col + 8 <= a.dim) {
        load_values<8>(x, f);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = col + e < a.dim ? to_f32(x[e]) : 0.f;
    }
    constexpr int planes = sizeof(T) == 4 ? kPlanes : 1;
    uint16_t h[8][3];
#pragma unroll
    for (int e = 0; e < 8; ++e) planes_of<T>(f[e], h[e]);
#pragma unroll
    for (int p = 0; p < planes; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = h[2 * e][p] | ((uint32_t)h[2 * e + 1][p] << 16);
        store_words(a.out + p * a.plane + row * a.ld + col, make_uint4(w[0], w[1], w[2], w[3]));
    }
}

// ---- logits -------------------------------------------------------------------------------------------------
// Which tile of m_tiles x n_tiles is this workgroup's: every XCD (workgroups go round the eight of them) has a run of tiles, in which
// `group` tiles along m and all along n follow each other, so that what an XCD works on at a time meets in its L2.  False: none.
__device__ __forceinline__ bool my_tile(long long id, long long m_tiles, long long n_tiles, int group, long long* m, long long* n) {
    const long long total = m_tiles * n_tiles, q = total / 8, left = total % 8, xcd = id % 8, i = id / 8;
    if (i >= q + (xcd < left ? 1 : 0)) return false;
    const long long at = xcd * q + (xcd < left ? xcd : left) + i, g = at / (group * n_tiles), in = at - g * group * n_tiles;
    const long long high = m_tiles - g * group < group ? m_tiles - g * group : group;
    *n = in / high;
    *m = g * group + in - *n * high;
    return true;
}

struct LogitArgs {
    Operand w, h;                                    // weights, of the whole vocabulary or of a packed piece; the live rows' hidden states
    const Split* split;
    int k_steps;
    long long vocab, first;                          // tokens of the piece; its first one
    long long all;                                   // tokens of the vocabulary where the GPU decides on the pieces; 0: it does not
    int number;                                      // the piece's
    float scale;
    // values: [tile][top, sum, along][rows], the targets' logits [rows]
    const int *live;
    const int64_t* targets;
    float *part, *target_logit;
    long long part_rows, first_part;
    // gradient
    const RowInfo* info;
    uint16_t* dz;                                    // [row][dz_stride], planes apart
    long long dz_stride, dz_plane;
};

constexpr int pairs_of(int planes) { return planes == 1 ? 1 : kPairs; }
// The piece that is asked for, as decided on the GPU; `w`: the weights, moved on to it.  False: there is no such piece.
__device__ __forceinline__ bool my_piece(const Split& s, long long all, int number, long long* first, long long* n, Operand* w) {
    if (!all) return true;
    *first = (long long)number * s.piece;
    *n = all - *first < s.piece ? all - *first : s.piece;
    if (*n <= 0) return false;
    w->p += *first * w->ld;
    w->rows = *n;
    return true;
}

struct Joined {
    float top, sum, along;
};
// of two sets of logits: the largest, sum exp(scale d) and sum exp(scale d) d with d = x - top
__device__ __forceinline__ Joined join(Joined a, Joined b, float c) {
    const float top = fmaxf(a.top, b.top), base = top == -INFINITY ? 0.f : top;
    const float da = fmaxf(a.top - base, kLow), db = fmaxf(b.top - base, kLow);
    const float ea = __builtin_amdgcn_exp2f(da * c), eb = __builtin_amdgcn_exp2f(db * c);
    // sums that are NaN stay NaN: they are multiplied, not compared
    return Joined{top, a.sum * ea + b.sum * eb, ea * fmaf(a.sum, da, a.along) + eb * fmaf(b.sum, db, b.along)};
}

template <int B, int PLANES> __global__ __launch_bounds__(Shape<B>::kThreads, 2) void k_logits(const LogitArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int BM = B, BN = B;
    using Tl = typename Shape<B>::template Of<false, false>;
    const long long rows = a.split->rows;
    long long tm, tn;
    if (!my_tile(blockIdx.x, (a.vocab + BM - 1) / BM, (rows + BN - 1) / BN, 1024 / BM, &tm, &tn)) return;
    Tl t;
    t.clear();
    Operand h = a.h;
    h.rows = rows;
    t.template run<pairs_of(PLANES)>(a.w, h, tm * BM, tn * BN, 0, a.k_steps, lds);
    __syncthreads();
    const float c = a.scale * kLog2e;
    const int lane = threadIdx.x & 63;
    const long long v0 = tm * BM + Tl::at_m();       // this wave's first token of the piece
    if (v0 + BM / 2 > a.vocab) {                     // behind the vocabulary's end
#pragma unroll
        for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (v0 + 32 * i + Tl::row_of(r) >= a.vocab) {
#pragma unroll
                    for (int j = 0; j < Tl::kN; ++j) t.acc[i][j][r] = -INFINITY;
                }
    }
    Joined* shared = reinterpret_cast<Joined*>(lds);
#pragma unroll
    for (int j = 0; j < Tl::kN; ++j) {
        const int col = Tl::at_n() + 32 * j + (lane & 31);
        const long long row = tn * BN + col;
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, t.acc[i][j][r]);
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = top == -INFINITY ? 0.f : top;
        float sum = 0.f, along = 0.f;
#pragma unroll
        for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float d = max_nan(t.acc[i][j][r] - base, kLow), e = __builtin_amdgcn_exp2f(d * c);
                sum += e;
                along = fmaf(e, d, along);
            }
        sum += __shfl_xor(sum, 32);
        along += __shfl_xor(along, 32);
        if (lane < 32) shared[Tl::wave_m() * BN + col] = Joined{top, sum, along};
        if (a.targets) {
            const long long target = row < rows ? a.targets[a.live[row]] - a.first - v0 : -1;
            if (__any(target >= 0 && target < BM / 2)) {
#pragma unroll
                for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (target == 32 * i + Tl::row_of(r)) a.target_logit[row] = t.acc[i][j][r];
            }
        }
    }
    __syncthreads();
    if (threadIdx.x < BN) {
        const long long row = tn * BN + threadIdx.x;
        if (row < rows) {
            const Joined x = join(shared[threadIdx.x], shared[BN + threadIdx.x], c);
            float* to = a.part + (a.first_part + tm) * 3 * a.part_rows + row;
            to[0] = x.top;
            to[a.part_rows] = x.sum;
            to[2 * a.part_rows] = x.along;
        }
    }
}

// Writes a tile whose lanes hold four neighbours along m for a column n as rows n of BM values, through LDS so that whole lines are
// stored: `value(i, j, r)` gives it as bf16 bits.
template <typename Tl, int BM, int BN, typename F> __device__ __forceinline__ void store_across(char* lds, uint16_t* out, long long stride, long long n_left, long long m_left, bool whole, F value) {
    constexpr int pitch = BM * 2 + 16;
    const int lane = threadIdx.x & 63;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < Tl::kN; ++j)
#pragma unroll
        for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const uint32_t lo = value(i, j, r) | (value(i, j, r + 1) << 16), hi = value(i, j, r + 2) | (value(i, j, r + 3) << 16);
                store_words(lds + (Tl::at_n() + 32 * j + (lane & 31)) * pitch + (Tl::at_m() + 32 * i + Tl::row_of(r)) * 2, make_uint2(lo, hi));
            }
    __syncthreads();
    constexpr int pieces = BM / 8;
    if (whole) {
#pragma unroll 4
        for (int at = threadIdx.x; at < BN * pieces; at += Tl::kThreads) {
            const int n = at / pieces, piece = at % pieces;
            if (n < n_left && piece * 8 < m_left) store_words(out + n * stride + piece * 8, load_words4(lds + n * pitch + piece * 16));
        }
    } else {
        for (int at = threadIdx.x; at < BN * BM; at += Tl::kThreads) {
            const int n = at / BM, m = at % BM;
            if (n < n_left && m < m_left) out[n * stride + m] = *reinterpret_cast<const uint16_t*>(lds + n * pitch + m * 2);
        }
    }
}

template <int B, int PLANES> __global__ __launch_bounds__(Shape<B>::kThreads, 2) void k_logits_grad(const LogitArgs given) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int BM = B, BN = B;
    using Tl = typename Shape<B>::template Of<false, false>;
    LogitArgs a = given;
    const Split split = *a.split;
    const long long rows = split.rows;
    if (!my_piece(split, a.all, a.number, &a.first, &a.vocab, &a.w)) return;
    a.dz_stride = split.piece;
    long long tm, tn;
    if (!my_tile(blockIdx.x, (a.vocab + BM - 1) / BM, (rows + BN - 1) / BN, 1024 / BM, &tm, &tn)) return;
    Tl t;
    t.clear();
    Operand h = a.h;
    h.rows = rows;
    t.template run<pairs_of(PLANES)>(a.w, h, tm * BM, tn * BN, 0, a.k_steps, lds);
    const float c = a.scale * kLog2e;
    const int lane = threadIdx.x & 63;
    const long long v0 = tm * BM + Tl::at_m();
#pragma unroll
    for (int j = 0; j < Tl::kN; ++j) {
        const long long row = tn * BN + Tl::at_n() + 32 * j + (lane & 31);
        RowInfo f{0.f, INFINITY, 0.f, 0.f, 0.f, -1, {0, 0}};
        if (row < rows) f = a.info[row];
        const long long target = f.target >= 0 ? f.target - a.first - v0 : -1;
        if (__any(f.b != 0.f)) {                     // NaN too
#pragma unroll
            for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float x = fmaf(t.acc[i][j][r] - f.top, c, -f.log2sum), p = __builtin_amdgcn_exp2f(x);
                    t.acc[i][j][r] = -p * fmaf(f.b, fmaf(max_nan(x, kLow), 1.f / kLog2e, f.entropy), f.a);
                }
        } else {
#pragma unroll
            for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) t.acc[i][j][r] = -f.a * __builtin_amdgcn_exp2f(fmaf(t.acc[i][j][r] - f.top, c, -f.log2sum));
        }
        if (__any(target >= 0 && target < BM / 2)) {
#pragma unroll
            for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (target == 32 * i + Tl::row_of(r)) t.acc[i][j][r] += f.a;
        }
    }
    if (v0 + BM / 2 > a.vocab) {                     // behind the vocabulary's end
#pragma unroll
        for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (v0 + 32 * i + Tl::row_of(r) >= a.vocab) {
#pragma unroll
                    for (int j = 0; j < Tl::kN; ++j) t.acc[i][j][r] = 0.f;
                }
    }
#pragma unroll
    for (int p = 0; p < PLANES; ++p)
        store_across<Tl, BM, BN>(lds, a.dz + p * a.dz_plane + tn * BN * a.dz_stride + tm * BM, a.dz_stride, rows - tn * BN, BM, true,
                                 [&](int i, int j, int r) -> uint32_t {
                                     const uint32_t bits = to_bf16(t.acc[i][j][r]).bits;
                                     if (p + 1 < PLANES) t.acc[i][j][r] -= __uint_as_float(bits << 16);
                                     return bits;
                                 });
}

// ---- few rows -----------------------------------------------------------------------------------------------
// Logits of up to 16 rows: a wave takes 16 of the vocabulary and all k, both operands from memory straight into the registers of the
// matrix instruction, a token along four lanes.  What bounds it: the weights' memory.
struct FewArgs {
    const void *h, *w;
    long long h_stride, w_stride, vocab, rows, first_row;
    int dim;
    bool whole;
    float scale;
    const int64_t* targets;
    long long ignore;
    float *part, *target_logit;
    long long part_rows;
};
typedef float v4f __attribute__((ext_vector_type(4)));
constexpr int kFewWaves = 4, kFewAhead = 8;
template <typename T> struct FewStep;               // the k of a wave's load of 16 bytes a lane
template <> struct FewStep<bf16_t> { static constexpr int k = 32; };
template <> struct FewStep<float> { static constexpr int k = 16; };
__device__ __forceinline__ v4f few_product(const Vec16<bf16_t>& w, const Vec16<bf16_t>& h, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, w.raw), __builtin_bit_cast(v8bf, h.raw), c, 0, 0, 0);
}
__device__ __forceinline__ v4f few_product(const Vec16<float>& w, const Vec16<float>& h, v4f c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w.get(i), h.get(i), c, 0, 0, 0);
    return c;
}
template <typename T> __device__ __forceinline__ Vec16<T> few_load(const T* p, int k, int dim, bool there, bool whole) {
    Vec16<T> v;
    v.raw = make_uint4(0, 0, 0, 0);
    if (there && k < dim) {
        if (whole && k + Vec16<T>::N <= dim) {
            v.load(p + k);
        } else {
            float f[Vec16<T>::N];
#pragma unroll
            for (int e = 0; e < Vec16<T>::N; ++e) f[e] = k + e < dim ? to_f32(p[k + e]) : 0.f;
            v.set(f);
        }
    }
    return v;
}
template <typename T> __global__ __launch_bounds__(64 * kFewWaves) void k_few(const FewArgs a) {
    __shared__ Joined shared[kFewWaves][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15;
    const long long v0 = ((long long)blockIdx.x * kFewWaves + wave) * 16, row = a.first_row + col;
    const bool w_there = v0 + col < a.vocab, h_there = row < a.rows;
    const T* w = static_cast<const T*>(a.w) + (v0 + col) * a.w_stride;
    const T* h = static_cast<const T*>(a.h) + row * a.h_stride;
    constexpr int step = FewStep<T>::k;
    v4f acc = {0.f, 0.f, 0.f, 0.f};
    int k = (lane >> 4) * Vec16<T>::N;
    for (int at = 0; at < a.dim; at += step * kFewAhead) {
        Vec16<T> wv[kFewAhead], hv[kFewAhead];
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u) wv[u] = few_load(w, at + u * step + k, a.dim, w_there, a.whole);
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u) hv[u] = few_load(h, at + u * step + k, a.dim, h_there, a.whole);
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u) acc = few_product(wv[u], hv[u], acc);
    }
    // a lane has tokens v0 + 4 (lane / 16) + r of row `col`
    const float c = a.scale * kLog2e;
    const long long first = v0 + 4 * (lane >> 4);
    float top = -INFINITY;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (first + r >= a.vocab) acc[r] = -INFINITY;
        top = fmaxf(top, acc[r]);
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f, along = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float d = max_nan(acc[r] - base, kLow), e = __builtin_amdgcn_exp2f(d * c);
        sum += e;
        along = fmaf(e, d, along);
    }
    sum += __shfl_xor(sum, 16);
    along += __shfl_xor(along, 16);
    sum += __shfl_xor(sum, 32);
    along += __shfl_xor(along, 32);
    if (lane < 16) shared[wave][lane] = Joined{top, sum, along};
    if (a.targets && h_there) {
        const long long target = a.targets[row] - first;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (target == r && first + r < a.vocab) a.target_logit[row] = acc[r];
    }
    __syncthreads();
    if (threadIdx.x < 16 && h_there) {
        Joined x = shared[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < kFewWaves; ++i) x = join(x, shared[i][threadIdx.x], c);
        float* to = a.part + (long long)blockIdx.x * 3 * a.part_rows + row;
        to[0] = x.top;
        to[a.part_rows] = x.sum;
        to[2 * a.part_rows] = x.along;
    }
}

// ---- joining ------------------------------------------------------------------------------------------------
struct JoinArgs {
    const float *part, *target_logit;
    long long part_rows, parts, vocab, ignore;
    const Split* split;                              // nullable, with live: all `rows` rows as they are
    const int* live;
    long long rows;
    const int64_t* targets;
    float scale;
    float *logprob, *entropy, *stats;
    RowInfo* info;                                   // nullable; with it the weights
    const float *a, *b;
};
__device__ __forceinline__ void write_info(RowInfo* to, float top, float logsum, float entropy, float a, float b, float scale, int64_t target, long long vocab, bool given) {
    RowInfo f{top, logsum * kLog2e, a * scale, b * scale, entropy, (int)target, {0, 0}};
    if (top == -INFINITY) f = RowInfo{0.f, INFINITY, 0.f, 0.f, 0.f, -1, {0, 0}};      // nothing but -infinity: no gradient
    if (given && (target < 0 || target >= vocab)) { f.target = -1; f.log2sum = NAN; }
    if (!given) f.target = -1;
    *to = f;
}
// ROWS rows a workgroup, the parts of each shared out to 256 / ROWS threads
template <int ROWS> __global__ __launch_bounds__(256) void k_join(const JoinArgs a) {
    constexpr int kShares = 256 / ROWS;
    __shared__ Joined shared[kShares][ROWS];
    const int in = threadIdx.x % ROWS, share = threadIdx.x / ROWS;
    const long long rows = a.split ? a.split->rows : a.rows, at = (long long)blockIdx.x * ROWS + in;
    if ((long long)blockIdx.x * ROWS >= rows) return;
    const float c = a.scale * kLog2e;
    float top = -INFINITY;
    const float* p = a.part + at;
    if (at < rows)
        for (long long i = share; i < a.parts; i += kShares) top = fmaxf(top, p[i * 3 * a.part_rows]);
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f, along = 0.f;
    if (at < rows)
#pragma unroll 4
        for (long long i = share; i < a.parts; i += kShares) {
            const float* q = p + i * 3 * a.part_rows;
            const float d = fmaxf(q[0] - base, kLow), e = __builtin_amdgcn_exp2f(d * c), s = q[a.part_rows];
            sum = fmaf(s, e, sum);
            along = fmaf(fmaf(s, d, q[2 * a.part_rows]), e, along);
        }
    shared[share][in] = Joined{top, sum, along};
    __syncthreads();
    for (int n = kShares / 2; n; n >>= 1) {
        if (share < n) shared[share][in] = join(shared[share][in], shared[share + n][in], c);
        __syncthreads();
    }
    if (share || at >= rows) return;
    const Joined x = shared[0][in];
    const long long row = a.live ? a.live[at] : at;
    const bool empty = x.top == -INFINITY && !(x.sum != x.sum);
    const float logsum = empty ? 0.f : logf(x.sum), entropy = empty ? 0.f : fmaxf(logsum - a.scale * (x.along / x.sum), 0.f) + (x.sum - x.sum);
    const int64_t target = a.targets ? a.targets[row] : 0;
    const bool left_out = a.targets && target == a.ignore;      // where the rows have not been sorted out
    if (a.logprob) {
        float v = NAN;
        if (target >= 0 && target < a.vocab) v = empty ? -INFINITY : fmaf(a.scale, a.target_logit[at] - x.top, -logsum);
        if (x.sum != x.sum) v = NAN;
        a.logprob[row] = left_out ? 0.f : v;
    }
    if (a.entropy) a.entropy[row] = left_out ? 0.f : entropy;
    if (a.stats) {
        a.stats[2 * row] = left_out ? 0.f : x.top;
        a.stats[2 * row + 1] = left_out ? 0.f : logsum;
    }
    if (a.info) write_info(a.info + at, x.top, logsum, entropy, a.a ? a.a[row] : 0.f, a.b ? a.b[row] : 0.f, a.scale, target, a.vocab, a.targets != nullptr);
}

struct InfoArgs {
    const Split* split;
    const int* live;
    const int64_t* targets;
    const float *stats, *entropy, *a, *b;
    float scale;
    long long vocab;
    RowInfo* info;
};
__global__ __launch_bounds__(256) void k_info(const InfoArgs a) {
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at >= a.split->rows) return;
    const long long row = a.live[at];
    write_info(a.info + at, a.stats[2 * row], a.stats[2 * row + 1], a.b ? a.entropy[row] : 0.f, a.a ? a.a[row] : 0.f, a.b ? a.b[row] : 0.f, a.scale,
               a.targets ? a.targets[row] : 0, a.vocab, a.targets != nullptr);
}

// ---- the gradients' products ----------------------------------------------------------------------------------
struct ProductArgs {
    Operand dz, weights, hidden;                     // dz of the piece, weights as k_logits has them, hidden states
    const Split* split;
    long long vocab, first, all, dim;                // as k_logits has them
    int number;
    bool dhidden, dweight;
    // dH: sums in fp32, [part][live row][dim]
    float* sums;
    bool add;
    void* dw;                                        // all rows of dW
    bool whole;
};

// dH: rows along m, dim along n, the piece's vocabulary along k in `splits` parts
template <int B, int PLANES> __device__ __forceinline__ void dhidden_tile(const ProductArgs& a, long long id, long long rows, int splits, char* lds) {
    constexpr int BM = B, BN = B;
    using Tl = typename Shape<B>::template Of<false, true>;
    const long long n_tiles = (a.dim + BN - 1) / BN;
    long long tm, tn;
    if (!my_tile(id, (rows + BM - 1) / BM, n_tiles * splits, 1024 / BM, &tm, &tn)) return;
    const int split = (int)(tn / n_tiles);
    tn -= split * n_tiles;
    const int steps = (int)((a.vocab + kStep - 1) / kStep), from = (int)((long long)steps * split / splits), to = (int)((long long)steps * (split + 1) / splits);
    Tl t;
    t.clear();
    Operand dz = a.dz;
    dz.rows = rows;
    if (to > from) t.template run<pairs_of(PLANES)>(dz, a.weights, tm * BM, tn * BN, from, to - from, lds);
    float* out = a.sums + split * rows * a.dim;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const long long row = tm * BM + Tl::at_m() + 32 * i + Tl::row_of(r);
            if (row >= rows) continue;
#pragma unroll
            for (int j = 0; j < Tl::kN; ++j) {
                const long long col = tn * BN + Tl::at_n() + 32 * j + (lane & 31);
                if (col < a.dim) {
                    float* p = out + row * a.dim + col;
                    *p = a.add ? *p + t.acc[i][j][r] : t.acc[i][j][r];
                }
            }
        }
}

// dW: the rows are k.  bf16: dim along m, so that a lane has neighbours of a row of dW; fp32: dim along n, a line of a row a store
template <int B, typename T> __device__ __forceinline__ void dweight_tile(const ProductArgs& a, long long id, long long rows, char* lds) {
    constexpr int BM = B, BN = B;
    using Tl = typename Shape<B>::template Of<true, true>;
    constexpr bool kDimFirst = sizeof(T) == 2;
    const long long m_size = kDimFirst ? a.dim : a.vocab, n_size = kDimFirst ? a.vocab : a.dim;
    long long tm, tn;
    if (!my_tile(id, (m_size + BM - 1) / BM, (n_size + BN - 1) / BN, 1024 / BM, &tm, &tn)) return;
    Tl t;
    t.clear();
    Operand dz = a.dz, x = a.hidden;
    dz.rows = x.rows = rows;
    const int steps = (int)((rows + kStep - 1) / kStep);
    if (steps) t.template run<kDimFirst ? 1 : kPairs>(kDimFirst ? x : dz, kDimFirst ? dz : x, tm * BM, tn * BN, 0, steps, lds);
    if constexpr (kDimFirst) {
        store_across<Tl, BM, BN>(lds, static_cast<uint16_t*>(a.dw) + (a.first + tn * BN) * a.dim + tm * BM, a.dim, a.vocab - tn * BN, a.dim - tm * BM, a.whole,
                                 [&](int i, int j, int r) -> uint32_t { return to_bf16(t.acc[i][j][r]).bits; });
    } else {
        float* out = static_cast<float*>(a.dw) + a.first * a.dim;
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const long long row = tm * BM + Tl::at_m() + 32 * i + Tl::row_of(r);
                if (row >= a.vocab) continue;
#pragma unroll
                for (int j = 0; j < Tl::kN; ++j) {
                    const long long col = tn * BN + Tl::at_n() + 32 * j + (lane & 31);
                    if (col < a.dim) out[row * a.dim + col] = t.acc[i][j][r];
                }
            }
    }
}

// Both in one launch, dH's longer tiles first, so that neither waits for the other's last ones.
template <int B, typename T> __global__ __launch_bounds__(Shape<B>::kThreads, 2) void k_products(const ProductArgs given) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    ProductArgs a = given;
    const Split split = *a.split;
    const long long rows = split.rows, id = blockIdx.x;
    if (!my_piece(split, a.all, a.number, &a.first, &a.vocab, &a.weights)) return;
    a.dz.ld = a.dz.cols = split.piece;
    const long long tiles = (rows + B - 1) / B * ((a.dim + B - 1) / B) * split.splits, first = a.dhidden ? (tiles + 7) / 8 * 8 : 0;
    if (id < first) dhidden_tile<B, sizeof(T) == 4 ? kPlanes : 1>(a, id, rows, split.splits, lds);
    else if (a.dweight) dweight_tile<B, T>(a, id - first, rows, lds);
}

// dH's rows from their sums; zeros for rows that are left out
template <typename T> __global__ __launch_bounds__(256) void k_hidden(const float* sums, const Split* split, const int* place, long long rows, long long dim, T* out) {
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at >= rows * dim) return;
    const long long row = at / dim, from = place[row];
    float t = 0.f;
    if (from >= 0) {
        const float* p = sums + from * dim + (at - row * dim);
        for (int s = 0; s < split->splits; ++s) t += p[s * (split->rows * dim)];
    }
    out[at] = from_f32<T>(t);
}

// ---- host ----
struct Plan {
    bool f32, few, staged;                           // fp32; rows for k_few; weights are packed by pieces
    int planes, k_steps;
    long long rows, dim, vocab, packed_dim;
    int tile;                                        // 128 or 256
    bool flexible;
    long long parts;                                 // of the values
    long long piece;                                 // tokens of a piece of the gradient, and of packed weights
    long long most_sums, most_splits;
    size_t split, live, place, hidden, weights, part, target, info, dz, sums, bytes;      // offsets
};
long long up(long long x, long long to) { return (x + to - 1) / to * to; }

asi_status check(const asi_linear_logprob_desc* d) {
    if (!d || d->rows < 0 || d->dim < 1 || d->vocab < 1 || d->hidden_stride < d->dim || d->weight_stride < d->dim) return ASI_ERR_INVALID_ARG;
    if (!(d->scale > 0.f) || !(d->scale <= 3.4e38f) || (d->any_address & ~1) || d->reserved != 0) return ASI_ERR_INVALID_ARG;
    if (!dtype_ok(d->dtype) || d->scale < 1e-20f || d->scale > 1e20f) return ASI_ERR_UNSUPPORTED;
    if (d->rows >= (1 << 24) || d->dim >= (1 << 18) || d->vocab >= (1 << 28)) return ASI_ERR_UNSUPPORTED;
    if (up(d->rows, 128) / 128 * (up(d->vocab, 128) / 128) > (1 << 23)) return ASI_ERR_UNSUPPORTED;      // tiles of a launch
    if (up(d->dim, 128) / 128 * (up(d->vocab, 128) / 128) > (1 << 23)) return ASI_ERR_UNSUPPORTED;
    if (d->rows * up(d->dim, kStep) / 8 > most_workgroups(256) * 256) return ASI_ERR_UNSUPPORTED;          // threads of k_pack
    return ASI_OK;
}
Plan plan(const asi_linear_logprob_desc* d, bool grad) {
    Plan p{};
    p.f32 = d->dtype == ASI_F32;
    p.planes = p.f32 ? kPlanes : 1;
    p.rows = d->rows; p.dim = d->dim; p.vocab = d->vocab;
    p.packed_dim = up(d->dim, kStep);
    p.k_steps = (int)(p.packed_dim / kStep);
    p.few = !grad && d->rows <= kFew;
    p.staged = !p.few && (p.f32 || d->dim % kStep || d->weight_stride % 8 || d->weight_stride >= (1 << 21) || d->any_address);
    p.tile = up(d->rows, 256) / 256 * (up(d->vocab, 256) / 256) >= 256 ? 256 : 128;
    const long long rows_up = up(d->rows, p.tile);
    p.piece = (long long)(kPieceBytes / 2 / (size_t)rows_up) / 256 * 256;
    if (p.piece < 256) p.piece = 256;
    if (p.piece > up(d->vocab, 256)) p.piece = up(d->vocab, 256);
    // packed weights of a piece are no more than that either, but where 4096 of them are
    const long long most_packed = (long long)(kPieceBytes / (size_t)(p.planes * p.packed_dim * 2)) / 256 * 256;
    if (p.staged && p.piece > most_packed) p.piece = most_packed > 4096 ? most_packed : p.piece < 4096 ? p.piece : 4096;
    p.flexible = !p.staged;
    p.parts = p.few ? (d->vocab + 16 * kFewWaves - 1) / (16 * kFewWaves) : (d->vocab + p.tile - 1) / p.tile;
    // parts that the vocabulary of a piece may be cut in for dH, and the memory for their sums: twice what fills the chip, but no more than
    // half a piece's or twice dH's size in fp32
    const long long tiles = (rows_up / p.tile) * (up(d->dim, p.tile) / p.tile), slots = p.tile == 256 ? 256 : 512;
    const long long memory = (long long)(kPieceBytes / 2 / 4) / (d->rows * d->dim > 0 ? d->rows * d->dim : 1);
    p.most_splits = (2 * slots + tiles - 1) / (tiles > 0 ? tiles : 1);
    if (p.most_splits > (memory > 2 ? memory : 2)) p.most_splits = memory > 2 ? memory : 2;
    if (p.most_splits > 32) p.most_splits = 32;
    if (p.most_splits < 2) p.most_splits = 2;
    p.most_sums = d->rows * p.most_splits;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += round256(bytes); return here; };
    const size_t rows = (size_t)d->rows;
    if (!p.few) {
        p.split = take(sizeof(Split));
        p.live = take(rows * 4);
        p.place = take(rows * 4);
        p.hidden = take((size_t)p.planes * rows * p.packed_dim * 2);
        if (p.staged) p.weights = take((size_t)p.planes * p.piece * p.packed_dim * 2);
    }
    p.part = take((size_t)p.parts * 3 * rows * 4);
    p.target = take(rows * 4);
    if (grad) {
        p.info = take(rows * sizeof(RowInfo));
        p.dz = take((size_t)p.planes * (size_t)rows_up * p.piece * 2);
        p.sums = take((size_t)p.most_sums * d->dim * 4);
    }
    p.bytes = at;
    return p;
}

struct Call {
    const asi_linear_logprob_desc* d;
    Plan p;
    char* ws;
    const void *hidden, *weight;
    const int64_t* targets;
    hipStream_t st;
    asi_status status = ASI_OK;

    template <typename T> T* at(size_t offset) const { return reinterpret_cast<T*>(ws + offset); }
    Operand packed_hidden() const { return Operand{at<uint16_t>(p.hidden), p.packed_dim, p.rows * p.packed_dim, p.rows, p.packed_dim}; }

    void rows_of(float* logprob, float* entropy, float* stats, bool grad, bool dhidden, bool dweight) {
        const SplitArgs how{p.vocab, p.dim, up(p.rows, p.tile) * p.piece, p.piece, p.most_sums, p.most_splits, p.tile, p.f32 ? kPairs : 1, grad, p.flexible, dhidden, dweight};
        const LiveArgs a{targets, p.rows, d->ignore_index, at<Split>(p.split), at<int>(p.live), at<int>(p.place), logprob, entropy, stats, how};
        if (targets) hipLaunchKernelGGL(k_live, 1, 1024, 0, st, a);
        else hipLaunchKernelGGL(k_all_live, dim3((unsigned)((p.rows + 255) / 256)), 256, 0, st, a);
        pack(hidden, d->hidden_stride, p.rows, a.split, a.live, at<uint16_t>(p.hidden), p.rows * p.packed_dim);
    }
    void pack(const void* x, long long stride, long long rows, const Split* split, const int* live, uint16_t* out, long long plane) {
        const size_t es = p.f32 ? 4 : 2;
        const PackArgs a{x, stride, rows, split, live, (int)p.dim, (int)(p.packed_dim / 8), out, p.packed_dim, plane, aligned(x, 16) && stride * es % 16 == 0};
        const dim3 grid((unsigned)((rows * a.pieces + 255) / 256));
        if (p.f32) hipLaunchKernelGGL(k_pack<float>, grid, 256, 0, st, a);
        else hipLaunchKernelGGL(k_pack<bf16_t>, grid, 256, 0, st, a);
    }
    // the weights of tokens first .. first + n - 1 as an operand
    Operand weights(long long first, long long n) {
        const char* from = static_cast<const char*>(weight) + first * d->weight_stride * (p.f32 ? 4 : 2);
        if (!p.staged) return Operand{reinterpret_cast<const uint16_t*>(from), d->weight_stride, 0, n, p.dim};
        uint16_t* out = at<uint16_t>(p.weights);
        pack(from, d->weight_stride, n, nullptr, nullptr, out, p.piece * p.packed_dim);
        return Operand{out, p.packed_dim, p.piece * p.packed_dim, n, p.packed_dim};
    }
    template <int B, typename K, typename A> void tiles(K kernel, LdsAllowed& allowed, long long count, const A& a) {
        if (status != ASI_OK) return;
        if (allow_lds(reinterpret_cast<const void*>(kernel), Shape<B>::kLds, allowed) != hipSuccess) { status = ASI_ERR_HIP; return; }
        hipLaunchKernelGGL(kernel, dim3((unsigned)count), Shape<B>::kThreads, Shape<B>::kLds, st, a);
    }
    LogitArgs logit_args(const Operand& w, long long first, long long n) const {
        LogitArgs a{};
        a.w = w; a.h = packed_hidden(); a.split = at<Split>(p.split); a.k_steps = p.k_steps;
        a.vocab = n; a.first = first; a.scale = d->scale;
        return a;
    }
    template <int B> void logits(const LogitArgs& a) {
        static LdsAllowed one, three;
        const long long count = up(a.vocab, B) / B * (up(p.rows, B) / B);
        if (p.f32) tiles<B>(k_logits<B, kPlanes>, three, count, a);
        else tiles<B>(k_logits<B, 1>, one, count, a);
    }
    template <int B> void products(const LogitArgs& a, const ProductArgs& b) {
        static LdsAllowed grad1, grad3, products2, products4;
        const long long row_tiles = up(p.rows, B) / B, dim_tiles = up(p.dim, B) / B;
        // no more tiles of logits in a piece than its memory holds, however it is cut
        const long long logit_tiles = up(p.piece, B) / B * row_tiles;
        if (p.f32) tiles<B>(k_logits_grad<B, kPlanes>, grad3, logit_tiles, a);
        else tiles<B>(k_logits_grad<B, 1>, grad1, logit_tiles, a);
        const long long hidden_tiles = b.dhidden ? up((up(p.most_sums, B) / B + p.most_splits) * dim_tiles, 8) : 0;
        const long long tokens = !b.all ? b.vocab : b.all < 2 * p.piece ? b.all : 2 * p.piece;
        const long long weight_tiles = b.dweight ? up(tokens, B) / B * dim_tiles : 0;
        if (p.f32) tiles<B>(k_products<B, float>, products4, hidden_tiles + weight_tiles, b);
        else tiles<B>(k_products<B, bf16_t>, products2, hidden_tiles + weight_tiles, b);
    }
    void values(float* logprob, float* entropy, float* stats, RowInfo* info, const float* wa, const float* wb) {
        JoinArgs j{};
        if (p.few) {
            FewArgs a{hidden, weight, d->hidden_stride, d->weight_stride, p.vocab, p.rows, 0, (int)p.dim, false, d->scale, targets, d->ignore_index,
                      at<float>(p.part), at<float>(p.target), p.rows};
            const size_t es = p.f32 ? 4 : 2;
            a.whole = aligned(hidden, 16) && aligned(weight, 16) && d->hidden_stride * es % 16 == 0 && d->weight_stride * es % 16 == 0;
            const dim3 grid((unsigned)p.parts);
            if (p.f32) hipLaunchKernelGGL(k_few<float>, grid, 64 * kFewWaves, 0, st, a);
            else hipLaunchKernelGGL(k_few<bf16_t>, grid, 64 * kFewWaves, 0, st, a);
        } else {
            const long long each = p.staged ? p.piece : p.vocab;
            for (long long first = 0; first < p.vocab; first += each) {
                const long long n = p.vocab - first < each ? p.vocab - first : each;
                LogitArgs a = logit_args(weights(first, n), first, n);
                a.live = at<int>(p.live); a.targets = targets; a.part = at<float>(p.part); a.target_logit = at<float>(p.target);
                a.part_rows = p.rows; a.first_part = first / p.tile;
                if (p.tile == 256) logits<256>(a);
                else logits<128>(a);
            }
            j.split = at<Split>(p.split);
            j.live = at<int>(p.live);
        }
        j.part = at<float>(p.part); j.target_logit = at<float>(p.target); j.part_rows = p.rows; j.parts = p.parts; j.vocab = p.vocab;
        j.ignore = d->ignore_index; j.rows = p.rows; j.targets = targets; j.scale = d->scale;
        j.logprob = logprob; j.entropy = entropy; j.stats = stats; j.info = info; j.a = wa; j.b = wb;
        if (p.rows > 512) hipLaunchKernelGGL(k_join<32>, dim3((unsigned)((p.rows + 31) / 32)), 256, 0, st, j);
        else hipLaunchKernelGGL(k_join<1>, dim3((unsigned)p.rows), 256, 0, st, j);
    }
    void gradients(void* dhidden, void* dweight) {
        int number = 0;
        for (long long first = 0; first < p.vocab && (dhidden || dweight); first += p.piece, ++number) {
            const long long n = p.vocab - first < p.piece ? p.vocab - first : p.piece;
            LogitArgs a = p.flexible ? logit_args(weights(0, p.vocab), 0, p.vocab) : logit_args(weights(first, n), first, n);
            a.all = p.flexible ? p.vocab : 0;
            a.number = number;
            a.info = at<RowInfo>(p.info); a.dz = at<uint16_t>(p.dz); a.dz_plane = p.rows * p.piece;
            ProductArgs b{};
            b.dz = Operand{a.dz, p.piece, a.dz_plane, p.rows, p.piece};
            b.weights = a.w; b.hidden = a.h; b.split = a.split; b.vocab = a.vocab; b.first = a.first; b.all = a.all; b.number = number; b.dim = p.dim;
            b.dhidden = dhidden; b.dweight = dweight;
            b.sums = at<float>(p.sums); b.add = first > 0;
            b.dw = dweight;
            b.whole = p.dim % 8 == 0 && aligned(dweight, 16);
            if (p.tile == 256) products<256>(a, b);
            else products<128>(a, b);
        }
        if (dhidden) {
            const dim3 grid((unsigned)((p.rows * p.dim + 255) / 256));
            if (p.f32) hipLaunchKernelGGL(k_hidden<float>, grid, 256, 0, st, at<float>(p.sums), at<Split>(p.split), at<int>(p.place), p.rows, p.dim, static_cast<float*>(dhidden));
            else hipLaunchKernelGGL(k_hidden<bf16_t>, grid, 256, 0, st, at<float>(p.sums), at<Split>(p.split), at<int>(p.place), p.rows, p.dim, static_cast<bf16_t*>(dhidden));
        }
    }
};

template <typename T> __global__ __launch_bounds__(256) void k_zeros(T* p, long long n) {
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at < n) p[at] = from_f32<T>(0.f);
}

}  // namespace
}  // namespace asi

using namespace asi;

extern "C" {

size_t asi_linear_logprobs_workspace_bytes(const asi_linear_logprob_desc* desc) {
    if (check(desc) != ASI_OK || desc->rows == 0) return 0;
    return plan(desc, false).bytes;
}

asi_status asi_linear_logprobs(const asi_linear_logprob_desc* desc, const void* hidden, const void* weight,
                               const int64_t* targets, float* logprob, float* entropy, float* stats, void* ws,
                               size_t ws_bytes, asi_stream_t stream) {
    if (asi_status why = check(desc); why != ASI_OK) return why;
    const size_t es = dtype_size(desc->dtype);
    if (!aligned(hidden, es) || !aligned(weight, desc->any_address ? es : 16) || !aligned(targets, 8) || !aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(stats, 4)) return ASI_ERR_INVALID_ARG;
    if (desc->rows == 0) return ASI_OK;
    if (!hidden || !weight || (logprob && !targets)) return ASI_ERR_INVALID_ARG;
    if (!ws || !aligned(ws, 256) || ws_bytes < asi_linear_logprobs_workspace_bytes(desc)) return ASI_ERR_WORKSPACE;
    Call c{desc, plan(desc, false), static_cast<char*>(ws), hidden, weight, targets, static_cast<hipStream_t>(stream)};
    if (!c.p.few) c.rows_of(logprob, entropy, stats, false, false, false);
    c.values(logprob, entropy, stats, nullptr, nullptr, nullptr);
    return c.status != ASI_OK ? c.status : launched();
}

size_t asi_linear_logprobs_grad_workspace_bytes(const asi_linear_logprob_desc* desc) {
    if (check(desc) != ASI_OK || desc->rows == 0) return 0;
    return plan(desc, true).bytes;
}

asi_status asi_linear_logprobs_grad(const asi_linear_logprob_desc* desc, int given, const void* hidden, const void* weight,
                                    const int64_t* targets, const float* stats, float* logprob, float* entropy,
                                    const float* grad_logprob, const float* grad_entropy, void* dhidden, void* dweight,
                                    void* ws, size_t ws_bytes, asi_stream_t stream) {
    if (asi_status why = check(desc); why != ASI_OK) return why;
    const size_t es = dtype_size(desc->dtype);
    if (!aligned(hidden, es) || !aligned(weight, desc->any_address ? es : 16) || !aligned(dhidden, es) || !aligned(dweight, es) || !aligned(targets, 8) || !aligned(logprob, 4) ||
        !aligned(entropy, 4) || !aligned(stats, 4) || !aligned(grad_logprob, 4) || !aligned(grad_entropy, 4) || (given & ~1)) return ASI_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (desc->rows == 0) {
        if (!dweight) return ASI_OK;
        const long long n = desc->vocab * desc->dim;
        if (n > most_workgroups(256) * 256) return ASI_ERR_UNSUPPORTED;
        const dim3 grid((unsigned)((n + 255) / 256));
        if (desc->dtype == ASI_F32) hipLaunchKernelGGL(k_zeros<float>, grid, 256, 0, st, static_cast<float*>(dweight), n);
        else hipLaunchKernelGGL(k_zeros<bf16_t>, grid, 256, 0, st, static_cast<bf16_t*>(dweight), n);
        return launched();
    }
    if (!hidden || !weight || ((logprob || grad_logprob) && !targets) || (given && (!stats || (grad_entropy && !entropy)))) return ASI_ERR_INVALID_ARG;
    if (desc->rows * desc->dim > most_workgroups(256) * 256) return ASI_ERR_UNSUPPORTED;
    if (!ws || !aligned(ws, 256) || ws_bytes < asi_linear_logprobs_grad_workspace_bytes(desc)) return ASI_ERR_WORKSPACE;
    Call c{desc, plan(desc, true), static_cast<char*>(ws), hidden, weight, targets, st};
    RowInfo* info = c.at<RowInfo>(c.p.info);
    c.rows_of(given ? nullptr : logprob, given ? nullptr : entropy, nullptr, true, dhidden, dweight);
    if (given) {
        hipLaunchKernelGGL(k_info, dim3((unsigned)((desc->rows + 255) / 256)), 256, 0, st,
                           InfoArgs{c.at<Split>(c.p.split), c.at<int>(c.p.live), targets, stats, entropy, grad_logprob, grad_entropy, desc->scale, desc->vocab, info});
    } else {
        c.values(logprob, entropy, nullptr, info, grad_logprob, grad_entropy);
    }
    c.gradients(dhidden, dweight);
    return c.status != ASI_OK ? c.status : launched();
}

}  // extern "C"
