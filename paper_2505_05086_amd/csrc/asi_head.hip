// Token log probabilities from hidden states and the output layer's weights, and their gradients, without the logits
// (include/asi_lm.h, asi_linear_logprobs).
//
//   k_live        the rows that have a target, in order, and how many: every kernel behind it reads that number, the host does not
//   k_pack        their hidden states next to each other, k filled up with zeros to whole steps; fp32 as three planes of bf16.  The
//                 same for a piece of the weights where they cannot be read as they lie (fp32, rows that are no whole vectors)
//   k_logits      a tile of logits, vocabulary along the registers of a lane and tokens along the lanes, so that a token's maximum
//                 and sums over 128 (64) of the vocabulary stay in a lane but for one exchange.  Values: x_max, how many logits are
//                 as large, sum e over the others and sum e d of each token, d = x - x_max, e = exp(scale d), and the target's logit
//   k_logits_grad the same tiles as dz, in two parts of bf16 for bf16 inputs and three for fp32
//   k_few         the values for few rows, left out or not, the weights from memory straight into the matrix instructions; k_few_grad and
//                 k_few_grad_tiles their gradients from the logits that it leaves, 16 rows a column
//   k_join        joins the tiles' values
//   k_products    the products of dz with weights (dH) and hidden states (dW), read across as they lie (asi_tiles.h)
//   k_hidden      the sums of dH, in fp32 over the pieces of the vocabulary and the parts of a piece, to their rows
//
// What bounds it: the matrix products, 2 rows dim vocab for the values and with the gradients 12 for bf16, whose dz has two parts, or six times 8 for
// fp32 (2 less where the logits are kept): 2731 rows x 2048 x 32000 bf16 344 us of values (1.04 PFLOP/s), 2.06 ms with gradients (1.04); 8190 x
// 2048 x 100003 2.76 ms (1.22), 18.5 ms (1.09).  The weights' memory for few rows: 8 x 2048 x 32000 28.1 us, 4.7 TB/s.  From 17 rows on k_few is
// bound by the caches instead: each wave reads all hidden states for its 16 tokens, 1 GB for 64 x 2048 x 32000 fp32, 177 us.
#include <math.h>

#include "asi_head_plan.h"
#include "asi_lds.h"
#include "asi_tiles.h"

namespace asi {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLow = -1e30f;                       // stands for -infinity where that is multiplied by 0
typedef float v4f __attribute__((ext_vector_type(4)));
constexpr int kLeftOut = -2;                         // a RowInfo's target: the row is left out

// Tiles of 256 x 256 by 8 waves where they fill the chip (8190 x 2048 logits of 100003: 2.76 ms, with tiles of 128 3.26), of 128 x 128 by
// 4 waves, two workgroups a CU, where they would not.
template <int B> struct Shape {
    static constexpr int WN = B == 256 ? 4 : 2, kThreads = 128 * WN;
    template <bool A, bool X> using Of = Tile<B, B, A, X, WN>;
    static constexpr size_t kLds = 4 * B * kStep * 2 > B * (2 * B + 16) ? 4 * B * kStep * 2 : B * (2 * B + 16);      // two buffers, or a tile in bf16
};

// ---- rows ---------------------------------------------------------------------------------------------------
struct SplitArgs {
    long long vocab, dim, elements, piece, most_sums, most_splits;      // elements of dz and rows of sums that there is memory for
    int tile, pairs;
    bool grad, flexible, dhidden, dweight;           // flexible: pieces may be larger than `piece` where rows are fewer
};
// The number of parts that ends a launch of dH's tiles, then dW's, soonest, `slots` workgroups at a time: lengths in steps of 64 k, to which
// writing a tile adds about 6.  A lane of the wave for each number of parts.  (2731 x 2048 x 32000: 2076 us so, 2310 with one.)
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
// A number's planes.  What bf16 leaves out is exact in fp32.  A number above bf16's largest has that for its first plane, and the rest, so that it
// stays finite.  An infinity is (1, 0, infinity) with its sign: of the six products of planes infinity then meets the other side's first plane
// alone, which has that side's sign and is 0 only with it, and every other one is finite.  (As (infinity, 0, 0) it would meet the other
// side's lower planes too, which may be 0 or have the other sign.)
template <typename T> __device__ __forceinline__ void planes_of(float x, uint16_t* h) {
    h[0] = to_bf16(x).bits;
    if constexpr (sizeof(T) == 4) {
        const uint16_t sign = (uint16_t)(__float_as_uint(x) >> 16) & 0x8000u;
        if (fabsf(x) == INFINITY) {
            h[0] = sign | 0x3f80u; h[1] = 0; h[2] = sign | 0x7f80u;
            return;
        }
        if ((h[0] & 0x7fffu) == 0x7f80u) h[0] = sign | 0x7f7fu;
        const float r = x - to_f32(bf16_t{h[0]}), q = r - to_f32(to_bf16(r));
        const bool number = x == x;
        h[1] = number ? to_bf16(r).bits : 0;
        h[2] = number ? to_bf16(q).bits : 0;
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
    // values: [tile][top, ones, rest, along][rows], the targets' logits [rows]
    const int *live;
    const int64_t* targets;
    float *part, *target_logit;
    long long part_rows, first_part;
    float* kept;                                     // the tiles' logits as lanes hold them, from the values to the gradient
    // gradient
    const RowInfo* info;
    uint16_t* dz;                                    // [row][dz_stride], planes apart
    long long dz_stride, dz_plane;
};

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

// Of a set of logits: the largest, how many are as large, the sum of exp(scale d) over the others (d = x - top), and sum exp(scale d) d.
// The ones are counted apart: where one token is nearly sure, the others' sum is all that its log probability is made of, and added to
// 1 it would lose its last bits.
struct Joined {
    float top, ones, rest, along;
    __device__ __forceinline__ float all() const { return ones + rest; }
};
__device__ __forceinline__ Joined join(Joined a, Joined b, float c) {
    const float top = fmaxf(a.top, b.top), base = top == -INFINITY ? 0.f : top;
    const float da = fmaxf(a.top - base, kLow), db = fmaxf(b.top - base, kLow);
    const float ea = __builtin_amdgcn_exp2f(da * c), eb = __builtin_amdgcn_exp2f(db * c), sa = a.all(), sb = b.all();
    const bool as = a.top == top, bs = b.top == top;
    // sums that are NaN stay NaN: they are multiplied, not compared
    return Joined{top, (as ? a.ones : 0.f) + (bs ? b.ones : 0.f), (as ? a.rest : sa * ea) + (bs ? b.rest : sb * eb),
                  ea * fmaf(sa, da, a.along) + eb * fmaf(sb, db, b.along)};
}
// The sums over logits of a lane, base being the largest (0 if that is -infinity).  exp2 of 0 is 1 exactly, and its fraction 0.
struct Summed {
    float all = 0.f, rest = 0.f, along = 0.f;
    __device__ __forceinline__ void add(float x, float base, float c) {
        const float d = max_nan(x - base, kLow), e = __builtin_amdgcn_exp2f(d * c);
        all += e;
        rest += __builtin_amdgcn_fractf(e);
        along = fmaf(e, d, along);
    }
    __device__ __forceinline__ void across(int lanes) {
        all += __shfl_xor(all, lanes);
        rest += __shfl_xor(rest, lanes);
        along += __shfl_xor(along, lanes);
    }
    __device__ __forceinline__ Joined joined(float top) const { return Joined{top, rintf(all - rest), rest, along}; }
};
__device__ __forceinline__ void store_joined(float* to, long long apart, const Joined& x) {
    to[0] = x.top;
    to[apart] = x.ones;
    to[2 * apart] = x.rest;
    to[3 * apart] = x.along;
}

// A lane's logits of its workgroup's tile, four at a time, the lanes' next to each other.  Values and gradient have the same tiles in the same
// order, so each lane finds its own again.
template <typename Tl, typename F> __device__ __forceinline__ void each_kept(float* kept, F f) {
    v4f* at = reinterpret_cast<v4f*>(kept) + (long long)blockIdx.x * (Tl::kM * Tl::kN * 4 * Tl::kThreads) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
        for (int j = 0; j < Tl::kN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) f(at[((i * Tl::kN + j) * 4 + q) * Tl::kThreads], i, j, 4 * q);
}

template <int B, int PLANES, bool KEEP> __global__ __launch_bounds__(Shape<B>::kThreads, 2) void k_logits(const LogitArgs a) {
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
    t.template run<PLANES == 1 ? kOne : kSix>(a.w, h, tm * BM, tn * BN, 0, a.k_steps, lds);
    if constexpr (KEEP)
        each_kept<Tl>(a.kept, [&](v4f& at, int i, int j, int r) { at = v4f{t.acc[i][j][r], t.acc[i][j][r + 1], t.acc[i][j][r + 2], t.acc[i][j][r + 3]}; });
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
        Summed sum;
#pragma unroll
        for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum.add(t.acc[i][j][r], base, c);
        sum.across(32);
        if (lane < 32) shared[Tl::wave_m() * BN + col] = sum.joined(top);
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
            store_joined(a.part + (a.first_part + tm) * 4 * a.part_rows + row, a.part_rows, x);
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

// dz of a logit that is not the target's, and of the target's
__device__ __forceinline__ float of_logit(float z, const RowInfo& f, float c) {
    const float x = fmaf(z - f.top, c, -f.log2sum), p = __builtin_amdgcn_exp2f(x);
    return -p * (f.b != 0.f ? fmaf(f.b, fmaf(max_nan(x, kLow), 1.f / kLog2e, f.entropy), f.a) : f.a);
}
__device__ __forceinline__ float of_target(float z, const RowInfo& f, float c) {
    const float logp = max_nan(fmaf(z - f.top, c, -f.log2sum), kLow) * (1.f / kLog2e);
    const float d = -f.a * expm1f(logp);
    return f.b != 0.f ? fmaf(-expf(logp) * f.b, logp + f.entropy, d) : d;
}

// PLANES: of the inputs, 0 where the logits were kept; DZ: of dz
template <int B, int PLANES, int DZ> __global__ __launch_bounds__(Shape<B>::kThreads, 2) void k_logits_grad(const LogitArgs given) {
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
    if constexpr (PLANES == 0) {
        each_kept<Tl>(a.kept, [&](const v4f& at, int i, int j, int r) {
#pragma unroll
            for (int e = 0; e < 4; ++e) t.acc[i][j][r + e] = at[e];
        });
    } else {
        t.clear();
        Operand h = a.h;
        h.rows = rows;
        t.template run<PLANES == 1 ? kOne : kSix>(a.w, h, tm * BM, tn * BN, 0, a.k_steps, lds);
    }
    const float c = a.scale * kLog2e;
    const int lane = threadIdx.x & 63;
    const long long v0 = tm * BM + Tl::at_m();
#pragma unroll
    for (int j = 0; j < Tl::kN; ++j) {
        const long long row = tn * BN + Tl::at_n() + 32 * j + (lane & 31);
        RowInfo f{0.f, INFINITY, 0.f, 0.f, 0.f, -1, {0, 0}};
        if (row < rows) f = a.info[row];
        const long long target = f.target >= 0 ? f.target - a.first - v0 : -1;
        const bool here = __any(target >= 0 && target < BM / 2);
        float hit = 0.f;                             // the target's logit
        if (here) {
#pragma unroll
            for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) hit = target == 32 * i + Tl::row_of(r) ? t.acc[i][j][r] : hit;
        }
        if (__any(f.b != 0.f)) {                     // NaN too
#pragma unroll
            for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) t.acc[i][j][r] = of_logit(t.acc[i][j][r], f, c);
        } else {
#pragma unroll
            for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) t.acc[i][j][r] = -f.a * __builtin_amdgcn_exp2f(fmaf(t.acc[i][j][r] - f.top, c, -f.log2sum));
        }
        if (here) {
            const float of = of_target(hit, f, c);
#pragma unroll
            for (int i = 0; i < Tl::kM; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (target == 32 * i + Tl::row_of(r)) t.acc[i][j][r] = of;
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
    // a turn for each part, and no more than that in registers
#pragma unroll 1
    for (int p = 0; p < DZ; ++p)
        store_across<Tl, BM, BN>(lds, a.dz + p * a.dz_plane + tn * BN * a.dz_stride + tm * BM, a.dz_stride, rows - tn * BN, BM, true,
                                 [&](int i, int j, int r) -> uint32_t {
                                     // an infinity, of a row's factor that is one, is 1 and infinity in the last part, as in planes_of
                                     const uint32_t bits = to_bf16(t.acc[i][j][r]).bits;
                                     const bool number = (bits & 0x7fffu) != 0x7f80u;
                                     if (number) t.acc[i][j][r] -= __uint_as_float(bits << 16);
                                     return number || p + 1 == DZ ? bits : p == 0 ? (bits & 0x8000u) | 0x3f80u : 0u;
                                 });
}

// ---- few rows -----------------------------------------------------------------------------------------------
// Logits of up to 64 rows: a wave takes 16 of the vocabulary and all k, both operands from memory straight into the registers of the
// matrix instruction, a token along four lanes.  What bounds it: the weights' memory.
struct FewArgs {
    const void *h, *w;
    long long h_stride, w_stride, vocab, rows;
    int dim;
    float scale;
    const int64_t* targets;
    float *part, *target_logit;                      // nullable, both
    float* logits;                                   // [16 rows][token][16], for the gradients; nullable
};
constexpr int kFewAhead = 8;
template <typename T> struct FewStep;               // the k of a wave's load of 16 bytes a lane
template <> struct FewStep<bf16_t> { static constexpr int k = 32; };
template <> struct FewStep<float> { static constexpr int k = 16; };
// Products of load number u, added to one of several sums: short chains are faster, and their roundings fewer: one chain over 3875 entries in
// fp32 left 1.3e-5 of a log probability near 0, eight 8e-6.
__device__ __forceinline__ void few_product(const Vec16<bf16_t>& w, const Vec16<bf16_t>& h, int u, v4f* sums, int count) {
    sums[u % count] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, w.raw), __builtin_bit_cast(v8bf, h.raw), sums[u % count], 0, 0, 0);
}
__device__ __forceinline__ void few_product(const Vec16<float>& w, const Vec16<float>& h, int u, v4f* sums, int count) {
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[(4 * u + i) % count] = __builtin_amdgcn_mfma_f32_16x16x4f32(w.get(i), h.get(i), sums[(4 * u + i) % count], 0, 0, 0);
}
template <typename T> __device__ __forceinline__ Vec16<T> few_load(const T* p, int count) {
    Loose<T, Vec16<T>::N> v;
    v.load(p, count);
    return Vec16<T>{make_uint4(v.w[0], v.w[1], v.w[2], v.w[3])};
}
// NB: 16s of rows
template <typename T, int NB> __global__ __launch_bounds__(64 * kFewWaves) void k_few(const FewArgs a) {
    __shared__ Joined shared[kFewWaves][16 * NB];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15;
    const long long v0 = ((long long)blockIdx.x * kFewWaves + wave) * 16;
    // behind the end of either the first row is read, and what comes of it left alone
    const T* w = static_cast<const T*>(a.w) + (v0 + col < a.vocab ? v0 + col : 0) * a.w_stride;
    const T* h[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) h[b] = static_cast<const T*>(a.h) + (16 * b + col < a.rows ? 16 * b + col : 0) * a.h_stride;
    constexpr int step = FewStep<T>::k, ahead = NB > 2 ? kFewAhead / 2 : kFewAhead, all = Vec16<T>::N;
    constexpr int sums = NB == 1 ? 8 : 4;
    v4f part[NB][sums], acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < sums; ++i) part[b][i] = v4f{0.f, 0.f, 0.f, 0.f};
    const int k = (lane >> 4) * all;
    int at = 0;
    for (; at + step * ahead <= a.dim; at += step * ahead) {
        Vec16<T> wv[ahead], hv[NB][ahead];
#pragma unroll
        for (int u = 0; u < ahead; ++u) wv[u] = few_load(w + at + u * step + k, all);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int u = 0; u < ahead; ++u) hv[b][u] = few_load(h[b] + at + u * step + k, all);
#pragma unroll
        for (int u = 0; u < ahead; ++u)
#pragma unroll
            for (int b = 0; b < NB; ++b) few_product(wv[u], hv[b][u], u, part[b], sums);
    }
    for (; at < a.dim; at += step) {
        const int count = at + k < a.dim ? a.dim - at - k : 0;
        const Vec16<T> wv = few_load(w + at + k, count);
#pragma unroll
        for (int b = 0; b < NB; ++b) few_product(wv, few_load(h[b] + at + k, count), 0, part[b], sums);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int n = sums / 2; n; n >>= 1)
#pragma unroll
            for (int i = 0; i < n; ++i) part[b][i] += part[b][i + n];
        acc[b] = part[b][0];
    }
    // a lane has tokens v0 + 4 (lane / 16) + r of rows 16 b + col; logits have room for the groups of 16 that have a row, and no others
    const float c = a.scale * kLog2e;
    const long long first = v0 + 4 * (lane >> 4);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (first + r >= a.vocab) acc[b][r] = -INFINITY;
            else if (a.logits && 16 * b < a.rows) a.logits[((long long)b * a.vocab + first + r) * 16 + col] = acc[b][r];
            top = fmaxf(top, acc[b][r]);
        }
        if (!a.part) continue;
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = top == -INFINITY ? 0.f : top;
        Summed sum;
#pragma unroll
        for (int r = 0; r < 4; ++r) sum.add(acc[b][r], base, c);
        sum.across(16);
        sum.across(32);
        if (lane < 16) shared[wave][16 * b + lane] = sum.joined(top);
        const long long row = 16 * b + col;
        if (a.targets && row < a.rows) {
            const long long target = a.targets[row] - first;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (target == r && first + r < a.vocab) a.target_logit[row] = acc[b][r];
        }
    }
    if (!a.part) return;
    __syncthreads();
    if (threadIdx.x < 16 * NB && (int)threadIdx.x < a.rows) {
        Joined x = shared[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < kFewWaves; ++i) x = join(x, shared[i][threadIdx.x], c);
        store_joined(a.part + (long long)blockIdx.x * 4 * a.rows + threadIdx.x, a.rows, x);
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
__device__ __forceinline__ void write_info(RowInfo* to, float top, float logsum, float entropy, float a, float b, float scale, int64_t target, long long vocab, bool given, bool left_out) {
    RowInfo f{top, logsum * kLog2e, a * scale, b * scale, entropy, (int)target, {0, 0}};
    if (top == -INFINITY) f = RowInfo{0.f, INFINITY, 0.f, 0.f, 0.f, -1, {0, 0}};      // nothing but -infinity: no gradient
    if (left_out) f = RowInfo{0.f, INFINITY, 0.f, 0.f, 0.f, kLeftOut, {0, 0}};
    else if (given && (target < 0 || target >= vocab)) { f.target = -1; f.log2sum = NAN; }
    if (!given) f.target = -1;
    if (left_out) f.target = kLeftOut;
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
        for (long long i = share; i < a.parts; i += kShares) top = fmaxf(top, p[i * 4 * a.part_rows]);
    const float base = top == -INFINITY ? 0.f : top;
    Joined sum{top, 0.f, 0.f, 0.f};
    if (at < rows)
#pragma unroll 4
        for (long long i = share; i < a.parts; i += kShares) {
            const float* q = p + i * 4 * a.part_rows;
            const float own = q[0], ones = q[a.part_rows], rest = q[2 * a.part_rows];
            const float d = fmaxf(own - base, kLow), e = __builtin_amdgcn_exp2f(d * c);
            sum.ones += own == top ? ones : 0.f;
            sum.rest += own == top ? rest : (ones + rest) * e;
            sum.along = fmaf(fmaf(ones + rest, d, q[3 * a.part_rows]), e, sum.along);
        }
    shared[share][in] = sum;
    __syncthreads();
    for (int n = kShares / 2; n; n >>= 1) {
        if (share < n) shared[share][in] = join(shared[share][in], shared[share + n][in], c);
        __syncthreads();
    }
    if (share || at >= rows) return;
    const Joined x = shared[0][in];
    const long long row = a.live ? a.live[at] : at;
    const float all = x.all();
    const bool nan = all != all, empty = x.top == -INFINITY && !nan;
    const float logsum = empty ? 0.f : nan ? NAN : logf(x.ones) + log1pf(x.rest / x.ones);
    const float entropy = empty ? 0.f : nan ? NAN : fmaxf(logsum - a.scale * (x.along / all), 0.f);
    const int64_t target = a.targets ? a.targets[row] : 0;
    const bool left_out = a.targets && target == a.ignore;      // where the rows have not been sorted out
    if (a.logprob) {
        float v = NAN;
        if (target >= 0 && target < a.vocab) {
            const float z = a.target_logit[at], d = z - x.top;
            // finite logits farther apart than fp32 reaches: both scaled first
            v = empty || z == -INFINITY ? -INFINITY : d == -INFINITY ? fmaf(z, a.scale, -x.top * a.scale) - logsum : fmaf(a.scale, d, -logsum);
        }
        if (nan) v = NAN;
        a.logprob[row] = left_out ? 0.f : v;
    }
    if (a.entropy) a.entropy[row] = left_out ? 0.f : entropy;
    if (a.stats) {
        a.stats[2 * row] = left_out ? 0.f : x.top;
        a.stats[2 * row + 1] = left_out ? 0.f : logsum;
    }
    if (a.info) write_info(a.info + at, x.top, logsum, entropy, a.a ? a.a[row] : 0.f, a.b ? a.b[row] : 0.f, a.scale, target, a.vocab, a.targets != nullptr, left_out);
}

struct InfoArgs {
    const Split* split;                              // nullable, with live: all `rows` rows as they are
    const int* live;
    long long rows, ignore;
    const int64_t* targets;
    const float *stats, *entropy, *a, *b;
    float scale;
    long long vocab;
    RowInfo* info;
};
__global__ __launch_bounds__(256) void k_info(const InfoArgs a) {
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at >= (a.split ? a.split->rows : a.rows)) return;
    const long long row = a.live ? a.live[at] : at;
    write_info(a.info + at, a.stats[2 * row], a.stats[2 * row + 1], a.b ? a.entropy[row] : 0.f, a.a ? a.a[row] : 0.f, a.b ? a.b[row] : 0.f, a.scale,
               a.targets ? a.targets[row] : 0, a.vocab, a.targets != nullptr, a.targets && a.targets[row] == a.ignore);
}

// ---- few rows' gradients ------------------------------------------------------------------------------------
// dz of 64 tokens is made in LDS from their logits; then every token's row of the weights is read once, for dH, and its row of dW written
// once, by lanes of COLS neighbouring columns that hold ROWS rows' hidden states and sums of dH in registers.  Where a row needs fewer
// lanes than the workgroup has, tokens go round groups of lanes.  What bounds it: memory.
struct FewGradArgs {
    const void *h, *w;
    long long h_stride, w_stride, vocab, dim;
    int rows, lanes, blocks;                         // lanes of a row (a power of two, up to 256); blocks of the vocabulary
    float scale;
    const float* logits;                             // [16 rows][token][16]
    const RowInfo* info;
    float* sums;                                     // [block][row][dim], nullable
    void* dw;                                        // nullable
};
template <typename T, int ROWS, int COLS> __global__ __launch_bounds__(256) void k_few_grad(const FewGradArgs a) {
    static_assert(ROWS <= 16, "logits of one group of 16 rows");
    __shared__ __attribute__((aligned(16))) float dz[kFewTokens][ROWS];
    __shared__ float share[256 * COLS];
    __shared__ RowInfo info[ROWS];
    if (threadIdx.x < ROWS) info[threadIdx.x] = (int)threadIdx.x < a.rows ? a.info[threadIdx.x] : RowInfo{0.f, INFINITY, 0.f, 0.f, 0.f, kLeftOut, {0, 0}};
    const int lane = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes, groups = 256 / a.lanes;
    const long long col = ((long long)blockIdx.x * a.lanes + lane) * COLS;
    const int count = a.dim - col >= COLS ? COLS : a.dim > col ? (int)(a.dim - col) : 0;
    __syncthreads();
    float h[ROWS][COLS], sum[ROWS][COLS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        // a row that is left out is not read
        load_some<COLS>(static_cast<const T*>(a.h) + r * a.h_stride + col, info[r].target != kLeftOut ? count : 0, h[r]);
#pragma unroll
        for (int e = 0; e < COLS; ++e) sum[r][e] = 0.f;
    }
    const float c = a.scale * kLog2e;
    const long long steps = (a.vocab + kFewTokens - 1) / kFewTokens, from = steps * blockIdx.y / a.blocks, to = steps * (blockIdx.y + 1) / a.blocks;
    for (long long step = from; step < to; ++step) {
        const long long v0 = step * kFewTokens;
        const int tokens = a.vocab - v0 < kFewTokens ? (int)(a.vocab - v0) : kFewTokens;
        for (int i = threadIdx.x; i < kFewTokens * ROWS; i += 256) {
            const int v = i / ROWS, r = i % ROWS;
            const RowInfo f = info[r];
            float d = 0.f;
            if (v < tokens && f.target != kLeftOut) {
                const float z = a.logits[(v0 + v) * 16 + r];
                d = f.target == v0 + v ? of_target(z, f, c) : of_logit(z, f, c);
            }
            dz[v][r] = d;
        }
        __syncthreads();
        constexpr int ahead = 4;
        for (int v = group; v < tokens; v += groups * ahead) {
            Loose<T, COLS> w[ahead];
            if (a.sums) {
#pragma unroll
                for (int u = 0; u < ahead; ++u)
                    w[u].load(static_cast<const T*>(a.w) + (v0 + v + u * groups) * a.w_stride + col, v + u * groups < tokens ? count : 0);
            }
#pragma unroll
            for (int u = 0; u < ahead; ++u) {
                const int at = v + u * groups;
                if (at >= tokens) break;
                float out[COLS];
#pragma unroll
                for (int e = 0; e < COLS; ++e) out[e] = 0.f;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const float d = dz[at][r];
#pragma unroll
                    for (int e = 0; e < COLS; ++e) {
                        out[e] = fmaf(d, h[r][e], out[e]);
                        if (a.sums) sum[r][e] = fmaf(d, w[u].get(e), sum[r][e]);
                    }
                }
                if (a.dw) store_some<COLS>(static_cast<T*>(a.dw) + (v0 + at) * a.dim + col, count, out);
            }
        }
        __syncthreads();
    }
    if (!a.sums) return;
    // the groups' sums in their order; 0 of a row that is left out, whatever the weights that its dz of 0 has met
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (info[r].target == kLeftOut) {
#pragma unroll
            for (int e = 0; e < COLS; ++e) sum[r][e] = 0.f;
        }
        if (groups > 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < COLS; ++e) share[threadIdx.x * COLS + e] = sum[r][e];
            __syncthreads();
            if (group == 0) {
                for (int g = 1; g < groups; ++g)
#pragma unroll
                    for (int e = 0; e < COLS; ++e) sum[r][e] += share[(g * a.lanes + lane) * COLS + e];
            }
        }
        if (group == 0 && r < a.rows) store_some<COLS>(a.sums + ((long long)blockIdx.y * a.rows + r) * a.dim + col, count, sum[r]);
    }
}
// The same for 5 to 64 rows by matrix instructions (16 x 16 x 4, fp32 throughout), where 2 rows vocab dim multiply-adds a side on
// the vector units would take longer than the memory.  A wave has 64 columns, lane l the four from 4 (l % 16) on, so that 16 lanes read a
// row of W, or write one of dW, side by side: column 4 n + e is column n of block e of a matrix instruction.  TB: 16s of rows.
template <typename T, int TB> __global__ __launch_bounds__(256) void k_few_grad_tiles(const FewGradArgs a) {
    __shared__ float dz[2][16 * TB][17];             // two turns of 16 tokens
    __shared__ RowInfo info[16 * TB];
    if (threadIdx.x < 16 * TB) info[threadIdx.x] = (int)threadIdx.x < a.rows ? a.info[threadIdx.x] : RowInfo{0.f, INFINITY, 0.f, 0.f, 0.f, kLeftOut, {0, 0}};
    const int lane = threadIdx.x & 63, n = lane & 15, k = lane >> 4;
    const long long col = ((long long)blockIdx.x * 4 + (threadIdx.x >> 6)) * 64 + 4 * n;
    const int count = a.dim - col >= 4 ? 4 : a.dim > col ? (int)(a.dim - col) : 0;
    __syncthreads();
    const T *hidden = static_cast<const T*>(a.h), *weights = static_cast<const T*>(a.w);
    float h[4 * TB][4];                              // rows 4 j + k
    v4f sum[TB][4];
#pragma unroll
    for (int j = 0; j < 4 * TB; ++j) load_some<4>(hidden + (4 * j + k) * a.h_stride + col, info[4 * j + k].target != kLeftOut ? count : 0, h[j]);
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[t][e] = v4f{0.f, 0.f, 0.f, 0.f};
    const float c = a.scale * kLog2e;
    const long long turns = (a.vocab + 15) / 16, from = turns * blockIdx.y / a.blocks, to = turns * (blockIdx.y + 1) / a.blocks;
    auto load = [&](long long turn, Loose<T, 4>* w) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long v = turn * 16 + 4 * i + k;
            w[i].load(weights + v * a.w_stride + col, a.sums && turn < to && v < a.vocab ? count : 0);
        }
    };
    auto gradients = [&](long long turn) {           // of 16 tokens' logits, a thread for a token and every 16th row
        const int v = threadIdx.x & 15;
#pragma unroll
        for (int i = 0; i < TB; ++i) {
            const int r = 16 * i + (threadIdx.x >> 4);
            const RowInfo f = info[r];
            float d = 0.f;
            if (turn < to && turn * 16 + v < a.vocab && f.target != kLeftOut) {
                const float z = a.logits[((long long)i * a.vocab + turn * 16 + v) * 16 + r % 16];
                d = f.target == turn * 16 + v ? of_target(z, f, c) : of_logit(z, f, c);
            }
            dz[turn & 1][r][v] = d;
        }
    };
    Loose<T, 4> w[4];
    load(from, w);
    gradients(from);
    __syncthreads();
    for (long long turn = from; turn < to; ++turn) {
        Loose<T, 4> ahead[4];
        load(turn + 1, ahead);
        gradients(turn + 1);
        const float(*d)[17] = dz[turn & 1];
        if (a.sums) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < TB; ++t) {
                    const float x = d[16 * t + n][4 * i + k];
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[t][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, w[i].get(e), sum[t][e], 0, 0, 0);
                }
        }
        if (a.dw) {
            v4f out[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4 * TB; ++j) {
                const float x = d[4 * j + k][n];
#pragma unroll
                for (int e = 0; e < 4; ++e) out[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, h[j][e], out[e], 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float f[4] = {out[0][r], out[1][r], out[2][r], out[3][r]};
                const long long v = turn * 16 + 4 * k + r;
                T* to = static_cast<T*>(a.dw) + v * a.dim + col;
                store_some<4>(to, v < a.vocab ? count : 0, f);
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = ahead[i];
    }
    if (!a.sums) return;
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * t + 4 * k + r;
            const bool out = info[row].target == kLeftOut;      // 0, whatever the weights that its dz of 0 has met
            const float f[4] = {out ? 0.f : sum[t][0][r], out ? 0.f : sum[t][1][r], out ? 0.f : sum[t][2][r], out ? 0.f : sum[t][3][r]};
            store_some<4>(a.sums + ((long long)blockIdx.y * a.rows + row) * a.dim + col, row < a.rows ? count : 0, f);
        }
}
// dH's rows from the blocks' sums, in their order: 8 threads share a column
template <typename T> __global__ __launch_bounds__(256) void k_few_hidden(const float* sums, int blocks, long long rows, long long dim, T* out) {
    __shared__ float lds[8][32];
    const int in = threadIdx.x % 32, share = threadIdx.x / 32;
    const long long at = (long long)blockIdx.x * 32 + in, n = rows * dim;
    float t = 0.f;
    if (at < n) {
        constexpr int ahead = 8;
        for (int b = share; b < blocks; b += 8 * ahead) {
            float f[ahead];
#pragma unroll
            for (int u = 0; u < ahead; ++u) f[u] = b + 8 * u < blocks ? sums[(b + 8 * u) * n + at] : 0.f;
#pragma unroll
            for (int u = 0; u < ahead; ++u) t += f[u];
        }
    }
    lds[share][in] = t;
    __syncthreads();
    if (share || at >= n) return;
    for (int i = 1; i < 8; ++i) t += lds[i][in];
    out[at] = from_f32<T>(t);
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
template <int B, int DZ> __device__ __forceinline__ void dhidden_tile(const ProductArgs& a, long long id, long long rows, int splits, char* lds) {
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
    if (to > from) t.template run<DZ == 2 ? kTwoA : kSix>(dz, a.weights, tm * BM, tn * BN, from, to - from, lds);
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
template <int B, typename T, int DZ> __device__ __forceinline__ void dweight_tile(const ProductArgs& a, long long id, long long rows, char* lds) {
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
    if (steps) t.template run<DZ == 2 ? kTwoB : kSix>(kDimFirst ? x : dz, kDimFirst ? dz : x, tm * BM, tn * BN, 0, steps, lds);
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
template <int B, typename T, int DZ> __global__ __launch_bounds__(Shape<B>::kThreads, 2) void k_products(const ProductArgs given) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    ProductArgs a = given;
    const Split split = *a.split;
    const long long rows = split.rows, id = blockIdx.x;
    if (!my_piece(split, a.all, a.number, &a.first, &a.vocab, &a.weights)) return;
    a.dz.ld = a.dz.cols = split.piece;
    const long long tiles = (rows + B - 1) / B * ((a.dim + B - 1) / B) * split.splits, first = a.dhidden ? (tiles + 7) / 8 * 8 : 0;
    if (id < first) dhidden_tile<B, DZ>(a, id, rows, split.splits, lds);
    else if (a.dweight) dweight_tile<B, T, DZ>(a, id - first, rows, lds);
}

// dH's rows from their sums, four entries a thread; zeros for rows that are left out
template <typename T> __global__ __launch_bounds__(256) void k_hidden(const float* sums, const Split* split, const int* place, long long rows, int dim, T* out) {
    const int pieces = (dim + 3) / 4;
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, row = at / pieces;
    if (row >= rows) return;
    const int col = (int)(at - row * pieces) * 4, count = dim - col, splits = split->splits;
    const long long from = place[row], plane = (long long)split->rows * dim;
    float t[4] = {0.f, 0.f, 0.f, 0.f};
    if (from >= 0) {
        const float* p = sums + from * dim + col;
        for (int s = 0; s < splits; ++s) {
            float f[4];
            load_some<4>(p + s * plane, count, f);
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] += f[e];
        }
    }
    store_some<4>(out + row * dim + col, count, t);
}

// ---- host ----
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
        const SplitArgs how{p.vocab, p.dim, up(p.rows, p.tile) * p.piece, p.piece, p.most_sums, p.most_splits, p.tile, p.f32 ? kPairs : p.dz_planes, grad, p.flexible, dhidden, dweight};
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
    // the weights of tokens first .. first + n - 1 as an operand; `packed`: the call before has packed the same
    Operand weights(long long first, long long n, bool packed = false) {
        const char* from = static_cast<const char*>(weight) + first * d->weight_stride * (p.f32 ? 4 : 2);
        if (!p.staged) return Operand{reinterpret_cast<const uint16_t*>(from), d->weight_stride, 0, n, p.dim};
        uint16_t* out = at<uint16_t>(p.weights);
        if (!packed) pack(from, d->weight_stride, n, nullptr, nullptr, out, p.piece * p.packed_dim);
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
    template <typename T> void few_logits(bool values, bool keep) {
        const FewArgs a{hidden, weight, d->hidden_stride, d->weight_stride, p.vocab, p.rows, (int)p.dim, d->scale,
                        targets, values ? at<float>(p.part) : nullptr, at<float>(p.target), keep ? at<float>(p.logits) : nullptr};
        const dim3 grid((unsigned)p.parts);
        if (p.rows <= 16) hipLaunchKernelGGL((k_few<T, 1>), grid, 64 * kFewWaves, 0, st, a);
        else if (p.rows <= 32) hipLaunchKernelGGL((k_few<T, 2>), grid, 64 * kFewWaves, 0, st, a);
        else hipLaunchKernelGGL((k_few<T, 4>), grid, 64 * kFewWaves, 0, st, a);
    }
    void few_logits(bool values, bool keep) {
        if (p.f32) few_logits<float>(values, keep);
        else few_logits<bf16_t>(values, keep);
    }
    FewGradArgs few_args(void* dhidden, void* dweight, int lanes) const {
        return FewGradArgs{hidden, weight, d->hidden_stride, d->weight_stride, p.vocab, p.dim, (int)p.rows, lanes, p.few_blocks, d->scale,
                           at<float>(p.logits), at<RowInfo>(p.info), dhidden ? at<float>(p.sums) : nullptr, dweight};
    }
    template <typename T> void few_grad_tiles(void* dhidden, void* dweight) {
        const FewGradArgs a = few_args(dhidden, dweight, 64);
        const dim3 grid((unsigned)((p.dim + 255) / 256), (unsigned)p.few_blocks);
        if (p.rows <= 16) hipLaunchKernelGGL((k_few_grad_tiles<T, 1>), grid, 256, 0, st, a);
        else if (p.rows <= 32) hipLaunchKernelGGL((k_few_grad_tiles<T, 2>), grid, 256, 0, st, a);
        else hipLaunchKernelGGL((k_few_grad_tiles<T, 4>), grid, 256, 0, st, a);
    }
    template <typename T, int ROWS, int COLS> void few_grad(void* dhidden, void* dweight) {
        int lanes = 8;
        while (lanes < 256 && lanes * COLS < p.dim) lanes *= 2;
        const FewGradArgs a = few_args(dhidden, dweight, lanes);
        hipLaunchKernelGGL((k_few_grad<T, ROWS, COLS>), dim3((unsigned)((p.dim + lanes * COLS - 1) / (lanes * COLS)), (unsigned)p.few_blocks), 256, 0, st, a);
    }
    template <typename T> void few_gradients(void* dhidden, void* dweight) {
        if (!dhidden && !dweight) return;
        if (p.rows <= kFewGradVector) few_grad<T, 4, 8>(dhidden, dweight);
        else few_grad_tiles<T>(dhidden, dweight);
        if (dhidden) hipLaunchKernelGGL(k_few_hidden<T>, dim3((unsigned)((p.rows * p.dim + 31) / 32)), 256, 0, st, at<float>(p.sums), p.few_blocks, p.rows, p.dim, static_cast<T*>(dhidden));
    }
    template <int B> void logits(const LogitArgs& a) {
        static LdsAllowed one, three, kept1, kept3;
        const long long count = up(a.vocab, B) / B * (up(p.rows, B) / B);
        if (a.kept && p.f32) tiles<B>(k_logits<B, kPlanes, true>, kept3, count, a);
        else if (a.kept) tiles<B>(k_logits<B, 1, true>, kept1, count, a);
        else if (p.f32) tiles<B>(k_logits<B, kPlanes, false>, three, count, a);
        else tiles<B>(k_logits<B, 1, false>, one, count, a);
    }
    template <int B> void products(const LogitArgs& a, const ProductArgs& b) {
        static LdsAllowed grad2, grad3, kept2, kept3, products2, products3;
        const long long row_tiles = up(p.rows, B) / B, dim_tiles = up(p.dim, B) / B;
        // no more tiles of logits in a piece than its memory holds, however it is cut
        const long long logit_tiles = up(p.piece, B) / B * row_tiles;
        if (a.kept && p.f32) tiles<B>(k_logits_grad<B, 0, kPlanes>, kept3, logit_tiles, a);
        else if (a.kept) tiles<B>(k_logits_grad<B, 0, kFineParts>, kept2, logit_tiles, a);
        else if (p.f32) tiles<B>(k_logits_grad<B, kPlanes, kPlanes>, grad3, logit_tiles, a);
        else tiles<B>(k_logits_grad<B, 1, kFineParts>, grad2, logit_tiles, a);
        const long long hidden_tiles = b.dhidden ? up((up(p.most_sums, B) / B + p.most_splits) * dim_tiles, 8) : 0;
        const long long tokens = !b.all ? b.vocab : b.all < 2 * p.piece ? b.all : 2 * p.piece;
        const long long weight_tiles = b.dweight ? up(tokens, B) / B * dim_tiles : 0;
        if (p.f32) tiles<B>(k_products<B, float, kPlanes>, products3, hidden_tiles + weight_tiles, b);
        else tiles<B>(k_products<B, bf16_t, kFineParts>, products2, hidden_tiles + weight_tiles, b);
    }
    void values(float* logprob, float* entropy, float* stats, RowInfo* info, const float* wa, const float* wb) {
        JoinArgs j{};
        if (p.few) {
            few_logits(true, info != nullptr);
        } else {
            each_piece(p, [&](long long first, long long n, int tile, long long first_part) {
                LogitArgs a = logit_args(weights(first, n), first, n);
                a.live = at<int>(p.live); a.targets = targets; a.part = at<float>(p.part); a.target_logit = at<float>(p.target);
                a.part_rows = p.rows; a.first_part = first_part;
                if (p.keep && info) a.kept = at<float>(p.kept);
                if (tile == 256) logits<256>(a);
                else logits<128>(a);
            });
            j.split = at<Split>(p.split);
            j.live = at<int>(p.live);
        }
        j.part = at<float>(p.part); j.target_logit = at<float>(p.target); j.part_rows = p.rows; j.parts = p.parts; j.vocab = p.vocab;
        j.ignore = d->ignore_index; j.rows = p.rows; j.targets = targets; j.scale = d->scale;
        j.logprob = logprob; j.entropy = entropy; j.stats = stats; j.info = info; j.a = wa; j.b = wb;
        // rows of a workgroup: more share their loads' lines, fewer leave more workgroups (8190 rows of 391 parts, us: 32 62, 16 38, 8 44; 2731
        // rows of 125: 32 25, 8 12)
        if (p.rows > 4096) hipLaunchKernelGGL(k_join<16>, dim3((unsigned)((p.rows + 15) / 16)), 256, 0, st, j);
        else if (p.rows > 512) hipLaunchKernelGGL(k_join<8>, dim3((unsigned)((p.rows + 7) / 8)), 256, 0, st, j);
        else hipLaunchKernelGGL(k_join<1>, dim3((unsigned)p.rows), 256, 0, st, j);
    }
    // `after_values`: values() of the same call has run
    void gradients(void* dhidden, void* dweight, bool after_values) {
        int number = 0;
        for (long long first = 0; first < p.vocab && (dhidden || dweight); first += p.piece, ++number) {
            const long long n = p.vocab - first < p.piece ? p.vocab - first : p.piece;
            LogitArgs a = p.flexible ? logit_args(weights(0, p.vocab), 0, p.vocab) : logit_args(weights(first, n, after_values && p.piece >= p.vocab), first, n);
            a.all = p.flexible ? p.vocab : 0;
            a.number = number;
            if (p.keep && after_values) a.kept = at<float>(p.kept);
            a.info = at<RowInfo>(p.info); a.dz = at<uint16_t>(p.dz); a.dz_plane = up(p.rows, p.tile) * p.piece;
            ProductArgs b{};
            b.dz = Operand{a.dz, p.piece, a.dz_plane, p.rows, p.piece};
            b.weights = a.w; b.hidden = a.h; b.split = a.split; b.vocab = a.vocab; b.first = a.first; b.all = a.all; b.number = number; b.dim = p.dim;
            b.dhidden = dhidden; b.dweight = dweight;
            b.sums = at<float>(p.sums); b.add = first > 0;
            b.dw = dweight;
            b.whole = p.dim % 8 == 0 && aligned(dweight, 16);
            if (piece_tile(p, n) == 256) products<256>(a, b);
            else products<128>(a, b);
        }
        if (dhidden) {
            const dim3 grid((unsigned)((p.rows * ((p.dim + 3) / 4) + 255) / 256));
            if (p.f32) hipLaunchKernelGGL(k_hidden<float>, grid, 256, 0, st, at<float>(p.sums), at<Split>(p.split), at<int>(p.place), p.rows, (int)p.dim, static_cast<float*>(dhidden));
            else hipLaunchKernelGGL(k_hidden<bf16_t>, grid, 256, 0, st, at<float>(p.sums), at<Split>(p.split), at<int>(p.place), p.rows, (int)p.dim, static_cast<bf16_t*>(dhidden));
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
        const long long n = desc->vocab * desc->dim, most = most_workgroups(256) * 256;
        for (long long first = 0; first < n; first += most) {
            const long long count = n - first < most ? n - first : most;
            const dim3 grid((unsigned)((count + 255) / 256));
            if (desc->dtype == ASI_F32) hipLaunchKernelGGL(k_zeros<float>, grid, 256, 0, st, static_cast<float*>(dweight) + first, count);
            else hipLaunchKernelGGL(k_zeros<bf16_t>, grid, 256, 0, st, static_cast<bf16_t*>(dweight) + first, count);
        }
        return launched();
    }
    if (!hidden || !weight || ((logprob || grad_logprob) && !targets) || (given && (!stats || (grad_entropy && !entropy)))) return ASI_ERR_INVALID_ARG;
    if (desc->rows * desc->dim > most_workgroups(256) * 256) return ASI_ERR_UNSUPPORTED;
    if (!ws || !aligned(ws, 256) || ws_bytes < asi_linear_logprobs_grad_workspace_bytes(desc)) return ASI_ERR_WORKSPACE;
    Call c{desc, plan(desc, true), static_cast<char*>(ws), hidden, weight, targets, st};
    RowInfo* info = c.at<RowInfo>(c.p.info);
    // Logits that are summed in another order than those that the statistics are of are off from them by their roundings, and where p is nearly
    // 1 that is more than 1 - p.  33 to 64 rows of bf16 may take k_few for their values and tiles here: these make their own statistics, of
    // logits that the gradient would need all the same.
    if (given && plan(desc, false).few != c.p.few) given = 0, logprob = entropy = nullptr;
    if (!c.p.few) c.rows_of(given ? nullptr : logprob, given ? nullptr : entropy, nullptr, true, dhidden, dweight);
    if (given) {
        if (c.p.few) c.few_logits(false, true);
        hipLaunchKernelGGL(k_info, dim3((unsigned)((desc->rows + 255) / 256)), 256, 0, st,
                           InfoArgs{c.p.few ? nullptr : c.at<Split>(c.p.split), c.p.few ? nullptr : c.at<int>(c.p.live), desc->rows, desc->ignore_index, targets, stats, entropy, grad_logprob, grad_entropy, desc->scale, desc->vocab, info});
    } else {
        c.values(logprob, entropy, nullptr, info, grad_logprob, grad_entropy);
    }
    if (!c.p.few) c.gradients(dhidden, dweight, !given);
    else if (c.p.f32) c.few_gradients<float>(dhidden, dweight);
    else c.few_gradients<bf16_t>(dhidden, dweight);
    return c.status != ASI_OK ? c.status : launched();
}

}  // extern "C"
