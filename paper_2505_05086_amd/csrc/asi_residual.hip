// The edge between two blocks (include/asi_lm.h, asi_residual_norm): the norm, gate, dropout and scale of a block's output, its sum
// with the stream and the next block's norm in one pass, and their backward pass in one pass and a sum over rows.
//
// LANES lanes have a row, each up to K pieces of eight entries, kept in registers from their only load to the last use: two chains of
// (sum of squares, rest) in the forward pass; in the backward pass one sum of three (squares of both rows, gradient times stream) and
// then that of the block's norm, which needs the stream's gradient.  What bounds it: memory, read x, y, write s, out (forward: 8188 x 4096,
// stream fp32, 73 us, 5.5 TB/s; 4096 x 2048 bf16 with dropout 18 us), read ds, dout, s, y, write dx, dy (backward: 12003 x 1000 fp32 62 us,
// 4.7 TB/s; 4096 x 2048 bf16 with dropout 33 us, where the generator and a row's chain of sums take as long).
//
// The gradients of gains and gate are sums over rows.  A workgroup of the backward pass goes through many rows and adds up its columns
// in registers; a second launch adds up the workgroups' sums in their order.
#include "asi_dropout_device.h"

namespace asi {
namespace {

constexpr int kSumColumns = 64, kSumShares = 16;

struct Args {
    const void *x, *y, *post, *gate, *pre, *ds, *dout;
    void *stream, *out, *dx, *dy;
    float *part, *unit_part, *dgate;               // sums of a workgroup: [workgroup][2][dim]; of a unit: [unit][dim]
    long long rows, dim, x_stride, y_stride, gate_rows, rows_a_gate, first;      // first: row with which the launch begins
    long long units;                               // of rows that share a gate row and a lane's sums: gate_rows * parts; 0: no such units
    int parts;
    bool post_norm, drop, gain_bf16;
    float scale, eps, inv_dim;
    Keep keep;
};

__device__ __forceinline__ void gain8(const Args& a, const void* p, long long at, int count, float* f) {
    if (!p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = 1.f;
    } else if (a.gain_bf16) {
        load8(static_cast<const bf16_t*>(p) + at, count, f);
    } else {
        load8(static_cast<const float*>(p) + at, count, f);
    }
}

// Sums of N numbers over the LANES lanes of a row (16, a wave or several), in all of them and always in the same order: turns within 16
// lanes, then the 16s of a wave, then the waves through LDS, which has N floats for each wave of the workgroup.
template <int CTRL> __device__ __forceinline__ float turned(float x) { return __uint_as_float(moved<CTRL>(__float_as_uint(x))); }
template <int LANES, int N> __device__ __forceinline__ void row_sums(float* v, float* lds) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += turned<0x128>(v[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += turned<0x124>(v[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += turned<0x122>(v[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += turned<0x121>(v[i]);
    if constexpr (LANES == 16) return;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int x = __float_as_int(v[i]);
        v[i] = (__int_as_float(__builtin_amdgcn_readlane(x, 0)) + __int_as_float(__builtin_amdgcn_readlane(x, 16))) +
               (__int_as_float(__builtin_amdgcn_readlane(x, 32)) + __int_as_float(__builtin_amdgcn_readlane(x, 48)));
    }
    if constexpr (LANES > 64) {
        constexpr int waves = LANES / 64;
        const int wave = threadIdx.x >> 6, first = wave / waves * waves;
        __syncthreads();                           // what was read from lds before
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) lds[wave * N + i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int w = 0; w < waves; ++w) v[i] += lds[(first + w) * N + i];
        }
    }
}

constexpr int threads_of(int lanes) { return lanes > 256 ? lanes : 256; }

template <int K> __device__ __forceinline__ int count_at(const Args& a, int col) { return a.dim - col >= 8 ? 8 : a.dim > col ? (int)(a.dim - col) : 0; }

template <typename S, typename T, int LANES, int K, bool DROP> __global__ __launch_bounds__(threads_of(LANES)) void k_residual(const Args a) {
    __shared__ float lds[threads_of(LANES) / 64];
    constexpr int kRows = threads_of(LANES) / LANES;
    const int lane = threadIdx.x % LANES;
    const long long row = a.first + (long long)blockIdx.x * kRows + threadIdx.x / LANES;
    const bool there = row < a.rows;
    Keep keep = a.keep;
    float x[K][8], y[K][8];
    int count[K];
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = (k * LANES + lane) * 8;
        count[k] = there ? count_at<K>(a, col) : 0;
        if (a.y) load8(static_cast<const T*>(a.y) + row * a.y_stride + col, count[k], y[k]);
        load8(static_cast<const S*>(a.x) + row * a.x_stride + col, count[k], x[k]);
    }
    if (a.y) {
        if constexpr (DROP) read_seed(&keep);
        float r = 1.f;
        if (a.post_norm) {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(y[k][e], y[k][e], sum);
            row_sums<LANES, 1>(&sum, lds);
            r = rsqrtf(sum * a.inv_dim + a.eps);
        }
        const long long gate_row = a.gate ? row / a.rows_a_gate : 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int col = (k * LANES + lane) * 8;
            float post[8], gate[8];
            gain8(a, a.post, col, count[k], post);
            gain8(a, a.gate, gate_row * a.dim + col, count[k], gate);
            uint32_t w[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
            if (DROP) drawn_from(keep, (unsigned long long)(row * a.dim + col), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float n = y[k][e] * r * post[e], d = DROP ? (kept(keep, w, e) ? n * keep.factor : 0.f) : n;
                x[k][e] = to_f32(from_f32<S>(fmaf(d * gate[e], a.scale, x[k][e])));
            }
            store8(static_cast<S*>(a.stream) + row * a.dim + col, count[k], x[k]);
        }
    }
    if (!a.out) return;
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < count[k]) sum = fmaf(x[k][e], x[k][e], sum);
    row_sums<LANES, 1>(&sum, lds);
    const float r = rsqrtf(sum * a.inv_dim + a.eps);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = (k * LANES + lane) * 8;
        float pre[8];
        gain8(a, a.pre, col, count[k], pre);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[k][e] = x[k][e] * r * pre[e];
        store8(static_cast<T*>(a.out) + row * a.dim + col, count[k], x[k]);
    }
}

template <typename S, typename T, int K> struct GradRow {
    Loose<S> ds[K], s[K];
    Loose<T> dout[K], y[K];
};

// Eight gains, as they were loaded
struct Gain8 {
    uint32_t w[8];
    __device__ __forceinline__ void load(const Args& a, const void* p, long long at, int count) {
        if (!p) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = 0x3f800000u;
        } else if (a.gain_bf16) {
            Loose<bf16_t> r;
            r.load(static_cast<const bf16_t*>(p) + at, count);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(r.get(i));
        } else {
            Loose<float> r;
            r.load(static_cast<const float*>(p) + at, count);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = r.w[i];
        }
    }
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(w[e]); }
};

// The rows that the lanes of a row go through: all of them in turns, or those of their units of rows with a gate row in common.
struct Walk {
    long long row, apart, unit, end;               // end: the unit's last row and one; without units, all rows'
    int at, most;
    __device__ __forceinline__ void enter(const Args& a) {
        const long long gate_row = unit / a.parts, part = unit - gate_row * a.parts, first = part * a.rows_a_gate / a.parts;
        row = gate_row * a.rows_a_gate + first;
        end = unit < a.units ? gate_row * a.rows_a_gate + (part + 1) * a.rows_a_gate / a.parts : row;
    }
    __device__ __forceinline__ void start(const Args& a, long long slot, long long slots) {
        apart = slots;
        at = 0;
        most = 1;
        row = unit = slot;
        end = a.rows;
        if (a.units) {
            most = (int)((a.rows_a_gate + a.parts - 1) / a.parts);
            enter(a);
        }
    }
    __device__ __forceinline__ bool there() const { return row < end; }
    __device__ __forceinline__ void next(const Args& a) {
        if (!a.units) { row += apart; return; }
        ++row;
        if (++at == most) { at = 0; unit += apart; enter(a); }
    }
};

// What bounds the backward pass besides memory is the chain load, sum, sum, store of a row: the next row's loads are on their way
// meanwhile (K = 1), and the gains stay in registers (K = 1, all but the gate of a unit).  Between gate and post gain one sum serves both:
// with q = sum over rows of t dropout' u it is post_gain q that is the gate's gradient and gate q the post gain's.
template <typename S, typename T, int LANES, int K, bool DROP> __global__ __launch_bounds__(threads_of(LANES), 2) void k_residual_grad(const Args a) {
    constexpr int kThreads = threads_of(LANES), kRows = kThreads / LANES;
    __shared__ float lds[kThreads * 8];
    const int lane = threadIdx.x % LANES;
    Keep keep = a.keep;
    if constexpr (DROP) read_seed(&keep);
    int col[K], count[K];
    float sum_pre[K][8], sum_q[K][8], sum_post[K][8];
    Gain8 pre, post, gate;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        col[k] = (k * LANES + lane) * 8;
        count[k] = count_at<K>(a, col[k]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum_pre[k][e] = sum_q[k][e] = sum_post[k][e] = 0.f;
    }
    if constexpr (K == 1) {
        pre.load(a, a.pre, col[0], count[0]);
        post.load(a, a.post, col[0], count[0]);
        gate.load(a, a.units ? nullptr : a.gate, col[0], count[0]);
    }
    auto load = [&](const Walk& at, bool go, GradRow<S, T, K>& r) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int n = go && at.there() ? count[k] : 0;
            r.s[k].load(static_cast<const S*>(a.x) + at.row * a.x_stride + col[k], a.dout ? n : 0);
            r.dout[k].load(static_cast<const T*>(a.dout) + at.row * a.dim + col[k], a.dout ? n : 0);
            r.y[k].load(static_cast<const T*>(a.y) + at.row * a.y_stride + col[k], a.y ? n : 0);
            r.ds[k].load(static_cast<const S*>(a.ds) + at.row * a.dim + col[k], a.ds ? n : 0);
        }
    };
    const long long slots = (long long)gridDim.x * kRows;
    Walk walk;
    walk.start(a, (long long)blockIdx.x * kRows + threadIdx.x / LANES, slots);
    const long long turns = ((a.units ? a.units : a.rows) + slots - 1) / slots * walk.most;
    GradRow<S, T, K> r;
    load(walk, true, r);
    for (long long turn = 0; turn < turns; ++turn) {
        const long long row = walk.row, unit = walk.unit;
        const bool there = walk.there(), ends = a.units && walk.at + 1 == walk.most;
        const bool mine = unit < a.units;
        const long long gate_at = mine ? unit / a.parts * a.dim : 0;
        if (K == 1 && a.units && walk.at == 0) gate.load(a, a.gate, gate_at + col[0], mine ? count[0] : 0);
        walk.next(a);
        GradRow<S, T, K> ahead;
        if constexpr (K == 1) load(walk, turn + 1 < turns, ahead);
        float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if constexpr (K > 1) pre.load(a, a.pre, col[k], count[k]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float s = r.s[k].get(e), y = r.y[k].get(e);
                v[0] = fmaf(s, s, v[0]);
                v[1] = fmaf(r.dout[k].get(e) * pre.get(e), s, v[1]);
                v[2] = fmaf(y, y, v[2]);
            }
        }
        row_sums<LANES, 3>(v, lds);
        const float rs = a.dout ? rsqrtf(v[0] * a.inv_dim + a.eps) : 0.f, ry = a.post_norm ? rsqrtf(v[2] * a.inv_dim + a.eps) : 1.f;
        const float along = v[1] * a.inv_dim * rs * rs;
        float w[K][8], dot = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int n = there ? count[k] : 0;
            if constexpr (K > 1) pre.load(a, a.pre, col[k], count[k]);
            float dx[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float s = r.s[k].get(e), go = r.dout[k].get(e);
                // where there is no row, or no norm behind the edge, s and go are 0; rs may be infinite where there is no row
                dx[e] = e < n ? fmaf(rs, fmaf(go, pre.get(e), -s * along), r.ds[k].get(e)) : 0.f;
                if (e < n) sum_pre[k][e] = fmaf(go, s * rs, sum_pre[k][e]);
            }
            if (a.dx) store8(static_cast<S*>(a.dx) + row * a.dim + col[k], n, dx);
            if (!a.y) continue;
            if constexpr (K > 1) {
                post.load(a, a.post, col[k], count[k]);
                gate.load(a, a.gate, gate_at + col[k], count[k]);
            }
            uint32_t bits[4];
            if constexpr (DROP) drawn_from(keep, (unsigned long long)(row * a.dim + col[k]), bits);
            const float size = DROP ? a.scale * keep.factor : a.scale;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[k][e] = 0.f;
                if (e < n && (!DROP || kept(keep, bits, e))) {
                    const float t = dx[e] * size, u = r.y[k].get(e) * ry;
                    sum_q[k][e] = fmaf(t, u, sum_q[k][e]);
                    w[k][e] = t * gate.get(e) * post.get(e);
                    dot = fmaf(w[k][e], u, dot);
                }
            }
        }
        if (a.y) {
            if (a.post_norm) {
                row_sums<LANES, 1>(&dot, lds);
                dot *= a.inv_dim * ry;
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (a.post_norm) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[k][e] = ry * fmaf(-r.y[k].get(e), dot, w[k][e]);
                }
                store8(static_cast<T*>(a.dy) + row * a.dim + col[k], there ? count[k] : 0, w[k]);
            }
            if (ends) {
                // a unit's rows are through: its gate row's gradient, and its share of the post gain's
                float* sum = a.parts > 1 ? a.unit_part : a.dgate;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    if constexpr (K > 1) {
                        post.load(a, a.post, col[k], count[k]);
                        gate.load(a, a.gate, gate_at + col[k], count[k]);
                    }
                    float d[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (mine && e < count[k]) sum_post[k][e] = fmaf(gate.get(e), sum_q[k][e], sum_post[k][e]);
                        d[e] = post.get(e) * sum_q[k][e];
                        sum_q[k][e] = 0.f;
                    }
                    if (sum) store8(sum + unit * a.dim + col[k], mine ? count[k] : 0, d);
                }
            }
        }
        if constexpr (K == 1) r = ahead;
        else load(walk, turn + 1 < turns, r);
    }
    if (!a.part) return;
    // two sums of a workgroup: those of the pre gain, and q or, where gate rows differ, the post gain's
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (which == 0 ? !a.dout : !a.y) continue;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) lds[threadIdx.x * 8 + e] = which == 0 ? sum_pre[k][e] : a.units ? sum_post[k][e] : sum_q[k][e];
            __syncthreads();
            for (int c = threadIdx.x; c < LANES * 8; c += kThreads) {
                float t = 0.f;
#pragma unroll
                for (int slot = 0; slot < kRows; ++slot) t += lds[slot * LANES * 8 + c];
                const long long at = (long long)k * LANES * 8 + c;
                if (at < a.dim) a.part[((long long)blockIdx.x * 2 + which) * a.dim + at] = t;
            }
        }
}

// Columns' sums over the workgroups, in their order: job 0 the pre gain's, job 1 what post gain and gate have in common, job 2 + g gate
// row g's from the `parts` rows of its units.  16 threads share a column, each with eight loads on their way.
struct SumArgs {
    const float *part, *unit_part;
    const void *post_gain, *gate_row;              // job 1: factors of the gate's and the post gain's gradients; nullable
    bool gain_bf16;
    float *pre, *post, *one_gate, *gate;           // one_gate: the gradient of a gate of one row; gate: of the jobs from 2 on
    long long dim, first_gate;
    int pre_blocks, blocks, parts;
};
__global__ __launch_bounds__(kSumColumns * kSumShares) void k_residual_sums(const SumArgs a) {
    __shared__ float lds[kSumShares][kSumColumns];
    const int c = threadIdx.x % kSumColumns, share = threadIdx.x / kSumColumns;
    const long long col = (long long)blockIdx.x * kSumColumns + c, g = a.first_gate + (int)blockIdx.y - 2;
    const int job = (int)blockIdx.y, n = job == 0 ? a.pre_blocks : job == 1 ? a.blocks : a.parts;
    if (job == 0 ? !a.pre : job == 1 ? !a.post && !a.one_gate : !a.gate) return;
    const float* in = (job < 2 ? a.part + job * a.dim : a.unit_part + g * a.parts * a.dim) + col;
    const long long apart = job < 2 ? 2 * a.dim : a.dim;
    float t = 0.f;
    if (col < a.dim) {
        constexpr int kAhead = 8;
        for (int i = share; i < n; i += kSumShares * kAhead) {
            float f[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) f[u] = i + u * kSumShares < n ? in[(i + u * kSumShares) * apart] : 0.f;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) t += f[u];
        }
    }
    lds[share][c] = t;
    __syncthreads();
    if (share || col >= a.dim) return;
    for (int i = 1; i < kSumShares; ++i) t += lds[i][c];
    auto factor = [&](const void* p) { return !p ? 1.f : a.gain_bf16 ? to_f32(static_cast<const bf16_t*>(p)[col]) : static_cast<const float*>(p)[col]; };
    if (job == 0) a.pre[col] = t;
    else if (job == 1) {
        if (a.post) a.post[col] = t * factor(a.gate_row);
        if (a.one_gate) a.one_gate[col] = t * factor(a.post_gain);
    } else a.gate[g * a.dim + col] = t;
}

// ---- host ----
int lanes_for(long long dim) {
    return dim <= 128 ? 16 : dim <= 512 ? 64 : dim <= 1024 ? 128 : dim <= 2048 ? 256 : 512;
}
int rows_a_block(long long dim) { return threads_of(lanes_for(dim)) / lanes_for(dim); }

// Workgroups of the backward pass: as many as are resident, three a CU of 256 threads, one of 512 (32768 x 1024 bf16 with dropout, us: two a CU
// 115, three 101, four 118; 8192 x 4096 with a stream in fp32: one a CU 176, one and a half 226, two 185).
int most_blocks(long long dim) { return threads_of(lanes_for(dim)) == 256 ? 768 : 256; }

asi_status check(const asi_residual_desc* d) {
    if (!d || d->rows < 0 || d->dim < 1 || d->x_stride < d->dim || d->y_stride < d->dim || d->gate_rows < 0 || d->gate_rows > d->rows ||
        (d->gate_rows && d->rows % d->gate_rows) || (d->post_norm & ~1) || !(d->eps >= 0.f && d->eps <= 3e38f) || !(d->scale >= -3e38f && d->scale <= 3e38f)) return ASI_ERR_INVALID_ARG;
    Keep k;
    if (!fill_keep(d->p, d->seed, d->offset, nullptr, &k)) return ASI_ERR_INVALID_ARG;
    if (!dtype_ok(d->stream_dtype) || !dtype_ok(d->dtype) || !dtype_ok(d->gain_dtype) || (d->dtype == ASI_F32 && d->stream_dtype == ASI_BF16)) return ASI_ERR_UNSUPPORTED;
    if (d->dim > ASI_RESIDUAL_MAX_DIM || d->rows > (int64_t(1) << 40)) return ASI_ERR_UNSUPPORTED;
    return ASI_OK;
}
void fill(const asi_residual_desc* d, const int64_t* seed, Args* a) {
    a->rows = d->rows; a->dim = d->dim; a->x_stride = d->x_stride; a->y_stride = d->y_stride; a->gate_rows = d->gate_rows;
    a->rows_a_gate = d->gate_rows ? d->rows / d->gate_rows : 1;
    a->post_norm = d->post_norm; a->gain_bf16 = d->gain_dtype == ASI_BF16;
    a->scale = d->scale; a->eps = d->eps; a->inv_dim = (float)(1.0 / (double)d->dim);
    fill_keep(d->p, d->seed, d->offset, seed, &a->keep);
    a->drop = a->keep.below != 0;
}
// How the backward pass goes through the rows: its workgroups, and the units of rows with a gate row in common (none where one gate row,
// or no gate, serves all of them).
struct Plan {
    int blocks, parts;
    long long units;
    size_t part_floats, unit_floats;
};
Plan plan(const asi_residual_desc* d) {
    Plan p{};
    const int slots = rows_a_block(d->dim);
    p.parts = 1;
    long long items = d->rows;
    if (d->gate_rows > 1) {
        const long long each = d->rows / d->gate_rows, want = (long long)most_blocks(d->dim) * slots / d->gate_rows;
        p.parts = (int)(want < 1 ? 1 : want > each ? each : want);
        items = p.units = d->gate_rows * p.parts;
        if (p.parts > 1) p.unit_floats = (size_t)p.units * d->dim;
    }
    const long long blocks = (items + slots - 1) / slots;
    p.blocks = (int)(blocks < most_blocks(d->dim) ? blocks : most_blocks(d->dim));
    p.part_floats = (size_t)p.blocks * 2 * d->dim;
    return p;
}

template <typename S, typename T, int LANES, int K, bool DROP> void launch(const Args& a, bool back, int blocks, hipStream_t st) {
    if (back) {
        hipLaunchKernelGGL((k_residual_grad<S, T, LANES, K, DROP>), dim3(blocks), threads_of(LANES), 0, st, a);
        return;
    }
    constexpr long long rows = threads_of(LANES) / LANES, most = most_workgroups(threads_of(LANES)) * rows;
    Args b = a;
    for (b.first = 0; b.first < a.rows; b.first += most) {
        const long long left = a.rows - b.first < most ? a.rows - b.first : most;
        hipLaunchKernelGGL((k_residual<S, T, LANES, K, DROP>), dim3((unsigned)((left + rows - 1) / rows)), threads_of(LANES), 0, st, b);
    }
}
template <typename S, typename T, bool DROP> void go(const Args& a, bool back, int blocks, hipStream_t st) {
    switch (lanes_for(a.dim)) {
        case 16: return launch<S, T, 16, 1, DROP>(a, back, blocks, st);
        case 64: return launch<S, T, 64, 1, DROP>(a, back, blocks, st);
        case 128: return launch<S, T, 128, 1, DROP>(a, back, blocks, st);
        case 256: return launch<S, T, 256, 1, DROP>(a, back, blocks, st);
        default:
            if (a.dim <= 4096) return launch<S, T, 512, 1, DROP>(a, back, blocks, st);
            if (a.dim <= 8192) return launch<S, T, 512, 2, DROP>(a, back, blocks, st);
            return launch<S, T, 512, 4, DROP>(a, back, blocks, st);
    }
}
template <typename S, typename T> void go(const Args& a, bool back, int blocks, hipStream_t st) {
    if (a.drop) go<S, T, true>(a, back, blocks, st);
    else go<S, T, false>(a, back, blocks, st);
}
void go(const asi_residual_desc* d, const Args& a, bool back, int blocks, hipStream_t st) {
    if (d->dtype == ASI_F32) go<float, float>(a, back, blocks, st);
    else if (d->stream_dtype == ASI_F32) go<float, bf16_t>(a, back, blocks, st);
    else go<bf16_t, bf16_t>(a, back, blocks, st);
}

}  // namespace
}  // namespace asi

using namespace asi;

extern "C" {

asi_status asi_residual_norm(const asi_residual_desc* desc, const void* x, const void* y, const void* post_gain,
                             const void* gate, const void* pre_gain, const int64_t* seed, void* stream_out, void* out,
                             asi_stream_t stream) {
    if (asi_status why = check(desc); why != ASI_OK) return why;
    const size_t ss = dtype_size(desc->stream_dtype), ts = dtype_size(desc->dtype), gs = dtype_size(desc->gain_dtype);
    if (!aligned(x, ss) || !aligned(stream_out, ss) || !aligned(y, ts) || !aligned(out, ts) || !aligned(post_gain, gs) || !aligned(gate, gs) ||
        !aligned(pre_gain, gs) || !aligned(seed, 8) || (post_gain && !desc->post_norm)) return ASI_ERR_INVALID_ARG;
    if (desc->rows == 0) return ASI_OK;
    if (!x || (!y) != (!stream_out) || (!stream_out && !out) || (desc->gate_rows != 0) != (gate != nullptr) || (!y && gate) ||
        (stream_out == x && desc->x_stride != desc->dim && desc->rows > 1)) return ASI_ERR_INVALID_ARG;
    Args a{};
    fill(desc, seed, &a);
    a.x = x; a.y = y; a.post = post_gain; a.gate = gate; a.pre = pre_gain; a.stream = stream_out; a.out = out;
    go(desc, a, false, 0, static_cast<hipStream_t>(stream));
    return launched();
}

size_t asi_residual_norm_grad_workspace_bytes(const asi_residual_desc* desc) {
    if (check(desc) != ASI_OK || desc->rows == 0) return 0;
    const Plan p = plan(desc);
    return round256(p.part_floats * sizeof(float)) + round256(p.unit_floats * sizeof(float));
}

asi_status asi_residual_norm_grad(const asi_residual_desc* desc, const void* grad_stream, const void* grad_out, const void* s,
                                  const void* y, const void* post_gain, const void* gate, const void* pre_gain,
                                  const int64_t* seed, void* dx, void* dy, float* dpost_gain, float* dgate, float* dpre_gain,
                                  void* ws, size_t ws_bytes, asi_stream_t stream) {
    if (asi_status why = check(desc); why != ASI_OK) return why;
    const size_t ss = dtype_size(desc->stream_dtype), ts = dtype_size(desc->dtype), gs = dtype_size(desc->gain_dtype);
    if (!aligned(grad_stream, ss) || !aligned(s, ss) || !aligned(dx, ss) || !aligned(grad_out, ts) || !aligned(y, ts) || !aligned(dy, ts) ||
        !aligned(post_gain, gs) || !aligned(gate, gs) || !aligned(pre_gain, gs) || !aligned(seed, 8) || !aligned(dpost_gain, 4) || !aligned(dgate, 4) ||
        !aligned(dpre_gain, 4) || (post_gain && !desc->post_norm)) return ASI_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    SumArgs sums{};
    sums.dim = desc->dim;
    Plan p{};
    if (desc->rows) {
        if ((!grad_stream && !grad_out) || (grad_out && !s) || (!y) != (!dy) || (desc->gate_rows != 0) != (gate != nullptr) || (!y && gate) || (dgate && !gate)) return ASI_ERR_INVALID_ARG;
        p = plan(desc);
        const bool gains = dpre_gain || dpost_gain || dgate;
        if (gains && (!ws || !aligned(ws, 256) || ws_bytes < asi_residual_norm_grad_workspace_bytes(desc))) return ASI_ERR_WORKSPACE;
        Args a{};
        fill(desc, seed, &a);
        a.x = s; a.y = y; a.post = post_gain; a.gate = gate; a.pre = pre_gain; a.ds = grad_stream; a.dout = grad_out; a.dx = dx; a.dy = dy;
        a.units = p.units; a.parts = p.parts;
        if (gains) a.part = static_cast<float*>(ws);
        if (dgate) {
            a.dgate = dgate;
            a.unit_part = p.unit_floats ? reinterpret_cast<float*>(static_cast<char*>(ws) + round256(p.part_floats * sizeof(float))) : nullptr;
        }
        go(desc, a, true, p.blocks, st);
        if (!gains) return launched();
        sums.part = a.part; sums.unit_part = a.unit_part;
    }
    // what has no summands (no rows, no block, no norm behind the edge) is zero; one gate row's gradient is made with the post gain's
    const unsigned columns = (unsigned)((desc->dim + kSumColumns - 1) / kSumColumns);
    sums.parts = p.parts;
    sums.pre_blocks = grad_out ? p.blocks : 0;
    sums.blocks = y ? p.blocks : 0;
    sums.pre = dpre_gain; sums.post = dpost_gain; sums.one_gate = desc->gate_rows == 1 ? dgate : nullptr;
    sums.post_gain = post_gain; sums.gate_row = p.units ? nullptr : gate; sums.gain_bf16 = desc->gain_dtype == ASI_BF16;
    if (dpre_gain || dpost_gain || sums.one_gate) hipLaunchKernelGGL(k_residual_sums, dim3(columns, 2), kSumColumns * kSumShares, 0, st, sums);
    if (dgate && p.units && p.parts > 1) {
        constexpr long long most = 65000;
        sums.pre = sums.post = nullptr;
        sums.gate = dgate;
        for (sums.first_gate = 0; sums.first_gate < desc->gate_rows; sums.first_gate += most) {
            const long long n = desc->gate_rows - sums.first_gate < most ? desc->gate_rows - sums.first_gate : most;
            hipLaunchKernelGGL(k_residual_sums, dim3(columns, (unsigned)(n + 2)), kSumColumns * kSumShares, 0, st, sums);
        }
    }
    return launched();
}

}  // extern "C"
