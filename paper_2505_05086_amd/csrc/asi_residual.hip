// The edge between two blocks (include/asi_lm.h, asi_residual_norm): the norm, gate, dropout and scale of a block's output, its sum
// with the stream and the next block's norm in one pass, and their backward pass in one pass and a sum over rows.
//
// LANES lanes have a row, each up to K pieces of eight entries, kept in registers from their only load to the last use: two chains of
// (sum of squares, rest) in the forward pass; in the backward pass one sum of three (squares of both rows, gradient times stream) and
// then that of the block's norm, which needs the stream's gradient.  What bounds it: memory, read x, y, write s, out (forward), read
// ds, dout, s, y, write dx, dy (backward).
//
// The gradients of gains and gate are sums over rows.  A workgroup of the backward pass goes through many rows and adds up its columns
// in registers; a second launch adds up the workgroups' sums in their order.
#include "asi_dropout_device.h"

namespace asi {
namespace {

constexpr int kMostBlocks = 512;                   // workgroups of the backward pass
constexpr int kSumColumns = 64, kSumShares = 16;

struct Args {
    const void *x, *y, *post, *gate, *pre, *ds, *dout;
    void *stream, *out, *dx, *dy;
    float *part, *unit_part, *dgate;               // sums of a workgroup: [workgroup][pre, post, gate][dim]; of a unit: [unit][dim]
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

// Sums of N numbers over the LANES lanes of a row, in all of them.  `lds` has N floats for each wave of the workgroup.
template <int LANES, int N> __device__ __forceinline__ void row_sums(float* v, float* lds) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lanes_sum<(LANES < 64 ? LANES : 64)>(v[i]);
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

template <int LANES> constexpr int threads_of() { return LANES > 256 ? LANES : 256; }

template <int K> __device__ __forceinline__ int count_at(const Args& a, int col) { return a.dim - col >= 8 ? 8 : a.dim > col ? (int)(a.dim - col) : 0; }

template <typename S, typename T, int LANES, int K> __global__ __launch_bounds__(threads_of<LANES>()) void k_residual(const Args a) {
    __shared__ float lds[threads_of<LANES>() / 64];
    constexpr int kRows = threads_of<LANES>() / LANES;
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
        if (a.drop) read_seed(&keep);
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
            if (a.drop) drawn_from(keep, (unsigned long long)(row * a.dim + col), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float n = y[k][e] * r * post[e], d = a.drop ? (kept(keep, w, e) ? n * keep.factor : 0.f) : n;
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

// The sums of a lane's columns over the rows that it has been through.
template <int K> struct Sums {
    float pre[K][8], post[K][8], gate[K][8];
};

// One row of the backward pass.
template <typename S, typename T, int LANES, int K> __device__ __forceinline__ void grad_row(const Args& a, const Keep& keep, long long row, bool there, Sums<K>& sums, float* lds) {
    const int lane = threadIdx.x % LANES;
    float s[K][8], go[K][8], ds[K][8], y[K][8];
    int count[K];
    float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = (k * LANES + lane) * 8;
        count[k] = there ? count_at<K>(a, col) : 0;
        load8(static_cast<const S*>(a.ds) + row * a.dim + col, a.ds ? count[k] : 0, ds[k]);
        load8(static_cast<const T*>(a.dout) + row * a.dim + col, a.dout ? count[k] : 0, go[k]);
        load8(static_cast<const S*>(a.x) + row * a.x_stride + col, a.dout ? count[k] : 0, s[k]);
        load8(static_cast<const T*>(a.y) + row * a.y_stride + col, a.y ? count[k] : 0, y[k]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float pre[8];
        gain8(a, a.pre, (k * LANES + lane) * 8, count[k], pre);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[0] = fmaf(s[k][e], s[k][e], v[0]);
            v[1] = fmaf(go[k][e] * pre[e], s[k][e], v[1]);
            v[2] = fmaf(y[k][e], y[k][e], v[2]);
        }
    }
    row_sums<LANES, 3>(v, lds);
    const float rs = a.dout ? rsqrtf(v[0] * a.inv_dim + a.eps) : 0.f, ry = a.post_norm ? rsqrtf(v[2] * a.inv_dim + a.eps) : 1.f;
    const float along = v[1] * a.inv_dim * rs * rs;
    const long long gate_row = a.gate ? row / a.rows_a_gate : 0;
    float dot = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = (k * LANES + lane) * 8;
        if (a.dout) {
            float pre[8];
            gain8(a, a.pre, col, count[k], pre);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ds[k][e] = fmaf(rs, fmaf(go[k][e], pre[e], -s[k][e] * along), ds[k][e]);
                sums.pre[k][e] = fmaf(go[k][e], s[k][e] * rs, sums.pre[k][e]);
            }
        }
        if (a.dx) store8(static_cast<S*>(a.dx) + row * a.dim + col, count[k], ds[k]);
        if (a.y) {
            float post[8], gate[8];
            gain8(a, a.post, col, count[k], post);
            gain8(a, a.gate, gate_row * a.dim + col, count[k], gate);
            uint32_t w[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
            if (a.drop) drawn_from(keep, (unsigned long long)(row * a.dim + col), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool keeps = !a.drop || kept(keep, w, e);
                const float t = ds[k][e] * a.scale * (a.drop ? keep.factor : 1.f), u = y[k][e] * ry;
                if (e < count[k] && keeps) sums.gate[k][e] = fmaf(t, u * post[e], sums.gate[k][e]);
                const float d = keeps ? t * gate[e] : 0.f;
                if (e < count[k]) sums.post[k][e] = fmaf(d, u, sums.post[k][e]);
                ds[k][e] = d * post[e];
                y[k][e] = u;
                if (e < count[k]) dot = fmaf(ds[k][e], u, dot);
            }
        }
    }
    if (!a.y) return;
    if (a.post_norm) {
        row_sums<LANES, 1>(&dot, lds);
        dot *= a.inv_dim;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int col = (k * LANES + lane) * 8;
        if (a.post_norm) {
#pragma unroll
            for (int e = 0; e < 8; ++e) ds[k][e] = ry * fmaf(-y[k][e], dot, ds[k][e]);
        }
        store8(static_cast<T*>(a.dy) + row * a.dim + col, count[k], ds[k]);
    }
}

template <typename S, typename T, int LANES, int K> __global__ __launch_bounds__(threads_of<LANES>()) void k_residual_grad(const Args a) {
    constexpr int kThreads = threads_of<LANES>(), kRows = kThreads / LANES;
    __shared__ float lds[kThreads * 8];
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    Keep keep = a.keep;
    if (a.drop) read_seed(&keep);
    Sums<K> sums;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) sums.pre[k][e] = sums.post[k][e] = sums.gate[k][e] = 0.f;
    if (!a.units) {
        for (long long at = (long long)blockIdx.x * kRows; at < a.rows; at += (long long)gridDim.x * kRows)
            grad_row<S, T, LANES, K>(a, keep, at + slot, at + slot < a.rows, sums, lds);
    } else {
        // rows [part * rows_a_gate / parts, (part + 1) * rows_a_gate / parts) of a gate row, by the lanes of one row; the workgroup's
        // others go on with it, so that all of it comes to its barriers
        const long long most = (a.rows_a_gate + a.parts - 1) / a.parts;
        for (long long at = (long long)blockIdx.x * kRows; at < a.units; at += (long long)gridDim.x * kRows) {
            const long long unit = at + slot, gate_row = unit / a.parts, part = unit - gate_row * a.parts;
            const long long from = part * a.rows_a_gate / a.parts, to = (part + 1) * a.rows_a_gate / a.parts;
            const bool mine = unit < a.units;
            for (long long i = 0; i < most; ++i) grad_row<S, T, LANES, K>(a, keep, gate_row * a.rows_a_gate + from + i, mine && from + i < to, sums, lds);
            float* sum = a.parts > 1 ? a.unit_part : a.dgate;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int col = (k * LANES + lane) * 8;
                if (sum) store8(sum + unit * a.dim + col, mine ? count_at<K>(a, col) : 0, sums.gate[k]);
#pragma unroll
                for (int e = 0; e < 8; ++e) sums.gate[k][e] = 0.f;
            }
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int k = 0; k < K; ++k)
        for (int which = 0; which < 3; ++which) {
            if ((which == 0 && !a.dout) || (which > 0 && !a.y) || (which == 2 && a.units)) continue;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) lds[threadIdx.x * 8 + e] = which == 0 ? sums.pre[k][e] : which == 1 ? sums.post[k][e] : sums.gate[k][e];
            __syncthreads();
            for (int c = threadIdx.x; c < LANES * 8; c += kThreads) {
                float t = 0.f;
#pragma unroll
                for (int r = 0; r < kRows; ++r) t += lds[r * LANES * 8 + c];
                const long long col = (long long)k * LANES * 8 + c;
                if (col < a.dim) a.part[((long long)blockIdx.x * 3 + which) * a.dim + col] = t;
            }
        }
}

// Columns' sums over the workgroups, in their order: `count` rows for gains, and for gate row g the `parts` rows of its units.
struct SumArgs {
    const float *part, *unit_part;
    float *pre, *post, *gate;
    long long dim, first_gate;
    int blocks, parts;
    bool units;
};
__global__ __launch_bounds__(kSumColumns * kSumShares) void k_residual_sums(const SumArgs a) {
    __shared__ float lds[kSumShares][kSumColumns];
    const int c = threadIdx.x % kSumColumns, share = threadIdx.x / kSumColumns;
    const long long col = (long long)blockIdx.x * kSumColumns + c;
    const int job = (int)blockIdx.y;
    const float* in;
    float* out;
    long long apart;
    int n;
    if (job < 2 || !a.units) {
        in = a.part + job * a.dim; apart = 3 * a.dim; n = a.blocks;
        out = job == 0 ? a.pre : job == 1 ? a.post : a.gate;
    } else {
        const long long g = a.first_gate + job - 2;
        in = a.unit_part + g * a.parts * a.dim; apart = a.dim; n = a.parts;
        out = a.gate + g * a.dim;
    }
    if (!out) return;
    float t = 0.f;
    if (col < a.dim)
        for (int i = share; i < n; i += kSumShares) t += in[i * apart + col];
    lds[share][c] = t;
    __syncthreads();
    if (share == 0 && col < a.dim) {
        for (int i = 1; i < kSumShares; ++i) t += lds[i][c];
        out[col] = t;
    }
}

// ---- host ----
int lanes_for(long long dim) {
    int lanes = 8;
    while (lanes < 512 && lanes * 8 < dim) lanes *= 2;
    return lanes;
}
int rows_a_block(long long dim) {
    const int lanes = lanes_for(dim);
    return lanes >= 256 ? 1 : 256 / lanes;
}

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
        const long long each = d->rows / d->gate_rows, want = (long long)kMostBlocks * slots / d->gate_rows;
        p.parts = (int)(want < 1 ? 1 : want > each ? each : want);
        items = p.units = d->gate_rows * p.parts;
        if (p.parts > 1) p.unit_floats = (size_t)p.units * d->dim;
    }
    const long long blocks = (items + slots - 1) / slots;
    p.blocks = (int)(blocks < kMostBlocks ? blocks : kMostBlocks);
    p.part_floats = (size_t)p.blocks * 3 * d->dim;
    return p;
}

template <typename S, typename T, int LANES, int K> void launch(const Args& a, bool back, int blocks, hipStream_t st) {
    if (back) {
        hipLaunchKernelGGL((k_residual_grad<S, T, LANES, K>), dim3(blocks), threads_of<LANES>(), 0, st, a);
        return;
    }
    constexpr long long rows = threads_of<LANES>() / LANES, most = most_workgroups(threads_of<LANES>()) * rows;
    Args b = a;
    for (b.first = 0; b.first < a.rows; b.first += most) {
        const long long left = a.rows - b.first < most ? a.rows - b.first : most;
        hipLaunchKernelGGL((k_residual<S, T, LANES, K>), dim3((unsigned)((left + rows - 1) / rows)), threads_of<LANES>(), 0, st, b);
    }
}
template <typename S, typename T> void go(const Args& a, bool back, int blocks, hipStream_t st) {
    switch (lanes_for(a.dim)) {
        case 8: return launch<S, T, 8, 1>(a, back, blocks, st);
        case 16: return launch<S, T, 16, 1>(a, back, blocks, st);
        case 32: return launch<S, T, 32, 1>(a, back, blocks, st);
        case 64: return launch<S, T, 64, 1>(a, back, blocks, st);
        case 128: return launch<S, T, 128, 1>(a, back, blocks, st);
        case 256: return launch<S, T, 256, 1>(a, back, blocks, st);
        default:
            if (a.dim <= 4096) return launch<S, T, 512, 1>(a, back, blocks, st);
            if (a.dim <= 8192) return launch<S, T, 512, 2>(a, back, blocks, st);
            return launch<S, T, 512, 4>(a, back, blocks, st);
    }
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
    sums.pre = dpre_gain; sums.post = dpost_gain; sums.gate = dgate;
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
    // what has no summands (no rows, no block, no norm behind the edge) is zero
    const dim3 grid_x((unsigned)((desc->dim + kSumColumns - 1) / kSumColumns));
    sums.parts = p.parts;
    auto go_sums = [&](float* pre, float* post, float* gate, int blocks, bool units, unsigned jobs, long long first) {
        SumArgs b = sums;
        b.pre = pre; b.post = post; b.gate = gate; b.blocks = blocks; b.units = units; b.first_gate = first;
        hipLaunchKernelGGL(k_residual_sums, dim3(grid_x.x, jobs), kSumColumns * kSumShares, 0, st, b);
    };
    const int pre_blocks = grad_out ? p.blocks : 0, post_blocks = y ? p.blocks : 0;
    const bool by_unit = p.units != 0;
    float* gate_sum = desc->gate_rows == 1 ? dgate : nullptr;
    if (pre_blocks == post_blocks) {
        go_sums(dpre_gain, dpost_gain, gate_sum, pre_blocks, false, 3, 0);
    } else {
        if (dpre_gain) go_sums(dpre_gain, nullptr, nullptr, pre_blocks, false, 3, 0);
        if (dpost_gain || gate_sum) go_sums(nullptr, dpost_gain, gate_sum, post_blocks, false, 3, 0);
    }
    if (dgate && by_unit && p.parts > 1) {
        constexpr long long most = 65000;
        for (long long g = 0; g < desc->gate_rows; g += most) {
            const long long n = desc->gate_rows - g < most ? desc->gate_rows - g : most;
            go_sums(nullptr, nullptr, dgate, 0, true, (unsigned)(n + 2), g);
        }
    }
    return launched();
}

}  // extern "C"
