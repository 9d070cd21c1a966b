// Dropout without a stored mask (include/asi_lm.h, asi_dropout).
//
// A lane takes eight neighbouring elements, one call of the generator.  What bounds it: memory, read + write (12003 x 1001 fp32, rows 1008
// apart, 20.7 us, 4.6 TB/s; 4096 x 2048 bf16 8.2 us, from and to the caches).
#include "asi_dropout_device.h"

namespace asi {
namespace {

constexpr int kThreads = 256;

struct Args {
    const void* x;
    void* y;
    long long rows, dim, x_stride, y_stride, total, first;      // first: group of eight with which the launch begins
    Keep keep;
};

// A lane has one group; with two or four each 12003 x 1001 fp32 takes 25.3 or 26.5 us and not 20.7, 4096 x 2048 bf16 9.2 or 9.6 and not 8.6.
template <typename T, bool FLAT> __global__ __launch_bounds__(kThreads) void k_dropout(const Args a) {
    Keep k = a.keep;
    const long long begin = a.first + (long long)blockIdx.x * kThreads, group = begin + threadIdx.x, at = group * 8;
    if (at >= a.total) return;
    const T* x = static_cast<const T*>(a.x);
    T* y = static_cast<T*>(a.y);
    read_seed(&k);
    float f[8];
    uint32_t w[4];
    if constexpr (FLAT) {
        const int count = a.total - at < 8 ? (int)(a.total - at) : 8;
        load8(x + at, count, f);
        drawn(k, (unsigned long long)group, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = kept(k, w, e) ? f[e] * k.factor : 0.f;
        store8(y + at, count, f);
    } else {
        // columns are below 2^31 and what a workgroup takes is small: 32 bits
        const long long row0 = begin * 8 / a.dim, col0 = begin * 8 - row0 * a.dim;
        const uint32_t along = (uint32_t)col0 + 8u * threadIdx.x, over = along / (uint32_t)a.dim;
        long long row = row0 + over, col = along - over * (uint32_t)a.dim;
        if (col + 8 <= a.dim) {
            load8(x + row * a.x_stride + col, 8, f);
            drawn(k, (unsigned long long)group, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = kept(k, w, e) ? f[e] * k.factor : 0.f;
            store8(y + row * a.y_stride + col, 8, f);
        } else {
            drawn(k, (unsigned long long)group, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (row < a.rows) y[row * a.y_stride + col] = kept(k, w, e) ? from_f32<T>(to_f32(x[row * a.x_stride + col]) * k.factor) : from_f32<T>(0.f);
                if (++col == a.dim) { col = 0; ++row; }
            }
        }
    }
}

template <typename T> void go(Args a, hipStream_t st) {
    const bool flat = a.rows == 1 || (a.x_stride == a.dim && a.y_stride == a.dim);
    const long long groups = (a.total + 7) / 8, most = most_workgroups(kThreads) * kThreads;
    for (a.first = 0; a.first < groups; a.first += most) {
        const long long left = groups - a.first < most ? groups - a.first : most;
        const dim3 grid((unsigned)((left + kThreads - 1) / kThreads));
        if (flat) hipLaunchKernelGGL((k_dropout<T, true>), grid, kThreads, 0, st, a);
        else hipLaunchKernelGGL((k_dropout<T, false>), grid, kThreads, 0, st, a);
    }
}

}  // namespace
}  // namespace asi

using namespace asi;

extern "C" asi_status asi_dropout(const asi_dropout_desc* desc, const void* x, const int64_t* seed, void* y, asi_stream_t stream) {
    if (!desc || desc->rows < 0 || desc->dim < 1 || desc->x_stride < desc->dim || desc->y_stride < desc->dim || desc->reserved != 0) return ASI_ERR_INVALID_ARG;
    Args a{};
    if (!fill_keep(desc->p, desc->seed, desc->offset, seed, &a.keep) || !aligned(seed, 8)) return ASI_ERR_INVALID_ARG;
    if (!dtype_ok(desc->dtype)) return ASI_ERR_UNSUPPORTED;
    const int64_t limit = int64_t(1) << 31;
    if (desc->rows == 0) return ASI_OK;
    // rows that lie behind each other are one row of any length; others are counted in 32 bits
    const bool flat = desc->rows == 1 || (desc->x_stride == desc->dim && desc->y_stride == desc->dim);
    if ((!flat && desc->dim >= limit) || desc->rows > (int64_t(1) << 44) / desc->dim) return ASI_ERR_UNSUPPORTED;
    const size_t es = dtype_size(desc->dtype);
    if (!x || !y || !aligned(x, es) || !aligned(y, es) || (x == y && desc->rows > 1 && desc->x_stride != desc->y_stride)) return ASI_ERR_INVALID_ARG;
    a.x = x; a.y = y;
    a.rows = desc->rows; a.dim = desc->dim; a.x_stride = desc->x_stride; a.y_stride = desc->y_stride; a.total = desc->rows * desc->dim;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (desc->dtype == ASI_F32) go<float>(a, st);
    else go<bf16_t>(a, st);
    return launched();
}
