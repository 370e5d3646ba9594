// Root-mean-square norm of rows with the residual's addition and an 8-bit output, and its gradients.

#include "rows_device.h"

namespace aug {
namespace {

// One wavefront per row: the sum of squares, then block by block the largest magnitude and the outputs.
template <class T>
__global__ __launch_bounds__(64) void norm_kernel(NormArgs a) {
    const int lane = threadIdx.x, dim = a.cfg.dim;
    const int64_t r = blockIdx.x;
    const T* x = row_in<T>(a.x, r);
    const T* res = a.residual.data ? row_in<T>(a.residual, r) : nullptr;
    float ss = 0.f;
    for (int d = lane; d < dim; d += 64) {
        const float s = (float)x[d] + (res ? (float)res[d] : 0.f);
        ss += s * s;
    }
    const float rstd = 1.f / sqrtf(wave_sum(ss) / (float)dim + a.cfg.eps);
    if (a.rstd && lane == 0) a.rstd[r] = rstd;
    const int width = a.cfg.q_block ? a.cfg.q_block : dim, n_blocks = (dim + width - 1) / width;
    for (int b = 0; b < n_blocks; ++b) {
        const int from = b * width, to = min(from + width, dim);
        float scale = 0.f;
        if (a.q.data) {
            unsigned most = 0;
            for (int d = from + lane; d < to; d += 64) {
                const float s = (float)x[d] + (res ? (float)res[d] : 0.f);
                const unsigned m = __float_as_uint(s * rstd * (a.weight ? a.weight[d] : 1.f)) & 0x7fffffffu;
                most = most > m ? most : m;
            }
            scale = __uint_as_float(wave_max(most)) / 448.f;
            if (lane == 0) a.scale[r * n_blocks + b] = scale;
        }
        for (int d = from + lane; d < to; d += 64) {
            const float s = (float)x[d] + (res ? (float)res[d] : 0.f);
            const float y = s * rstd * (a.weight ? a.weight[d] : 1.f);
            if (a.sum.data) row_out<T>(a.sum, r)[d] = (T)s;
            if (a.y.data) row_out<T>(a.y, r)[d] = (T)y;
            if (a.q.data) {
                const float v = scale == 0.f ? 0.f : y / scale;
                row_out<uint8_t>(a.q, r)[d] = (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false) & 0xff);
            }
        }
    }
}

// dweight's part of 64 rows, a thread per column.
template <class T>
__global__ __launch_bounds__(64) void norm_dweight_kernel(NormBackArgs a, int rows) {
    const int d = blockIdx.x * 64 + threadIdx.x;
    if (d >= a.dim) return;
    float acc = 0.f;
    const int64_t from = (int64_t)blockIdx.y * rows, to = min(from + rows, a.n_rows);
    for (int64_t r = from; r < to; ++r) acc += (float)row_in<T>(a.dy, r)[d] * ((float)row_in<T>(a.sum, r)[d] * a.rstd[r]);
    a.partial[(int64_t)blockIdx.y * a.dim + d] = acc;
}

template <class T>
__global__ __launch_bounds__(64) void norm_backward_kernel(NormBackArgs a) {
    const int lane = threadIdx.x;
    const int64_t r = blockIdx.x;
    const T* x = row_in<T>(a.sum, r);
    const T* dy = row_in<T>(a.dy, r);
    const float rstd = a.rstd[r];
    float dot = 0.f;
    for (int d = lane; d < a.dim; d += 64) dot += (float)x[d] * ((float)dy[d] * (a.weight ? a.weight[d] : 1.f));
    const float slope = wave_sum(dot) / (float)a.dim * rstd * rstd * rstd;
    for (int d = lane; d < a.dim; d += 64) {
        float g = (float)dy[d] * (a.weight ? a.weight[d] : 1.f) * rstd - (float)x[d] * slope;
        if (a.dsum.data) g += (float)row_in<T>(a.dsum, r)[d];
        row_out<T>(a.dx, r)[d] = (T)g;
    }
}

int rows_per_partial(int64_t n_rows) { return (int)((n_rows + 1023) / 1024 < 64 ? 64 : (n_rows + 1023) / 1024); }

}  // namespace

hipError_t launch_norm(hipStream_t s, const NormArgs& a, int) {
    return with_type(a.cfg.dtype, [&](auto t) {
        norm_kernel<decltype(t)><<<dim3((unsigned)a.n_rows), dim3(64), 0, s>>>(a);
        return hipGetLastError();
    });
}

int norm_partials(int64_t n_rows, int, int) { return (int)((n_rows + rows_per_partial(n_rows) - 1) / rows_per_partial(n_rows)); }

hipError_t launch_norm_backward(hipStream_t s, const NormBackArgs& a, int n_cu) {
    return with_type(a.dtype, [&](auto t) {
        if (a.dweight) {                 // first: dx may take dy's place
            const int n = norm_partials(a.n_rows, a.dim, n_cu);
            norm_dweight_kernel<decltype(t)><<<dim3((unsigned)((a.dim + 63) / 64), (unsigned)n), dim3(64), 0, s>>>(a, rows_per_partial(a.n_rows));
            hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            e = launch_sum_partials(s, a.partial, n, a.dim, {{{a.dweight, a.dim}, {}, {}}});
            if (e != hipSuccess) return e;
        }
        if (a.dx.data) norm_backward_kernel<decltype(t)><<<dim3((unsigned)a.n_rows), dim3(64), 0, s>>>(a);
        return hipGetLastError();
    });
}

}  // namespace aug
