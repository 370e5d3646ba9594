// Root-mean-square norm of rows with the residual's addition and an 8-bit output, and its gradients.
//
// Both are bound by memory.  A row belongs to TPR lanes, each with NV stretches of eight columns in registers from the first read
// to the last write, so that every matrix goes over the bus once; lanes go from row to row with their columns' weights (and
// the weights' gradients) in registers.

#include <type_traits>

#include "rows_device.h"

namespace aug {
namespace {

constexpr int kVec = 8;
template <int TPR> constexpr int kThreads = TPR < 256 ? 256 : TPR;      // a group's

// The sum over a row's lanes, in all of them.
template <int TPR> __device__ inline float row_sum(float v, float* exchange) {
    v = lanes_sum<(TPR < 64 ? TPR : 64)>(v);
    if constexpr (TPR > 64) {
        __syncthreads();                                 // (the last row's sums have been read)
        if (threadIdx.x % 64 == 0) exchange[threadIdx.x / 64] = v;
        __syncthreads();
        v = exchange[0];
#pragma unroll
        for (int i = 1; i < TPR / 64; ++i) v += exchange[i];
    }
    return v;
}

// The largest of a row's lanes' values, in all of them.
template <int TPR> __device__ inline unsigned row_max(unsigned v, float* exchange) {
    v = lanes_max(v, TPR < 64 ? TPR : 64);
    if constexpr (TPR > 64) {
        __syncthreads();                                 // (the last ones have been read)
        if (threadIdx.x % 64 == 0) exchange[threadIdx.x / 64] = __uint_as_float(v);
        __syncthreads();
        for (int i = 0; i < TPR / 64; ++i) v = max(v, __float_as_uint(exchange[i]));
    }
    return v;
}

template <int NV> __device__ inline float squares(const float (&s)[NV][kVec]) {
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float part = 0.f;                                // (the squares of a stretch by themselves: shorter sums)
#pragma unroll
        for (int i = 0; i < kVec; ++i) part = fmaf(s[j][i], s[j][i], part);
        ss += part;
    }
    return ss;
}

template <class T, int TPR, int NV>
__global__ __launch_bounds__(kThreads<TPR>) void norm_kernel(NormArgs a) {
    __shared__ float exchange[32];
    const int lane = threadIdx.x % TPR, dim = a.cfg.dim;
    const int64_t step = (int64_t)gridDim.x * (kThreads<TPR> / TPR);
    const int width = a.cfg.q_block && a.cfg.q_block < kVec * TPR ? a.cfg.q_block : dim;      // columns of a block; no block ends inside a lane's eight
    const bool whole = width >= dim;
    const int n_blocks = a.cfg.q_block ? (dim + a.cfg.q_block - 1) / a.cfg.q_block : 1;
    const float least = a.cfg.eps < 0x1p-120f ? 0x1p-100f : 0.f;      // of a sum of squares that nothing is lost of next to eps
    float w[NV][kVec];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * TPR + lane) * kVec;
        const Pack<float, kVec> v = a.weight ? load_pack<float, kVec>(a.weight + c, dim - c) : Pack<float, kVec>{1, 1, 1, 1, 1, 1, 1, 1};
#pragma unroll
        for (int i = 0; i < kVec; ++i) w[j][i] = v.v[i];
    }
    for (int64_t r = (int64_t)blockIdx.x * (kThreads<TPR> / TPR) + threadIdx.x / TPR; r < a.n_rows; r += step) {
        float s[NV][kVec];
        Pack<T, kVec> x[NV], res[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TPR + lane) * kVec;
            x[j] = load_pack<T, kVec>(row_in<T>(a.x, r) + c, dim - c);
            if (a.residual.data) res[j] = load_pack<T, kVec>(row_in<T>(a.residual, r) + c, dim - c);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TPR + lane) * kVec;
#pragma unroll
            for (int i = 0; i < kVec; ++i) s[j][i] = (float)x[j].v[i] + (a.residual.data ? (float)res[j].v[i] : 0.f);
            if (a.sum.data) {
                Pack<T, kVec> out;
#pragma unroll
                for (int i = 0; i < kVec; ++i) out.v[i] = (T)s[j][i];
                store_pack<T, kVec>(row_out<T>(a.sum, r) + c, out, dim - c);
            }
        }
        float total = row_sum<TPR>(squares(s), exchange), eps = a.cfg.eps;
        int e = 0;
        // Squares out of the range of 32 bits (or NaN), where the row's values are not and eps does not outweigh what is lost: the row is divided
        // by a power of two first, of its largest value or of eps' root.  (Nothing helps a row that holds a NaN or an infinity.)  The question costs
        // 16-bit rows 2 % (64 utterances of 2048 columns into 8 bits 152.6 us without it, 155.5 with), 32-bit ones nothing.
        if (__builtin_expect(__builtin_amdgcn_fmed3f(total, least, 3.4e38f) != total, 0)) {
            unsigned most = 0;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < kVec; ++i) most = max(most, __float_as_uint(s[j][i]) & 0x7fffffffu);
            most = row_max<TPR>(most, exchange + 16);
            if (most > 0 && most < 0x7f800000u) {
                e = (int)(most >> 23) - 127;
                if (eps > 0.f) e = max(e, ((int)(__float_as_uint(eps) >> 23) - 127) / 2);
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < kVec; ++i) s[j][i] = ldexpf(s[j][i], -e);
                total = row_sum<TPR>(squares(s), exchange);
                eps = ldexpf(eps, -2 * e);
            }
        }
        const float rstd = 1.f / sqrtf(total / (float)dim + eps);      // of the row divided by 2^e
        if (a.rstd && lane == 0) a.rstd[r] = ldexpf(rstd, -e);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TPR + lane) * kVec;
#pragma unroll
            for (int i = 0; i < kVec; ++i) s[j][i] *= rstd * w[j][i];
            if (a.y.data) {
                Pack<T, kVec> out;
#pragma unroll
                for (int i = 0; i < kVec; ++i) out.v[i] = (T)s[j][i];
                store_pack<T, kVec>(row_out<T>(a.y, r) + c, out, dim - c);
            }
        }
        if (!a.q.data) continue;
        // the largest magnitude by its bits: a NaN's are larger than any number's
        unsigned most[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            most[j] = 0;
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const unsigned m = __float_as_uint(s[j][i]) & 0x7fffffffu;
                most[j] = most[j] > m ? most[j] : m;
            }
        }
        if (whole) {
#pragma unroll
            for (int j = 1; j < NV; ++j) most[0] = most[0] > most[j] ? most[0] : most[j];
            most[0] = row_max<TPR>(most[0], exchange + 16);
#pragma unroll
            for (int j = 1; j < NV; ++j) most[j] = most[0];
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TPR + lane) * kVec;
            if (!whole) most[j] = lanes_max(most[j], width / kVec);
            float scale = __uint_as_float(most[j]) / 448.f;
            float by = scale;
            if (__builtin_expect(scale < 0x1p-126f, 0)) {      // not a normal number: rounded down, y / scale may be beyond e4m3's largest
                if (scale * 448.f < __uint_as_float(most[j])) scale = __uint_as_float(__float_as_uint(scale) + 1);
                by = scale == 0.f ? 1.f : scale;
            }
            if (c < dim && (whole ? c == 0 : c % width == 0)) a.scale[r * n_blocks + (whole ? 0 : c / width)] = scale;
            Pack<unsigned, 2> out;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                unsigned v = __builtin_amdgcn_cvt_pk_fp8_f32(s[j][4 * i] / by, s[j][4 * i + 1] / by, 0, false);
                out.v[i] = __builtin_amdgcn_cvt_pk_fp8_f32(s[j][4 * i + 2] / by, s[j][4 * i + 3] / by, v, true);
            }
            Pack<uint8_t, kVec> bytes;
            __builtin_memcpy(bytes.v, out.v, kVec);
            store_pack<uint8_t, kVec>(row_out<uint8_t>(a.q, r) + c, bytes, dim - c);
        }
    }
}

template <class T, int TPR, int NV>
__global__ __launch_bounds__(kThreads<TPR>) void norm_backward_kernel(NormBackArgs a) {
    constexpr int kGroups = kThreads<TPR> / TPR;
    __shared__ float exchange[16];
    __shared__ float sums[TPR >= 256 ? 1 : kGroups][TPR >= 256 ? 1 : TPR * NV * kVec];
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR, dim = a.dim;
    float w[NV][kVec], dw[NV][kVec] = {};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * TPR + lane) * kVec;
        const Pack<float, kVec> v = a.weight ? load_pack<float, kVec>(a.weight + c, dim - c) : Pack<float, kVec>{1, 1, 1, 1, 1, 1, 1, 1};
#pragma unroll
        for (int i = 0; i < kVec; ++i) w[j][i] = v.v[i];
    }
    for (int64_t r = (int64_t)blockIdx.x * kGroups + group; r < a.n_rows; r += (int64_t)gridDim.x * kGroups) {
        const float rstd = a.rstd[r];
        Pack<T, kVec> x[NV], dy[NV], ds[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TPR + lane) * kVec;
            x[j] = load_pack<T, kVec>(row_in<T>(a.sum, r) + c, dim - c);
            dy[j] = load_pack<T, kVec>(row_in<T>(a.dy, r) + c, dim - c);
            if (a.dsum.data) ds[j] = load_pack<T, kVec>(row_in<T>(a.dsum, r) + c, dim - c);
        }
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                // (the normalised row as one value in both sums, and again below, would be kept: 18 to 48 registers too many at 16384 columns)
                const float xi = (float)x[j].v[i], g = (float)dy[j].v[i];
                part = fmaf(xi * rstd, g * w[j][i], part);
                dw[j][i] = fmaf(g * rstd, xi, dw[j][i]);
            }
            dot += part;
        }
        if (!a.dx.data) continue;
        // dx = rstd (w dy - x rstd mean(x rstd w dy)): the powers of rstd by themselves leave the range of 32 bits at rows of 1e13
        const float slope = row_sum<TPR>(dot, exchange) / (float)dim;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * TPR + lane) * kVec;
            Pack<T, kVec> out;
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                float g = rstd * fmaf(-(float)x[j].v[i] * rstd, slope, (float)dy[j].v[i] * w[j][i]);
                if (a.dsum.data) g += (float)ds[j].v[i];
                out.v[i] = (T)g;
            }
            store_pack<T, kVec>(row_out<T>(a.dx, r) + c, out, dim - c);
        }
    }
    if (!a.partial) return;
    float* const out = a.partial + (int64_t)blockIdx.x * dim;
    if constexpr (TPR >= 256) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if ((j * TPR + lane) * kVec + i < dim) out[(j * TPR + lane) * kVec + i] = dw[j][i];
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < kVec; ++i) sums[group][(j * TPR + lane) * kVec + i] = dw[j][i];
        __syncthreads();
        for (int c = threadIdx.x; c < dim; c += kThreads<TPR>) {
            float sum = 0.f;
            for (int g = 0; g < kGroups; ++g) sum += sums[g][c];
            out[c] = sum;
        }
    }
}

// How a row of so many columns is dealt out: lanes per row, stretches per lane, and how many work groups go through the rows together per
// compute unit.
struct RowShape {
    int lanes, vecs, groups;
};
// Forward: a row's whole width to a group where it takes one, so that many wavefronts have loads on their way (64 utterances at 2048
// columns into 8 bits 198 us with a wavefront per row; 32 groups a compute unit 149, 16 162, 8 183: the last round is half empty).
constexpr RowShape forward_shape(int dim) {
    return dim <= 128 ? RowShape{16, 1, 16} : dim <= 512 ? RowShape{64, 1, 16} : dim <= 2048 ? RowShape{256, 1, 32}
         : dim <= 4096 ? RowShape{512, 1, 8} : dim <= 8192 ? RowShape{1024, 1, 4} : RowShape{1024, 2, 4};
}
// Gradients: each group leaves a row of sums, so few groups with much on their way each (20011 rows of 1001 columns: 69 us, with four groups a
// compute unit 12 more, with a group per row 10.  20000 of 2048: 85, with a wavefront per row 106).
constexpr RowShape backward_shape(int dim) {
    return dim <= 128 ? RowShape{16, 1, 4} : dim <= 512 ? RowShape{64, 1, 4} : dim <= 1024 ? RowShape{64, 2, 2} : dim <= 2048 ? RowShape{256, 1, 4}
         : dim <= 4096 ? RowShape{512, 1, 2} : dim <= 8192 ? RowShape{1024, 1, 1} : RowShape{1024, 2, 1};
}
// Calls f with a shape's lanes and stretches.
template <class F> hipError_t with_shape(const RowShape& s, F f) {
    using std::integral_constant;
    if (s.lanes == 16) return f(integral_constant<int, 16>(), integral_constant<int, 1>());
    if (s.lanes == 64 && s.vecs == 1) return f(integral_constant<int, 64>(), integral_constant<int, 1>());
    if (s.lanes == 64) return f(integral_constant<int, 64>(), integral_constant<int, 2>());
    if (s.lanes == 256) return f(integral_constant<int, 256>(), integral_constant<int, 1>());
    if (s.lanes == 512) return f(integral_constant<int, 512>(), integral_constant<int, 1>());
    if (s.vecs == 1) return f(integral_constant<int, 1024>(), integral_constant<int, 1>());
    return f(integral_constant<int, 1024>(), integral_constant<int, 2>());
}
int row_groups(int64_t n_rows, const RowShape& s, int n_cu) {
    const int64_t rows = s.lanes < 256 ? 256 / s.lanes : 1, groups = (n_rows + rows - 1) / rows, most = (int64_t)s.groups * n_cu;
    return (int)(groups < most ? groups : most);
}

}  // namespace

hipError_t launch_norm(hipStream_t s, const NormArgs& a, int n_cu) {
    return with_type(a.cfg.dtype, [&](auto t) {
        const RowShape shape = forward_shape(a.cfg.dim);
        return with_shape(shape, [&](auto tpr, auto nv) {
            norm_kernel<decltype(t), tpr.value, nv.value><<<dim3((unsigned)row_groups(a.n_rows, shape, n_cu)), dim3(kThreads<tpr.value>), 0, s>>>(a);
            return hipGetLastError();
        });
    });
}

int norm_partials(int64_t n_rows, int dim, int n_cu) { return row_groups(n_rows, backward_shape(dim), n_cu); }

hipError_t launch_norm_backward(hipStream_t s, const NormBackArgs& a, int n_cu) {
    const int groups = norm_partials(a.n_rows, a.dim, n_cu);
    hipError_t e = with_type(a.dtype, [&](auto t) {
        return with_shape(backward_shape(a.dim), [&](auto tpr, auto nv) {
            norm_backward_kernel<decltype(t), tpr.value, nv.value><<<dim3((unsigned)groups), dim3(kThreads<tpr.value>), 0, s>>>(a);
            return hipGetLastError();
        });
    });
    if (e == hipSuccess && a.dweight) e = launch_sum_partials(s, a.partial, groups, a.dim, {{{a.dweight, a.dim}, {}, {}}});
    return e;
}

}  // namespace aug
