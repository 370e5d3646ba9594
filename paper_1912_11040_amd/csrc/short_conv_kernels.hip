// Short causal convolution along time, a filter per channel: rows of packed sequences, its gradients, and single rows of streams.

#include "rows_device.h"

namespace aug {
namespace {

constexpr int kChannels = 64, kWaves = 4, kLgBlock = 6;

// Row t of the sequence that begins at row `begin`, those before it from the state (zeros without one).
template <class T>
__device__ inline float row_at(const ShortConvArgs& a, int seq, int64_t begin, int64_t t, int d) {
    const int held = a.cfg.taps - 1;
    if (t >= 0) return (float)row_in<T>(a.x, begin + t)[d];
    return a.state_in ? (float)static_cast<const T*>(a.state_in)[((int64_t)seq * held + held + t) * a.cfg.dim + d] : 0.f;
}

template <class T>
__device__ inline float filtered(const ShortConvArgs& a, int seq, int64_t begin, int64_t t, int d) {
    float p = a.bias ? a.bias[d] : 0.f;
    for (int k = 0; k < a.cfg.taps; ++k)
        p = fmaf(a.weight[(int64_t)d * a.cfg.taps + k], row_at<T>(a, seq, begin, t - (a.cfg.taps - 1) + k, d), p);
    return p;
}

// A group: 64 channels of a block of rows, every fourth row a wavefront's.
template <class T>
__global__ __launch_bounds__(64 * kWaves) void short_conv_kernel(ShortConvArgs a) {
    const int2 item = a.rows.items[blockIdx.x];
    const int d = blockIdx.y * kChannels + threadIdx.x % 64, wave = threadIdx.x / 64, seq = item.x;
    const int64_t begin = a.rows.begin[seq], len = a.rows.end[seq] - begin;
    const int64_t from = (int64_t)item.y << a.rows.lg, to = min(from + (1 << a.rows.lg), len);
    if (d < a.cfg.dim)
        for (int64_t t = from + wave; t < to; t += kWaves) {
            const float p = filtered<T>(a, seq, begin, t, d);
            row_out<T>(a.y, begin + t)[d] = (T)(a.cfg.silu ? p * sigmoid(p) : p);
        }
    // Only a sequence's first group reads the state, so it may write it in place once all of it has.
    if (!a.state_out || item.y != 0) return;
    __syncthreads();
    if (d >= a.cfg.dim || wave != 0) return;
    const int held = a.cfg.taps - 1;
    T* const out = static_cast<T*>(a.state_out) + (int64_t)seq * held * a.cfg.dim + d;
    float v[AUG_MAX_TAPS - 1];
    for (int k = 0; k < held; ++k) v[k] = row_at<T>(a, seq, begin, len - held + k, d);
    for (int k = 0; k < held; ++k) out[(int64_t)k * a.cfg.dim] = (T)v[k];
}

template <class T>
__device__ inline float dfiltered(const ShortConvArgs& a, int seq, int64_t begin, int64_t t, int d) {
    const float dy = (float)row_in<T>(a.dy, begin + t)[d];
    if (!a.cfg.silu) return dy;
    const float p = filtered<T>(a, seq, begin, t, d), sg = sigmoid(p);
    return dy * sg * (1.f + p * (1.f - sg));
}

template <class T>
__global__ __launch_bounds__(64) void short_conv_backward_kernel(ShortConvArgs a) {
    const int2 item = a.rows.items[blockIdx.x];
    const int d = blockIdx.y * kChannels + threadIdx.x, seq = item.x, taps = a.cfg.taps;
    if (d >= a.cfg.dim) return;
    const int64_t begin = a.rows.begin[seq], len = a.rows.end[seq] - begin;
    const int64_t from = (int64_t)item.y << a.rows.lg, to = min(from + (1 << a.rows.lg), len);
    float dw[AUG_MAX_TAPS] = {}, db = 0.f;
    for (int64_t t = from; t < to; ++t) {
        const float dp = dfiltered<T>(a, seq, begin, t, d);
        db += dp;
        for (int k = 0; k < taps; ++k) dw[k] = fmaf(dp, row_at<T>(a, seq, begin, t - (taps - 1) + k, d), dw[k]);
        if (a.dx.data) {
            float dx = 0.f;
            for (int k = 0; k < taps; ++k)
                if (t + taps - 1 - k < len) dx = fmaf(a.weight[(int64_t)d * taps + k], dfiltered<T>(a, seq, begin, t + taps - 1 - k, d), dx);
            row_out<T>(a.dx, begin + t)[d] = (T)dx;
        }
    }
    if (!a.partial) return;
    float* const out = a.partial + (int64_t)blockIdx.x * a.cfg.dim * (taps + 1);
    for (int k = 0; k < taps; ++k) out[(int64_t)d * taps + k] = dw[k];
    out[(int64_t)a.cfg.dim * taps + d] = db;
}

template <class T>
__global__ __launch_bounds__(64) void short_conv_step_kernel(ShortConvArgs a) {
    const int d = blockIdx.y * kChannels + threadIdx.x, held = a.cfg.taps - 1;
    const int64_t i = blockIdx.x;
    if (d >= a.cfg.dim) return;
    const T* const in = static_cast<const T*>(a.state_in) + i * held * a.cfg.dim + d;
    T* const out = static_cast<T*>(a.state_out) + i * held * a.cfg.dim + d;
    const T x = row_in<T>(a.x, i)[d];
    T v[AUG_MAX_TAPS];
    for (int k = 0; k < held; ++k) v[k] = in[(int64_t)k * a.cfg.dim];
    v[held] = x;
    float p = a.bias ? a.bias[d] : 0.f;
    for (int k = 0; k <= held; ++k) p = fmaf(a.weight[(int64_t)d * a.cfg.taps + k], (float)v[k], p);
    for (int k = 0; k < held; ++k) out[(int64_t)k * a.cfg.dim] = v[k + 1];
    row_out<T>(a.y, i)[d] = (T)(a.cfg.silu ? p * sigmoid(p) : p);
}

unsigned tiles(int dim) { return (unsigned)((dim + kChannels - 1) / kChannels); }

}  // namespace

int short_conv_lg_block(const aug_short_conv_cfg&, bool) { return kLgBlock; }
int short_conv_partials(const aug_short_conv_cfg&, int n_items, int) { return n_items; }

hipError_t launch_short_conv(hipStream_t s, const ShortConvArgs& a) {
    return with_type(a.cfg.dtype, [&](auto t) {
        short_conv_kernel<decltype(t)><<<dim3((unsigned)a.rows.n_items, tiles(a.cfg.dim)), dim3(64 * kWaves), 0, s>>>(a);
        return hipGetLastError();
    });
}

hipError_t launch_short_conv_backward(hipStream_t s, const ShortConvArgs& a, int) {
    hipError_t e = with_type(a.cfg.dtype, [&](auto t) {
        short_conv_backward_kernel<decltype(t)><<<dim3((unsigned)a.rows.n_items, tiles(a.cfg.dim)), dim3(64), 0, s>>>(a);
        return hipGetLastError();
    });
    const int64_t w = (int64_t)a.cfg.dim * a.cfg.taps, stride = w + a.cfg.dim;
    if (e == hipSuccess && a.partial) e = launch_sum_partials(s, a.partial, a.rows.n_items, stride, {{{a.dweight, w}, {a.dbias, a.cfg.dim}, {}}});
    return e;
}

hipError_t launch_short_conv_step(hipStream_t s, int n_seq, const ShortConvArgs& a) {
    return with_type(a.cfg.dtype, [&](auto t) {
        short_conv_step_kernel<decltype(t)><<<dim3((unsigned)n_seq, tiles(a.cfg.dim)), dim3(64), 0, s>>>(a);
        return hipGetLastError();
    });
}

}  // namespace aug
