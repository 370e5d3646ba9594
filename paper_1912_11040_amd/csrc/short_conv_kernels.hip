// Short causal convolution along time, a filter per channel: rows of packed sequences, its gradients, and single rows of streams.
//
// Bound by memory: an element is read once and written once for a few operations.  A lane takes a few neighbouring channels
// down some consecutive rows, the last taps - 1 of them always in registers, and asks for four rows at a time while it works on
// the four before.  Lanes of a group that have no channels left to take (narrow rows) take further rows.

#include <type_traits>

#include "rows_device.h"

namespace aug {
namespace {

constexpr int kThreads = 256;

// Channels and rows of a lane, forward and for the gradients, which keep the taps' too: with 8 and 4 channels fewer wavefronts fit and the loads
// are wider, which comes to the same forward (64 utterances of 2048 channels 95 us, the memory's rate) and to more for the gradients (206
// instead of 171); 16 rows instead of 32 read more of them twice (96 short utterances' gradients 56 instead of 48 us), 32 forward leave a
// small batch fewer groups (40 channels 18 instead of 15).
constexpr int kVec = 4, kBackVec = 2, kRows = 16, kBackRows = 32;
// Lanes across a row, a power of two up to 64.
__host__ __device__ inline int lanes_across(int dim, int vec) {
    int n = 1;
    while (n < 64 && n * vec < dim) n *= 2;
    return n;
}
int tiles_of(const aug_short_conv_cfg& cfg, int vec) {
    const int wide = lanes_across(cfg.dim, vec) * vec;
    return (cfg.dim + wide - 1) / wide;
}
int lg_rows(const aug_short_conv_cfg& cfg, int vec, int rows) {      // of a group's block
    int lg = 0;
    while ((1 << lg) < kThreads / lanes_across(cfg.dim, vec) * rows) ++lg;
    return lg;
}

// Rows t < 0 are those of the state (or zeros), oldest first.
template <class T, int VE>
__device__ inline Pack<T, VE> row_before(const ShortConvArgs& a, int seq, int64_t t, int col, int valid) {
    const int held = a.cfg.taps - 1;
    if (!a.state_in) return load_pack<T, VE>(static_cast<const T*>(nullptr), 0);
    return load_pack<T, VE>(static_cast<const T*>(a.state_in) + ((int64_t)seq * held + held + t) * a.cfg.dim + col, valid);
}

template <class T, int VE, int W>
__device__ inline void load_taps(const ShortConvArgs& a, int col, int valid, float (&w)[W][VE], float (&bias)[VE]) {
    const Pack<float, VE * W> all = load_pack<float, VE * W>(a.weight + (int64_t)col * W, valid * W);
    const Pack<float, VE> b = load_pack<float, VE>(a.bias + col, a.bias ? valid : 0);
#pragma unroll
    for (int i = 0; i < VE; ++i) {
        bias[i] = b.v[i];
#pragma unroll
        for (int k = 0; k < W; ++k) w[k][i] = all.v[i * W + k];
    }
}

template <class T, int W, bool FULL>
__global__ __launch_bounds__(kThreads) void short_conv_kernel(ShortConvArgs a, int tiles) {
    constexpr int VE = kVec, kAhead = 4;
    const int across = lanes_across(a.cfg.dim, VE), sub = threadIdx.x / across;
    const int col = ((int)(blockIdx.x % tiles) * across + threadIdx.x % across) * VE, valid = a.cfg.dim - col;
    const int2 item = a.rows.items[blockIdx.x / tiles];
    const int seq = item.x;
    const int64_t begin = a.rows.begin[seq], len = a.rows.end[seq] - begin;
    const int64_t from = ((int64_t)item.y << a.rows.lg) + sub * kRows;
    const int rows = (int)min(len - from, (int64_t)kRows);
    const bool keeps = a.state_out && from == 0;         // the lane that reads the state writes it, behind its reads
    if (valid <= 0 || (rows <= 0 && !keeps)) return;
    float w[W][VE], bias[VE];
    load_taps<T, VE, W>(a, col, valid, w, bias);
    // row `from` + j; behind the lane's rows the last one again, of which nothing is stored
    auto row = [&](int j) { return load_part<T, VE, FULL>(a.x, begin + from + min(j, rows - 1), col, valid); };
    Pack<T, VE> x[W - 1 + kAhead], next[kAhead] = {};
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int64_t t = from + j - (W - 1);
        x[j] = t < 0 ? row_before<T, VE>(a, seq, t, col, valid) : load_part<T, VE, FULL>(a.x, begin + t, col, valid);
    }
    if (rows > 0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) next[j] = row(j);
    }
    for (int r = 0; r < rows; r += kAhead) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) x[W - 1 + j] = next[j];
        if (r + kAhead < rows) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) next[j] = row(r + kAhead + j);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            float p[VE];
            Pack<T, VE> y;
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                p[i] = bias[i];
#pragma unroll
                for (int k = 0; k < W; ++k) p[i] = fmaf(w[k][i], (float)x[j + k].v[i], p[i]);
            }
            if (a.cfg.silu) {
#pragma unroll
                for (int i = 0; i < VE; ++i) p[i] *= sigmoid(p[i]);
            }
#pragma unroll
            for (int i = 0; i < VE; ++i) y.v[i] = (T)p[i];
            if (r + j < rows) store_part<T, VE, FULL>(a.y, begin + from + r + j, col, y, valid);
        }
#pragma unroll
        for (int j = 0; j < W - 1; ++j) x[j] = x[kAhead + j];
    }
    if (!keeps) return;
    // the last W - 1 of the state's rows and the sequence's; a row of the state is read before its place is written (it is never an
    // earlier one)
    T* const out = static_cast<T*>(a.state_out) + (int64_t)seq * (W - 1) * a.cfg.dim + col;
    for (int k = 0; k < W - 1; ++k) {
        const int64_t t = len - (W - 1) + k;
        const Pack<T, VE> v = t < 0 ? row_before<T, VE>(a, seq, t, col, valid) : load_pack<T, VE>(row_in<T>(a.x, begin + t) + col, valid);
        store_pack<T, VE>(out + (int64_t)k * a.cfg.dim, v, valid);
    }
}

// Gradients.  dx of a row needs dp of the taps - 1 rows behind it: a lane works them out too, for a tenth more operations at four taps
// and 32 rows, and keeps the last taps rows of x and of dp in registers.  The groups go through a run of blocks each with the
// gradients of their channels' taps in registers.
template <class T, int W, bool FULL>
__global__ __launch_bounds__(kThreads) void short_conv_backward_kernel(ShortConvArgs a, int tiles, int runs) {
    constexpr int VE = kBackVec, kAhead = W == 1 || W == 2 || W == 4 ? 4 : W == 3 ? 3 : W;      // a multiple of W
    __shared__ float sums[kThreads][VE + 1];
    const int across = lanes_across(a.cfg.dim, VE), sub = threadIdx.x / across, subs = kThreads / across, lane = threadIdx.x % across;
    const int tile = blockIdx.x % tiles, run = blockIdx.x / tiles;
    const int col = (tile * across + lane) * VE, valid = a.cfg.dim - col;
    const int first = (int)((int64_t)a.rows.n_items * run / runs), end_item = (int)((int64_t)a.rows.n_items * (run + 1) / runs);
    float w[W][VE], bias[VE], dw[W][VE] = {}, db[VE] = {};
    load_taps<T, VE, W>(a, col, valid, w, bias);
    for (int it = first; it < end_item; ++it) {
        const int2 item = a.rows.items[it];
        const int seq = item.x;
        const int64_t begin = a.rows.begin[seq], len = a.rows.end[seq] - begin;
        const int64_t from = ((int64_t)item.y << a.rows.lg) + sub * kBackRows;
        const int rows = (int)min(len - from, (int64_t)kBackRows), there = (int)min(len - from, (int64_t)(kBackRows + W - 1));
        if (valid <= 0 || rows <= 0) continue;
        // row `from` + j; behind the sequence its last one again, whose dp is put to zero
        auto row = [&](const aug_rows& m, int j) { return load_part<T, VE, FULL>(m, begin + from + min(j, there - 1), col, valid); };
        float x[W][VE], dp[W][VE];                       // row j in place j mod W
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int64_t t = from + j - (W - 1);
            const Pack<T, VE> v = t < 0 ? row_before<T, VE>(a, seq, t, col, valid) : load_part<T, VE, FULL>(a.x, begin + t, col, valid);
#pragma unroll
            for (int i = 0; i < VE; ++i) x[(j + 1) % W][i] = (float)v.v[i];
        }
        Pack<T, VE> next_x[kAhead], next_dy[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            next_x[j] = row(a.x, j);
            next_dy[j] = row(a.dy, j);
        }
        for (int r = 0; r < rows + W - 1; r += kAhead) {
            Pack<T, VE> now_x[kAhead], now_dy[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                now_x[j] = next_x[j];
                now_dy[j] = next_dy[j];
            }
            if (r + kAhead < there) {
#pragma unroll
                for (int j = 0; j < kAhead; ++j) {
                    next_x[j] = row(a.x, r + kAhead + j);
                    next_dy[j] = row(a.dy, r + kAhead + j);
                }
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int slot = j % W;
                float p[VE];
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    x[slot][i] = (float)now_x[j].v[i];
                    dp[slot][i] = (float)now_dy[j].v[i];
                }
                if (a.cfg.silu) {
#pragma unroll
                    for (int i = 0; i < VE; ++i) {
                        p[i] = bias[i];
#pragma unroll
                        for (int k = 0; k < W; ++k) p[i] = fmaf(w[k][i], x[(slot + 1 + k) % W][i], p[i]);
                        const float sg = sigmoid(p[i]);
                        dp[slot][i] *= sg * (1.f + p[i] * (1.f - sg));
                    }
                }
                if (r + j >= there) {                    // rows behind the sequence give nothing, whatever is in their windows
#pragma unroll
                    for (int i = 0; i < VE; ++i) dp[slot][i] = 0.f;
                }
                if (r + j < rows) {
#pragma unroll
                    for (int i = 0; i < VE; ++i) {
                        db[i] += dp[slot][i];
#pragma unroll
                        for (int k = 0; k < W; ++k) dw[k][i] = fmaf(dp[slot][i], x[(slot + 1 + k) % W][i], dw[k][i]);
                    }
                }
                const int done = r + j - (W - 1);        // the row whose gradient is whole now
                if (a.dx.data && done >= 0 && done < rows) {
                    Pack<T, VE> out;
#pragma unroll
                    for (int i = 0; i < VE; ++i) {
                        float g = 0.f;
#pragma unroll
                        for (int k = 0; k < W; ++k) g = fmaf(w[k][i], dp[(slot + W - k) % W][i], g);
                        out.v[i] = (T)g;
                    }
                    store_part<T, VE, FULL>(a.dx, begin + from + done, col, out, valid);
                }
            }
        }
    }
    if (!a.partial) return;
    // over the lanes of a channel, first rows first, value by value
    float* const out = a.partial + (int64_t)run * a.cfg.dim * (W + 1);
#pragma unroll
    for (int k = 0; k <= W; ++k) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VE; ++i) sums[threadIdx.x][i] = k < W ? dw[k < W ? k : 0][i] : db[i];
        __syncthreads();
        for (int c = threadIdx.x; c < across * VE; c += kThreads) {
            const int64_t d = (int64_t)tile * across * VE + c;
            if (d >= a.cfg.dim) break;
            float sum = 0.f;
            for (int s = 0; s < subs; ++s) sum += sums[s * across + c / VE][c % VE];
            out[k < W ? d * W + k : (int64_t)a.cfg.dim * W + d] = sum;
        }
    }
}

template <class T, int W>
__global__ __launch_bounds__(64) void short_conv_step_kernel(ShortConvArgs a, int n_seq, int across, int tiles) {
    constexpr int VE = kVec;
    const int col = ((int)(blockIdx.x % tiles) * across + threadIdx.x % across) * VE, valid = a.cfg.dim - col;
    const int64_t i = (int64_t)(blockIdx.x / tiles) * (64 / across) + threadIdx.x / across;
    if (valid <= 0 || i >= n_seq) return;
    const T* const in = static_cast<const T*>(a.state_in) + i * (W - 1) * a.cfg.dim + col;
    T* const out = static_cast<T*>(a.state_out) + i * (W - 1) * a.cfg.dim + col;
    Pack<T, VE> x[W], y;
#pragma unroll
    for (int k = 0; k < W - 1; ++k) x[k] = load_pack<T, VE>(in + (int64_t)k * a.cfg.dim, valid);
    x[W - 1] = load_pack<T, VE>(row_in<T>(a.x, i) + col, valid);
    float w[W][VE], p[VE];
    load_taps<T, VE, W>(a, col, valid, w, p);
#pragma unroll
    for (int k = 0; k < W - 1; ++k) store_pack<T, VE>(out + (int64_t)k * a.cfg.dim, x[k + 1], valid);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
#pragma unroll
        for (int k = 0; k < W; ++k) p[j] = fmaf(w[k][j], (float)x[k].v[j], p[j]);
    }
    if (a.cfg.silu) {
#pragma unroll
        for (int j = 0; j < VE; ++j) p[j] *= sigmoid(p[j]);
    }
#pragma unroll
    for (int j = 0; j < VE; ++j) y.v[j] = (T)p[j];
    store_pack<T, VE>(row_out<T>(a.y, i) + col, y, valid);
}

template <class F> hipError_t with_taps(int taps, F f) {
    using std::integral_constant;
    switch (taps) {
        case 1: return f(integral_constant<int, 1>());
        case 2: return f(integral_constant<int, 2>());
        case 3: return f(integral_constant<int, 3>());
        case 4: return f(integral_constant<int, 4>());
        case 5: return f(integral_constant<int, 5>());
        case 6: return f(integral_constant<int, 6>());
        case 7: return f(integral_constant<int, 7>());
        default: return f(integral_constant<int, 8>());
    }
}

}  // namespace

int short_conv_tiles(const aug_short_conv_cfg& cfg, bool backward) { return tiles_of(cfg, backward ? kBackVec : kVec); }
int short_conv_lg_block(const aug_short_conv_cfg& cfg, bool backward) { return backward ? lg_rows(cfg, kBackVec, kBackRows) : lg_rows(cfg, kVec, kRows); }
int short_conv_partials(const aug_short_conv_cfg& cfg, int n_items, int n_cu) {
    const int64_t runs = (4 * (int64_t)n_cu + short_conv_tiles(cfg, true) - 1) / short_conv_tiles(cfg, true);
    return (int)(runs < n_items ? runs : n_items);
}

hipError_t launch_short_conv(hipStream_t s, const ShortConvArgs& a) {
    const int tiles = short_conv_tiles(a.cfg, false);
    return with_type(a.cfg.dtype, [&](auto t) {
        return with_taps(a.cfg.taps, [&](auto w) {
            return with_full(a.cfg.dim % kVec == 0, [&](auto full) {
                short_conv_kernel<decltype(t), w.value, full.value><<<dim3((unsigned)(tiles * a.rows.n_items)), dim3(kThreads), 0, s>>>(a, tiles);
                return hipGetLastError();
            });
        });
    });
}

hipError_t launch_short_conv_backward(hipStream_t s, const ShortConvArgs& a, int n_cu) {
    const int tiles = short_conv_tiles(a.cfg, true), runs = short_conv_partials(a.cfg, a.rows.n_items, n_cu);
    hipError_t e = with_type(a.cfg.dtype, [&](auto t) {
        return with_taps(a.cfg.taps, [&](auto w) {
            return with_full(a.cfg.dim % kBackVec == 0, [&](auto full) {
                short_conv_backward_kernel<decltype(t), w.value, full.value><<<dim3((unsigned)(tiles * runs)), dim3(kThreads), 0, s>>>(a, tiles, runs);
                return hipGetLastError();
            });
        });
    });
    const int64_t w = (int64_t)a.cfg.dim * a.cfg.taps;
    if (e == hipSuccess && a.partial) e = launch_sum_partials(s, a.partial, runs, w + a.cfg.dim, {{{a.dweight, w}, {a.dbias, a.cfg.dim}, {}}});
    return e;
}

hipError_t launch_short_conv_step(hipStream_t s, int n_seq, const ShortConvArgs& a) {
    const int across = lanes_across(a.cfg.dim, kVec), tiles = short_conv_tiles(a.cfg, false), streams = 64 / across;
    return with_type(a.cfg.dtype, [&](auto t) {
        return with_taps(a.cfg.taps, [&](auto w) {
            short_conv_step_kernel<decltype(t), w.value><<<dim3((unsigned)(tiles * ((n_seq + streams - 1) / streams))), dim3(64), 0, s>>>(a, n_seq, across, tiles);
            return hipGetLastError();
        });
    });
}

}  // namespace aug
