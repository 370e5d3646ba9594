// Selective scan of a diagonal state space: rows of packed sequences, its gradients, and single rows of streams.

#include "rows_device.h"

namespace aug {
namespace {

constexpr int kChannels = 64;

__device__ inline float step_of(const aug_scan_cfg& cfg, float v) { return cfg.softplus ? softplus(v) : v; }

// A thread per (sequence, channel), the channel's states in LDS: [n_state][64].
template <class T>
__global__ __launch_bounds__(kChannels) void scan_kernel(ScanArgs a, bool streams) {
    extern __shared__ float h[];
    const int lane = threadIdx.x, d = blockIdx.y * kChannels + lane, n_state = a.cfg.n_state;
    const int64_t seq = blockIdx.x;
    if (d >= a.cfg.dim) return;
    const int64_t begin = streams ? seq : a.rows.begin[seq], end = streams ? seq + 1 : a.rows.end[seq];
    const int64_t at = (seq * a.cfg.dim + d) * n_state;
    const int g = d / (a.cfg.dim / a.cfg.n_group);
    const float bias = a.in.delta_bias ? a.in.delta_bias[d] : 0.f, skip = a.in.skip ? a.in.skip[d] : 0.f;
    for (int n = 0; n < n_state; ++n) h[n * kChannels + lane] = a.state_in ? a.state_in[at + n] : 0.f;
    for (int64_t r = begin; r < end; ++r) {
        const float u = (float)row_in<T>(a.in.u, r)[d], step = step_of(a.cfg, (float)row_in<T>(a.in.delta, r)[d] + bias);
        const T* b = row_in<T>(a.in.b, r) + (int64_t)g * n_state;
        const T* c = row_in<T>(a.in.c, r) + (int64_t)g * n_state;
        float p = skip * u;
        for (int n = 0; n < n_state; ++n) {
            const float v = fmaf(exp_fast(step * a.in.a[(int64_t)d * n_state + n]), h[n * kChannels + lane], step * u * (float)b[n]);
            h[n * kChannels + lane] = v;
            p = fmaf((float)c[n], v, p);
        }
        if (a.in.z.data) {
            const float z = (float)row_in<T>(a.in.z, r)[d];
            p *= z * sigmoid(z);
        }
        row_out<T>(a.y, r)[d] = (T)p;
    }
    if (a.state_out)
        for (int n = 0; n < n_state; ++n) a.state_out[at + n] = h[n * kChannels + lane];
}

// Workspace of the gradients: states behind every row [rows][dim][n_state], sums of a tile of channels for db and dc
// [tiles][rows][2 n_state], for da, dskip and ddelta_bias [n_seq][dim][n_state + 2].
struct BackWs {
    float *h, *bc, *par;
};
__host__ __device__ inline int tiles_of(const aug_scan_cfg& cfg) {
    return cfg.n_group * ((cfg.dim / cfg.n_group + kChannels - 1) / kChannels);
}
__host__ __device__ inline BackWs back_ws(const aug_scan_cfg& cfg, void* ws, int64_t n_rows) {
    BackWs w;
    w.h = static_cast<float*>(ws);
    w.bc = w.h + n_rows * cfg.dim * cfg.n_state;
    w.par = w.bc + (int64_t)tiles_of(cfg) * n_rows * 2 * cfg.n_state;
    return w;
}

// A wavefront per (sequence, tile of up to 64 channels of one group).
template <class T>
__global__ __launch_bounds__(kChannels) void scan_backward_kernel(ScanArgs a, int64_t n_rows) {
    extern __shared__ float g[];                        // decay times gradient of the row behind, then da: [2][n_state][64]
    const int lane = threadIdx.x, n_state = a.cfg.n_state, dim = a.cfg.dim, per_group = dim / a.cfg.n_group;
    const int tiles = (per_group + kChannels - 1) / kChannels, group = blockIdx.y / tiles;
    const int in_group = (blockIdx.y % tiles) * kChannels + lane;
    const bool live = in_group < per_group;
    const int d = group * per_group + (live ? in_group : 0);
    const int64_t seq = blockIdx.x, begin = a.rows.begin[seq], end = a.rows.end[seq];
    const BackWs ws = back_ws(a.cfg, a.ws, n_rows);
    const float* rate = a.in.a + (int64_t)d * n_state;
    float* const da = g + n_state * kChannels;
    const float bias = a.in.delta_bias ? a.in.delta_bias[d] : 0.f, skip = a.in.skip ? a.in.skip[d] : 0.f;
    float* const par = ws.par + (seq * dim + d) * (n_state + 2);
    for (int n = 0; n < n_state; ++n) g[n * kChannels + lane] = da[n * kChannels + lane] = 0.f;
    if (live)
        for (int64_t r = begin; r < end; ++r) {
            const float u = (float)row_in<T>(a.in.u, r)[d], step = step_of(a.cfg, (float)row_in<T>(a.in.delta, r)[d] + bias);
            const T* b = row_in<T>(a.in.b, r) + (int64_t)group * n_state;
            float* const h = ws.h + (r * dim + d) * n_state;
            const float* const before = r > begin ? h - (int64_t)dim * n_state : a.state_in ? a.state_in + (seq * dim + d) * n_state : nullptr;
            for (int n = 0; n < n_state; ++n) h[n] = fmaf(exp_fast(step * rate[n]), before ? before[n] : 0.f, step * u * (float)b[n]);
        }
    float dskip = 0.f, dbias = 0.f;
    for (int64_t r = end - 1; r >= begin; --r) {
        const float u = (float)row_in<T>(a.in.u, r)[d], raw = (float)row_in<T>(a.in.delta, r)[d] + bias, step = step_of(a.cfg, raw);
        const T* b = row_in<T>(a.in.b, r) + (int64_t)group * n_state;
        const T* c = row_in<T>(a.in.c, r) + (int64_t)group * n_state;
        const float dy = (float)row_in<T>(a.dy, r)[d], z = a.in.z.data ? (float)row_in<T>(a.in.z, r)[d] : 0.f;
        const float sz = sigmoid(z), dp = live ? (a.in.z.data ? dy * z * sz : dy) : 0.f;
        float* const h = ws.h + (r * dim + d) * n_state;
        const float* const before = r > begin ? h - (int64_t)dim * n_state : a.state_in ? a.state_in + (seq * dim + d) * n_state : nullptr;
        float p = skip * u, gb = 0.f, dstep = 0.f;
        float* const bc = ws.bc + ((int64_t)blockIdx.y * n_rows + r) * 2 * n_state;
        for (int n = 0; n < n_state; ++n) {
            const float e = exp_fast(step * rate[n]), gr = fmaf((float)c[n], dp, g[n * kChannels + lane]), eg = e * gr;
            const float eh = eg * (before ? before[n] : 0.f), hn = live ? h[n] : 0.f;
            g[n * kChannels + lane] = eg;
            p = fmaf((float)c[n], hn, p);
            gb = fmaf(gr, (float)b[n], gb);
            dstep = fmaf(eh, rate[n], dstep);
            da[n * kChannels + lane] += eh * step;
            const float db = wave_sum(live ? gr * step * u : 0.f), dc = wave_sum(live ? dp * hn : 0.f);
            if (lane == 0) bc[n] = db, bc[n_state + n] = dc;
        }
        if (!live) continue;
        dskip = fmaf(dp, u, dskip);
        dstep = fmaf(u, gb, dstep);
        const float dd = a.cfg.softplus ? dstep * sigmoid(raw) : dstep;
        dbias += dd;
        if (a.grad.du.data) row_out<T>(a.grad.du, r)[d] = (T)(step * gb + skip * dp);
        if (a.grad.ddelta.data) row_out<T>(a.grad.ddelta, r)[d] = (T)dd;
        if (a.grad.dz.data) row_out<T>(a.grad.dz, r)[d] = (T)(dy * p * sz * (1.f + z * (1.f - sz)));
    }
    if (!live) return;
    for (int n = 0; n < n_state; ++n) par[n] = da[n * kChannels + lane];
    par[n_state] = dskip;
    par[n_state + 1] = dbias;
}

// db and dc: sums over the tiles of a group.  A group per sequence, so that rows of none are left alone.
template <class T>
__global__ __launch_bounds__(256) void scan_bc_kernel(ScanArgs a, int64_t n_rows) {
    const int n_state = a.cfg.n_state, n_group = a.cfg.n_group, tiles = tiles_of(a.cfg) / n_group, width = 2 * n_state * n_group;
    const int64_t seq = blockIdx.x, begin = a.rows.begin[seq], n = (a.rows.end[seq] - begin) * width;
    const BackWs ws = back_ws(a.cfg, a.ws, n_rows);
    for (int64_t i = threadIdx.x; i < n; i += 256) {
        const int64_t r = begin + i / width;
        const int group = (int)(i % width) / (2 * n_state), k = (int)(i % width) % (2 * n_state);
        float acc = 0.f;
        for (int t = 0; t < tiles; ++t) acc += ws.bc[((int64_t)(group * tiles + t) * n_rows + r) * 2 * n_state + k];
        const aug_rows& out = k < n_state ? a.grad.db : a.grad.dc;
        if (out.data) row_out<T>(out, r)[group * n_state + k % n_state] = (T)acc;
    }
}

// Parameter gradients: sums over the sequences, a thread per (channel, value).
__global__ __launch_bounds__(64) void scan_par_kernel(ScanArgs a, int64_t n_rows) {
    const int n_state = a.cfg.n_state;
    const int64_t i = (int64_t)blockIdx.x * 64 + threadIdx.x, width = (int64_t)a.cfg.dim * (n_state + 2);
    if (i >= width) return;
    const float* par = back_ws(a.cfg, a.ws, n_rows).par + i;
    float acc = 0.f;
    for (int q = 0; q < a.rows.n_seq; ++q) acc += par[q * width];
    const int64_t d = i / (n_state + 2);
    const int k = (int)(i % (n_state + 2));
    if (k < n_state) {
        if (a.grad.da) a.grad.da[d * n_state + k] = acc;
    } else if (k == n_state) {
        if (a.grad.dskip) a.grad.dskip[d] = acc;
    } else if (a.grad.ddelta_bias) {
        a.grad.ddelta_bias[d] = acc;
    }
}

}  // namespace

int scan_lg_block(const aug_scan_cfg&, int, const int64_t*, const int64_t*, int, bool) { return 30; }
size_t scan_workspace(const aug_scan_cfg& cfg, int n_items, int64_t n_rows, int, bool backward) {
    if (!backward) return 0;
    return 4 * ((size_t)n_rows * cfg.dim * cfg.n_state + (size_t)tiles_of(cfg) * n_rows * 2 * cfg.n_state + (size_t)n_items * cfg.dim * (cfg.n_state + 2));
}

hipError_t launch_scan(hipStream_t s, const ScanArgs& a, int) {
    return with_type(a.cfg.dtype, [&](auto t) {
        scan_kernel<decltype(t)><<<dim3((unsigned)a.rows.n_seq, (unsigned)((a.cfg.dim + kChannels - 1) / kChannels)), dim3(kChannels),
                                   4 * kChannels * a.cfg.n_state, s>>>(a, false);
        return hipGetLastError();
    });
}

hipError_t launch_scan_step(hipStream_t s, int n_seq, const ScanArgs& a) {
    return with_type(a.cfg.dtype, [&](auto t) {
        scan_kernel<decltype(t)><<<dim3((unsigned)n_seq, (unsigned)((a.cfg.dim + kChannels - 1) / kChannels)), dim3(kChannels),
                                   4 * kChannels * a.cfg.n_state, s>>>(a, true);
        return hipGetLastError();
    });
}

hipError_t launch_scan_backward(hipStream_t s, const ScanArgs& a, int64_t n_rows, int) {
    return with_type(a.cfg.dtype, [&](auto t) {
        using T = decltype(t);
        scan_backward_kernel<T><<<dim3((unsigned)a.rows.n_seq, (unsigned)tiles_of(a.cfg)), dim3(kChannels), 8 * kChannels * a.cfg.n_state, s>>>(a, n_rows);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess && (a.grad.db.data || a.grad.dc.data)) {
            scan_bc_kernel<T><<<dim3((unsigned)a.rows.n_seq), dim3(256), 0, s>>>(a, n_rows);
            e = hipGetLastError();
        }
        const int64_t width = (int64_t)a.cfg.dim * (a.cfg.n_state + 2);
        if (e == hipSuccess && (a.grad.da || a.grad.dskip || a.grad.ddelta_bias)) {
            scan_par_kernel<<<dim3((unsigned)((width + 63) / 64)), dim3(64), 0, s>>>(a, n_rows);
            e = hipGetLastError();
        }
        return e;
    });
}

}  // namespace aug
