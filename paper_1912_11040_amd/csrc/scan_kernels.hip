// Selective scan of a diagonal state space: rows of packed sequences, its gradients, and single rows of streams.

#include <type_traits>

#include "rows_device.h"

namespace aug {
namespace {

constexpr int kChannels = 64;            // (of the gradients' and the streams' groups)

__device__ inline float step_of(const aug_scan_cfg& cfg, float v) { return cfg.softplus ? softplus(v) : v; }
// The rate for powers of two.  (The lowest finite numbers stay finite: a step of zero keeps their state.)
__device__ inline float rate2(float a) {
    const float r = a * kLog2e;
    return r < -3.4e38f && a > -INFINITY ? -3.4e38f : r;
}

// ---- rows of sequences ----
//
// A group of four wavefronts takes 256 / LN channels through a block of rows; LN neighbouring lanes share a channel, K states each
// in registers, and add up their part of the output.  Rows come in tiles of TT: all lanes turn EPT elements each of u and delta
// into steps and step u in LDS, walk the tile, and the same lanes finish their EPT outputs with the skip and the gate.
template <int LN, int K> struct Tile {
    static constexpr int CW = 256 / LN, TT = LN <= 4 ? 8 * LN : 32, EPT = TT * CW / 256, NP = LN * K, YP = CW + 16;
    static constexpr int BC = (TT * NP + 255) / 256;     // elements of b (and of c) that a lane fetches per tile
};

enum ScanMode { kWhole, kSums, kResume };                // the block is a sequence; its end state from zero and its steps' sum; from its first state

template <class T, int LN, int K, int MODE>
__global__ __launch_bounds__(256) void scan_kernel(ScanArgs a, float* first_state, float* step_sum) {
    using G = Tile<LN, K>;
    __shared__ float2 su[G::TT][G::CW];                  // (step, step u)
    __shared__ float sb[G::TT][G::NP], sc[MODE == kSums ? 1 : G::TT][G::NP];
    __shared__ float sy[MODE == kSums ? 1 : G::TT][G::YP];
    const int tid = threadIdx.x, dim = a.cfg.dim, n_state = a.cfg.n_state, per_group = dim / a.cfg.n_group;
    const int tiles = (per_group + G::CW - 1) / G::CW, group = blockIdx.x / tiles, in_group = (blockIdx.x % tiles) * G::CW;
    const int d0 = group * per_group + in_group, width = min(G::CW, per_group - in_group);
    const int2 item = a.rows.items[blockIdx.y];
    const int64_t seq = item.x, begin = a.rows.begin[seq] + ((int64_t)item.y << a.rows.lg), end = a.rows.end[seq];
    const bool last = a.rows.lg == 30 || blockIdx.y + 1 == gridDim.y || a.rows.items[blockIdx.y + 1].y == 0;
    if (MODE == kSums && last) return;                   // nobody asks for a sequence's last sums
    const int rows = (int)min(end - begin, (int64_t)1 << a.rows.lg);

    // as a walker: channel and states
    const int ch = tid / LN, nq = (tid % LN) * K;
    const bool walks = ch < width;
    const int64_t at = walks ? ((MODE == kWhole ? seq : (int64_t)blockIdx.y) * dim + d0 + ch) * n_state : 0;
    float h[K], rate[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const bool there = walks && nq + k < n_state;
        rate[k] = there ? rate2(a.in.a[(int64_t)(d0 + ch) * n_state + nq + k]) : 0.f;
        h[k] = 0.f;
        if (MODE == kWhole && there && a.state_in) h[k] = a.state_in[at + nq + k];
        if (MODE == kResume && there) h[k] = first_state[at + nq + k];
    }
    // as a loader: EPT channels of a row
    const int lt = tid / (G::CW / G::EPT), lc = tid % (G::CW / G::EPT) * G::EPT, valid = width - lc;
    float bias[G::EPT], skip[G::EPT];
#pragma unroll
    for (int i = 0; i < G::EPT; ++i) {
        bias[i] = a.in.delta_bias && i < valid ? a.in.delta_bias[d0 + lc + i] : 0.f;
        skip[i] = MODE != kSums && a.in.skip && i < valid ? a.in.skip[d0 + lc + i] : 0.f;
    }
    const bool gate = MODE != kSums && a.in.z.data;
    Pack<T, G::EPT> u, delta, z;
    T vb[G::BC], vc[G::BC];
    auto fetch = [&](int t0) {
        const int64_t r = begin + t0 + lt;
        const int v = t0 + lt < rows ? valid : 0;
        u = load_pack<T, G::EPT>(row_in<T>(a.in.u, r) + d0 + lc, v);
        delta = load_pack<T, G::EPT>(row_in<T>(a.in.delta, r) + d0 + lc, v);
        if (gate) z = load_pack<T, G::EPT>(row_in<T>(a.in.z, r) + d0 + lc, v);
#pragma unroll
        for (int j = 0; j < G::BC; ++j) {
            const int e = tid + 256 * j, t = t0 + e / G::NP, n = e % G::NP;
            const bool there = e < G::TT * G::NP && t < rows && n < n_state;
            const int64_t col = (int64_t)group * n_state + n;
            vb[j] = there ? row_in<T>(a.in.b, begin + t)[col] : (T)0;
            if (MODE != kSums) vc[j] = there ? row_in<T>(a.in.c, begin + t)[col] : (T)0;
        }
    };
    float sum = 0.f;
    if (rows > 0) fetch(0);
    for (int t0 = 0; t0 < rows; t0 += G::TT) {
        const int here = min(G::TT, rows - t0);
        float us[G::EPT];
#pragma unroll
        for (int i = 0; i < G::EPT; ++i) {
            us[i] = (float)u.v[i];
            const float step = step_of(a.cfg, (float)delta.v[i] + bias[i]);
            if (lt < here) su[lt][lc + i] = make_float2(step, step * us[i]);
        }
        const Pack<T, G::EPT> zs = z;
#pragma unroll
        for (int j = 0; j < G::BC; ++j) {
            const int e = tid + 256 * j;
            if (G::TT * G::NP % 256 == 0 || e < G::TT * G::NP) {
                (&sb[0][0])[e] = (float)vb[j];
                if (MODE != kSums) (&sc[0][0])[e] = (float)vc[j];
            }
        }
        __syncthreads();
        if (t0 + G::TT < rows) fetch(t0 + G::TT);
        auto walk = [&](int t) {                         // one row; the lane's part of the output
            const float2 s = su[t][ch];
            float p = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                h[k] = fmaf(__builtin_amdgcn_exp2f(s.x * rate[k]), h[k], s.y * sb[t][nq + k]);
                if (MODE != kSums) p = fmaf(sc[t][nq + k], h[k], p);
            }
            if (MODE == kSums) sum += s.x;
            return p;
        };
        constexpr int kTogether = LN < 4 ? 4 : LN;
        int t = 0;
        for (; t + kTogether <= here; t += kTogether) {
            float y = 0.f;
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const float p = walk(t + j);
                if (MODE == kSums) continue;
                const float all = lanes_sum<LN>(p);      // lane q of a channel keeps row q of LN
                y = j % LN == 0 || j % LN == tid % LN ? all : y;
                if (j % LN == LN - 1) sy[t + j - (LN - 1) + tid % LN][ch] = y;
            }
        }
        for (; t < here; ++t) {
            const float p = walk(t);
            if (MODE == kSums) continue;
            const float all = lanes_sum<LN>(p);
            if (tid % LN == 0) sy[t][ch] = all;
        }
        __syncthreads();
        if (MODE != kSums && lt < here) {
            Pack<T, G::EPT> out;
#pragma unroll
            for (int i = 0; i < G::EPT; ++i) {
                float p = fmaf(skip[i], us[i], sy[lt][lc + i]);
                if (gate) {
                    const float g = (float)zs.v[i];
                    p *= g * sigmoid(g);
                }
                out.v[i] = (T)p;
            }
            store_pack<T, G::EPT>(row_out<T>(a.y, begin + t0 + lt) + d0 + lc, out, valid);
        }
    }
    if (!walks) return;
    if (MODE == kSums) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (nq + k < n_state) first_state[at + nq + k] = h[k];
        if (tid % LN == 0) step_sum[(int64_t)blockIdx.y * dim + d0 + ch] = sum;
    } else if (a.state_out && last) {
        float* const out = a.state_out + (seq * dim + d0 + ch) * n_state;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (nq + k < n_state) out[nq + k] = h[k];
    }
}

// Turns each block's end state from zero (first_state as kSums leaves it) into its first state: a thread per (sequence, state) goes
// through the sequence's blocks, h' = F + exp(a sum of steps) h, with eight blocks' loads on their way at once.
__global__ __launch_bounds__(64) void scan_join_kernel(ScanArgs a, float* first_state, const float* step_sum) {
    const int64_t width = (int64_t)a.cfg.dim * a.cfg.n_state, i = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (i >= width) return;
    const int seq = blockIdx.y, from = a.rows.first[seq], to = a.rows.first[seq + 1];
    const int64_t d = i / a.cfg.n_state;
    const float rate = rate2(a.in.a[i]);
    float h = a.state_in ? a.state_in[seq * width + i] : 0.f;
    constexpr int kAhead = 8;
    for (int at = from; at < to; at += kAhead) {
        float f[kAhead], s[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const bool there = at + j < to - 1;          // the last block's end is not asked for
            f[j] = there ? first_state[(at + j) * width + i] : 0.f;
            s[j] = there ? step_sum[(int64_t)(at + j) * a.cfg.dim + d] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (at + j < to) first_state[(at + j) * width + i] = h;
            // (a state of zero stays out of it, also where a rate above zero makes the factor infinite)
            h = h == 0.f ? f[j] : fmaf(__builtin_amdgcn_exp2f(s[j] * rate), h, f[j]);
        }
    }
}

// ---- rows of streams ----
// The same lanes per channel; a group takes 256 / LN channels, whose rates stay in registers, through `streams` rows.
template <class T, int LN, int K>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanArgs a, int n_seq, int streams) {
    using G = Tile<LN, K>;
    const int tid = threadIdx.x, dim = a.cfg.dim, n_state = a.cfg.n_state, per_group = dim / a.cfg.n_group;
    const int tiles = (per_group + G::CW - 1) / G::CW, group = blockIdx.x / tiles;
    const int in_group = (blockIdx.x % tiles) * G::CW + tid / LN, nq = (tid % LN) * K, states = n_state - nq;
    if (in_group >= per_group) return;                   // (all lanes of a channel together)
    const int d = group * per_group + in_group;
    const Pack<float, K> rates = load_pack<float, K>(a.in.a + (int64_t)d * n_state + nq, states);
    float rate[K];
#pragma unroll
    for (int k = 0; k < K; ++k) rate[k] = rate2(rates.v[k]);
    const float bias = a.in.delta_bias ? a.in.delta_bias[d] : 0.f, skip = a.in.skip ? a.in.skip[d] : 0.f;
    const int from = blockIdx.y * streams, to = min(from + streams, n_seq);
    const int64_t col = (int64_t)group * n_state + nq;
#pragma unroll 4
    for (int r = from; r < to; ++r) {
        const int64_t at = ((int64_t)r * dim + d) * n_state + nq;
        Pack<float, K> h = load_pack<float, K>(a.state_in + at, states);
        const Pack<T, K> b = load_pack<T, K>(row_in<T>(a.in.b, r) + col, states), c = load_pack<T, K>(row_in<T>(a.in.c, r) + col, states);
        const float u = (float)row_in<T>(a.in.u, r)[d], step = step_of(a.cfg, (float)row_in<T>(a.in.delta, r)[d] + bias), su = step * u;
        float p = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            h.v[k] = fmaf(__builtin_amdgcn_exp2f(step * rate[k]), h.v[k], su * (float)b.v[k]);
            if (k < states) p = fmaf((float)c.v[k], h.v[k], p);
        }
        p = fmaf(skip, u, lanes_sum<LN>(p));
        store_pack<float, K>(a.state_out + at, h, states);
        if (a.in.z.data) {
            const float z = (float)row_in<T>(a.in.z, r)[d];
            p *= z * sigmoid(z);
        }
        if (tid % LN == 0) row_out<T>(a.y, r)[d] = (T)p;
    }
}

// ---- gradients ----
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

// Calls f with the lanes per channel and the states per lane for so many states, as integral constants.
template <class F> hipError_t with_lanes(int n_state, F f) {
    using std::integral_constant;
    if (n_state <= 4) return f(integral_constant<int, 1>(), integral_constant<int, 4>());
    if (n_state <= 8) return f(integral_constant<int, 2>(), integral_constant<int, 4>());
    if (n_state <= 16) return f(integral_constant<int, 4>(), integral_constant<int, 4>());
    if (n_state <= 32) return f(integral_constant<int, 4>(), integral_constant<int, 8>());
    if (n_state <= 64) return f(integral_constant<int, 8>(), integral_constant<int, 8>());
    return f(integral_constant<int, 16>(), integral_constant<int, 8>());
}
int lanes_of(int n_state) { return n_state <= 4 ? 1 : n_state <= 8 ? 2 : n_state <= 32 ? 4 : n_state <= 64 ? 8 : 16; }
int scan_tiles(const aug_scan_cfg& cfg) {
    const int cw = 256 / lanes_of(cfg.n_state);
    return cfg.n_group * ((cfg.dim / cfg.n_group + cw - 1) / cw);
}

int scan_lg_block(const aug_scan_cfg& cfg, int n_seq, const int64_t* begin, const int64_t* lengths, int n_cu, bool backward) {
    if (backward) return 30;
    // A row of a group's channels takes some 150 cycles of each of its four SIMDs; a sequence in one piece takes no less than its
    // length of them.  In blocks the walk is done nearly twice (end states, then outputs), with a launch and the joining between.
    int64_t rows = 0, longest = 0;
    for (int i = 0; i < n_seq; ++i) {
        const int64_t len = lengths ? lengths[i] : begin[i + 1] - begin[i];
        rows += len;
        longest = longest > len ? longest : len;
    }
    const int64_t tiles = scan_tiles(cfg), filled = rows * tiles / n_cu;      // rows per compute unit
    if (longest < 256 || (longest > filled ? longest : filled) < 2 * filled + 128) return 30;
    int lg = 10;
    while (lg > 6 && (rows >> lg) * tiles < 4 * (int64_t)n_cu) --lg;
    return lg;
}
size_t scan_workspace(const aug_scan_cfg& cfg, int n_items, int64_t n_rows, int, bool backward) {
    if (!backward) return 4 * (size_t)n_items * cfg.dim * (cfg.n_state + 1);      // first states, steps' sums
    return 4 * ((size_t)n_rows * cfg.dim * cfg.n_state + (size_t)tiles_of(cfg) * n_rows * 2 * cfg.n_state + (size_t)n_items * cfg.dim * (cfg.n_state + 2));
}

hipError_t launch_scan(hipStream_t s, const ScanArgs& a, int) {
    return with_type(a.cfg.dtype, [&](auto t) {
        return with_lanes(a.cfg.n_state, [&](auto ln, auto k) {
            using T = decltype(t);
            const dim3 grid((unsigned)scan_tiles(a.cfg), (unsigned)a.rows.n_items);
            float* const first_state = static_cast<float*>(a.ws);
            float* const step_sum = first_state + (int64_t)a.rows.n_items * a.cfg.dim * a.cfg.n_state;
            if (a.rows.lg == 30) {
                scan_kernel<T, ln.value, k.value, kWhole><<<grid, dim3(256), 0, s>>>(a, nullptr, nullptr);
                return hipGetLastError();
            }
            scan_kernel<T, ln.value, k.value, kSums><<<grid, dim3(256), 0, s>>>(a, first_state, step_sum);
            hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            const int64_t width = (int64_t)a.cfg.dim * a.cfg.n_state;
            scan_join_kernel<<<dim3((unsigned)((width + 63) / 64), (unsigned)a.rows.n_seq), dim3(64), 0, s>>>(a, first_state, step_sum);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
            scan_kernel<T, ln.value, k.value, kResume><<<grid, dim3(256), 0, s>>>(a, first_state, step_sum);
            return hipGetLastError();
        });
    });
}

hipError_t launch_scan_step(hipStream_t s, int n_seq, const ScanArgs& a, int n_cu) {
    // as many streams to a group as leave eight groups to a compute unit
    const int64_t tiles = scan_tiles(a.cfg), each = n_seq * tiles / (8 * (int64_t)n_cu);
    const int streams = each < 1 ? 1 : each > 16 ? 16 : (int)each;
    return with_type(a.cfg.dtype, [&](auto t) {
        return with_lanes(a.cfg.n_state, [&](auto ln, auto k) {
            scan_step_kernel<decltype(t), ln.value, k.value>
                <<<dim3((unsigned)tiles, (unsigned)((n_seq + streams - 1) / streams)), dim3(256), 0, s>>>(a, n_seq, streams);
            return hipGetLastError();
        });
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
