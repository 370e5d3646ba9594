// Selective scan of a diagonal state space: rows of packed sequences, its gradients, and single rows of streams.

#include <type_traits>

#include "rows_device.h"

namespace aug {
namespace {

__device__ inline float step_of(const aug_scan_cfg& cfg, float v) { return cfg.softplus ? softplus(v) : v; }
// Steps of N elements.  (The choice is the call's: made once, not per element, the elements' exponentials overlap.)
template <int N> __device__ inline void steps_of(const aug_scan_cfg& cfg, const float (&raw)[N], float (&step)[N]) {
    if (cfg.softplus) {
#pragma unroll
        for (int i = 0; i < N; ++i) step[i] = softplus(raw[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) step[i] = raw[i];
    }
}
// The rate for powers of two, finite also for the lowest numbers: a step of zero keeps the state.
__device__ inline float rate2(float a) {
    const float r = a * kLog2e;
    return r < -3.4e38f ? -3.4e38f : r;
}

// ---- rows of sequences ----
//
//   h = exp(step a) h + step u b,   y = (sum c h + skip u) z sigmoid(z)
// A state's row is a product, an exponential (of the time of two), a product and two multiply-adds: at sixteen states 96 slots a
// (row, channel) against 8 bytes of 16-bit rows, so vector issue bounds it (64 utterances of 98 to 1598 rows, 1024 channels, bf16: 235 us, with vector
// instructions under way all the time that its compute units are busy; these five alone take 159 at the rates that they reach by
// themselves, the bytes 97 at the rate of a copy).
// A group of four wavefronts takes 256 / LN channels through a block of rows; LN neighbouring lanes share a channel, K states each
// in registers, and add up their part of the output.  (A lane per channel would need no sums and a quarter of the groups; the chip is
// hard to fill as it is.)  Rows come in tiles of TT: all lanes turn EPT elements each of u and delta into steps and step u in LDS, once
// a (row, channel) whatever LN, walk the tile, and the same lanes finish their EPT outputs with the skip and the gate.
template <int LN, int K> struct Tile {
    static constexpr int CW = 256 / LN, TT = LN <= 4 ? 8 * LN : 32, EPT = TT * CW / 256, NP = LN * K, YP = CW + 16;
    static constexpr int BC = (TT * NP + 255) / 256;     // elements of b (and of c) that a lane fetches per tile
};

// SPARE: some lanes have states that the channel does not have (n_state is less than LN K).  Their b and c are zero, and they are put
// to zero after every row: a step, an input or a gradient that is infinite or NaN would make NaN of them, and of the sums that they are in.

enum ScanMode { kWhole, kSums, kResume };                // the block is a sequence; its end state from zero and its steps' sum; from its first state

template <class T, int LN, int K, int MODE, bool FULL, bool SPARE>
__global__ __launch_bounds__(256) void scan_kernel(ScanArgs a, int all_tiles, float* first_state, float* step_sum) {
    using G = Tile<LN, K>;
    __shared__ float2 su[G::TT][G::CW];                  // (step, step u)
    __shared__ float sb[G::TT][G::NP], sc[MODE == kSums ? 1 : G::TT][G::NP];
    __shared__ float sy[MODE == kSums ? 1 : G::TT][G::YP];
    const int tid = threadIdx.x, dim = a.cfg.dim, n_state = a.cfg.n_state, per_group = dim / a.cfg.n_group;
    const int tile = blockIdx.x % all_tiles, block = blockIdx.x / all_tiles;
    const int tiles = (per_group + G::CW - 1) / G::CW, group = tile / tiles, in_group = (tile % tiles) * G::CW;
    const int d0 = group * per_group + in_group, width = FULL ? G::CW : min(G::CW, per_group - in_group);
    const int2 item = a.rows.items[block];
    const int64_t seq = item.x, begin = a.rows.begin[seq] + ((int64_t)item.y << a.rows.lg), end = a.rows.end[seq];
    const bool last = a.rows.lg == kWholeLg || block + 1 == a.rows.n_items || a.rows.items[block + 1].y == 0;
    if (MODE == kSums && last) return;                   // nobody asks for a sequence's last sums
    const int rows = (int)min(end - begin, (int64_t)1 << a.rows.lg);

    // as a walker: channel and states
    const int ch = tid / LN, nq = (tid % LN) * K;
    const bool walks = ch < width;
    const int64_t at = walks ? ((MODE == kWhole ? seq : (int64_t)block) * dim + d0 + ch) * n_state : 0;
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
        const int64_t r = begin + min(t0 + lt, rows - 1);                  // (rows behind the block are not walked)
        u = load_part<T, G::EPT, FULL>(a.in.u, r, d0 + lc, valid);
        delta = load_part<T, G::EPT, FULL>(a.in.delta, r, d0 + lc, valid);
        if (gate) z = load_part<T, G::EPT, FULL>(a.in.z, r, d0 + lc, valid);
#pragma unroll
        for (int j = 0; j < G::BC; ++j) {
            const int e = tid + 256 * j, t = t0 + e / G::NP, n = e % G::NP;
            const bool there = e < G::TT * G::NP && n < n_state;
            const int64_t col = (int64_t)group * n_state + min(n, n_state - 1), at = begin + min(t, rows - 1);
            const T b = row_in<T>(a.in.b, at)[col], c = MODE != kSums ? row_in<T>(a.in.c, at)[col] : (T)0;
            vb[j] = there ? b : (T)0;
            vc[j] = there ? c : (T)0;
        }
    };
    float sum = 0.f;
    if (rows > 0) fetch(0);
    for (int t0 = 0; t0 < rows; t0 += G::TT) {
        const int here = min(G::TT, rows - t0);
        float us[G::EPT], raw[G::EPT], step[G::EPT];
#pragma unroll
        for (int i = 0; i < G::EPT; ++i) raw[i] = (float)delta.v[i] + bias[i];
        steps_of(a.cfg, raw, step);
#pragma unroll
        for (int i = 0; i < G::EPT; ++i) {
            us[i] = (float)u.v[i];
            su[lt][lc + i] = make_float2(step[i], step[i] * us[i]);      // (rows behind the block are not walked)
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
                if (SPARE && nq + k >= n_state) h[k] = 0.f;
                if (MODE != kSums) p = fmaf(sc[t][nq + k], h[k], p);
            }
            if (MODE == kSums) sum += s.x;
            return p;
        };
        constexpr int kTogether = LN < 4 ? 4 : LN;
        int t = 0;
        for (; t + kTogether <= here; t += kTogether) {
            float y = 0.f, p[kTogether];
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                p[j] = walk(t + j);
                if (MODE == kSums || LN == 4) continue;
                const float all = lanes_sum<LN>(p[j]);   // lane q of a channel keeps row q of LN
                y = j % LN == 0 || j % LN == tid % LN ? all : y;
                if (j % LN == LN - 1) sy[t + j - (LN - 1) + tid % LN][ch] = y;
            }
            if constexpr (MODE != kSums && LN == 4) sy[t + tid % LN][ch] = quad_sums(p);
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
            float p[G::EPT];
#pragma unroll
            for (int i = 0; i < G::EPT; ++i) p[i] = fmaf(skip[i], us[i], sy[lt][lc + i]);
            if (gate) {
#pragma unroll
                for (int i = 0; i < G::EPT; ++i) p[i] *= (float)zs.v[i] * sigmoid((float)zs.v[i]);
            }
#pragma unroll
            for (int i = 0; i < G::EPT; ++i) out.v[i] = (T)p[i];
            store_part<T, G::EPT, FULL>(a.y, begin + t0 + lt, d0 + lc, out, valid);
        }
    }
    if (!walks) return;
    if (MODE == kSums) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (nq + k < n_state) first_state[at + nq + k] = h[k];
        if (tid % LN == 0) step_sum[(int64_t)block * dim + d0 + ch] = sum;
    } else if (a.state_out && last) {
        float* const out = a.state_out + (seq * dim + d0 + ch) * n_state;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (nq + k < n_state) out[nq + k] = h[k];
    }
}

// Through the blocks of a sequence: values[j] becomes what comes into block j, h_0 = h, h_{j+1} = values[j] + exp(rate sum of j's steps) h_j,
// for one of `width` states.  GROUPS groups of lanes take eight blocks each at a time, whose loads are on their way together: with
// eight groups 64 blocks a round, where the states alone do not fill the chip (384 channels of 282 blocks: 10 us, with one group 35);
// with one nothing is exchanged (32 sequences of 27 blocks, 16384 states, both ways: 50 us, the memory's rate; with eight 67).  Block j
// lies at from + j dir; from block `known` on nothing is known or asked for.  All threads call it; states beyond the width are only
// there for the barriers.
constexpr int kJoinAhead = 8;
template <int GROUPS> constexpr int kJoinStates = GROUPS == 1 ? 64 : 32;
template <int GROUPS> struct JoinShared {
    float value[GROUPS][kJoinStates<GROUPS>], steps[GROUPS][kJoinStates<GROUPS>];
};
bool join_in_groups(int64_t width, int n_seq, int n_items, int n_cu) {
    return n_items / n_seq > 16 && width * n_seq < 64 * 8 * (int64_t)n_cu;       // fewer than eight wavefronts to a compute unit
}
// A state of `h` through a block.  A rate above zero, or steps below it, may make the factor infinite: a state of zero stays out of it, and a
// small one takes it by its root twice, which is infinite only where the state behind it is too unless the state is below 2^-128.
// RARE: by a branch around the root (a batch's join, bound by memory; with the root always the gradients of 32 utterances take 690 us instead of 667);
// else always (eight groups, whose chain is latency: a long recording 80 us, with the branch 85).
template <bool RARE> __device__ inline float pass_block(float h, float value, float steps, float rate) {
    const float factor = RARE ? __builtin_amdgcn_exp2f(steps * rate) : __builtin_amdgcn_exp2f(0.5f * steps * rate);
    if (h == 0.f) return value;
    if (!RARE) return fmaf(factor * h, factor, value);
    if (__builtin_expect(factor > 3.4e38f, 0)) {
        const float root = __builtin_amdgcn_exp2f(0.5f * steps * rate);
        return fmaf(root * h, root, value);
    }
    return fmaf(factor, h, value);
}
template <int GROUPS>
__device__ inline void join_blocks(JoinShared<GROUPS>& sh, float* values, const float* steps, int64_t width, int64_t i, int dim, int64_t d, float rate, float h,
                                   int from, int dir, int n, int known) {
    const int lane = threadIdx.x % kJoinStates<GROUPS>, group = threadIdx.x / kJoinStates<GROUPS>;
    for (int base = 0; base < n; base += GROUPS * kJoinAhead) {
        const int j0 = base + group * kJoinAhead;
        float f[kJoinAhead], s[kJoinAhead];
#pragma unroll
        for (int q = 0; q < kJoinAhead; ++q) {
            const bool there = i < width && j0 + q < known;
            const int64_t at = from + (int64_t)(j0 + q) * dir;
            f[q] = there ? values[at * width + i] : 0.f;
            s[q] = there ? steps[at * dim + d] : 0.f;
        }
        float in = h;
        if constexpr (GROUPS > 1) {
            float value = 0.f, sum = 0.f;
#pragma unroll
            for (int q = 0; q < kJoinAhead; ++q) {
                value = pass_block<false>(value, f[q], s[q], rate);
                sum += s[q];
            }
            sh.value[group][lane] = value;
            sh.steps[group][lane] = sum;
            __syncthreads();
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                if (g == group) in = h;
                h = pass_block<false>(h, sh.value[g][lane], sh.steps[g][lane], rate);
            }
        }
#pragma unroll
        for (int q = 0; q < kJoinAhead; ++q) {
            if (i < width && j0 + q < n) values[(from + (int64_t)(j0 + q) * dir) * width + i] = in;
            in = pass_block<GROUPS == 1>(in, f[q], s[q], rate);
        }
        if constexpr (GROUPS > 1) {
            __syncthreads();
        } else {
            h = in;
        }
    }
}

// Turns each block's end state from zero (first_state as kSums leaves it; the last block's is not known) into its first state.
template <int GROUPS> __global__ __launch_bounds__(kJoinStates<GROUPS> * GROUPS) void scan_join_kernel(ScanArgs a, float* first_state, const float* step_sum) {
    __shared__ JoinShared<GROUPS> sh;
    const int64_t width = (int64_t)a.cfg.dim * a.cfg.n_state, i = (int64_t)blockIdx.x * kJoinStates<GROUPS> + threadIdx.x % kJoinStates<GROUPS>;
    const int seq = blockIdx.y, from = a.rows.first[seq], n = a.rows.first[seq + 1] - from;
    const int64_t d = i / a.cfg.n_state;
    const float rate = i < width ? rate2(a.in.a[i]) : 0.f, h = a.state_in && i < width ? a.state_in[seq * width + i] : 0.f;
    join_blocks(sh, first_state, step_sum, width, i, a.cfg.dim, d, rate, h, from, 1, n, n - 1);
}

// ---- rows of streams ----
// Bound by memory: 8 n_state bytes of states a (stream, channel) and little else.  The same lanes per channel, so that states are read and
// written 16 bytes a lane side by side; a group takes 256 / LN channels, whose rates stay in registers, through `streams` rows (2048 streams
// of 2048 channels, 16 states: 134 us, 4.3 TB/s, where a large copy reaches 4.7; a thread per channel took 751).
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
//
// Sequences are cut into blocks of 1 << lg rows.  A first pass over each block forms, in one walk over its decays,
//   F, the end state from zero,  S, the sum of the steps,  R = sum_t (e_first .. e_t) c_t dp_t,
// the block's share of e_first g_first, which is what it hands to the rows before it.  scan_back_join_kernel then makes of F the state
// before each block and of R what comes in from behind.  With both the blocks are independent of one another: the main pass
// walks a block forward for its states and back for its gradients, in stretches of SUB rows whose states and decays stay in registers.
// Both are bound by vector issue: 32 utterances of 98 to 1598 rows, 1024 channels, 16 states, bf16 take 155 us (vector instructions under way 93 % of
// the time) and 440 (87 %), the join between them 51 (HBM), the sums over tiles and runs 19, 665 in all.  In blocks of 32 rows the sums are 8 of the 30 bytes moved a (row, channel); stretches of 16
// rows need more registers than two wavefronts per SIMD leave (1250 us with one).  So do, by 15 to 21 registers, which the compiler keeps in
// scratch, stretches of eight rows at four states a lane where a partial tile's accesses or 32-bit elements come on top; 16-bit ones of
// whole tiles do without.
template <int LN, int K> struct BackTile {
    static constexpr int CW = 256 / LN, NP = LN * K, LG = NP <= 64 ? 5 : 4, RT = 1 << LG, EPT = RT * CW / 256, SUB = K <= 2 ? 16 : 8;
    static constexpr int BC = (RT * NP + 255) / 256;
};

// Workspace: first states and what comes in from behind [items][dim][n_state], steps' sums [items][dim]; sums over a tile of channels for
// db and dc [tiles][n_rows][2 n_state]; sums over a run of blocks for da, dskip and ddelta_bias [runs][dim][n_state + 2].
struct BackWs {
    float *first, *behind, *steps, *bc, *par;
};
struct BackPlan {
    int tiles, runs;                     // channel tiles (all groups'); runs of blocks, a group's work in the main pass
};
__host__ __device__ inline BackWs back_ws(const aug_scan_cfg& cfg, void* ws, int n_items, int64_t n_rows, int tiles) {
    BackWs w;
    const int64_t states = (int64_t)n_items * cfg.dim * cfg.n_state;
    w.first = static_cast<float*>(ws);
    w.behind = w.first + states;
    w.steps = w.behind + states;
    w.bc = w.steps + (int64_t)n_items * cfg.dim;
    w.par = w.bc + (int64_t)tiles * n_rows * 2 * cfg.n_state;
    return w;
}

// Halves an array of N values by bit 5 or 4 of the lane: lanes without it keep the first half's sums over the two, lanes with
// it the second's.
template <int BIT, int N, int V> __device__ inline void halve(float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const unsigned x = __float_as_uint(v[i]), y = __float_as_uint(v[i + N / 2]);
        const auto r = BIT == 5 ? __builtin_amdgcn_permlane32_swap(x, y, false, false) : __builtin_amdgcn_permlane16_swap(x, y, false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
}

// Sums of 2 EPT values over the lanes of a wavefront that are APART apart (they hold the same channels of other rows).  The sums are
// dealt to these lanes: lane l keeps kept<EPT>() of them, from value kept_from<EPT>(l) on.
template <int EPT> __host__ __device__ constexpr int kept() { return EPT >= 2 ? EPT / 2 : 1; }
template <int EPT> __device__ inline int kept_from(int lane) { return EPT >= 2 ? ((lane >> 5) * 2 + (lane >> 4 & 1)) * (EPT / 2) : lane >> 5; }
template <int APART, int EPT> __device__ inline void sum_rows(float (&v)[2 * EPT]) {
    static_assert((APART == 8 && EPT >= 2) || (APART == 16 && EPT == 1), "the tiles' layouts");
    halve<5, 2 * EPT>(v);
    if constexpr (EPT >= 2) {
        halve<4, EPT>(v);
#pragma unroll
        for (int i = 0; i < EPT / 2; ++i) v[i] = dpp_add<0x128>(v[i]);
    } else {
        const unsigned x = __float_as_uint(v[0]);
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        v[0] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
}

template <class T, int LN, int K, bool FULL>
__global__ __launch_bounds__(256) void scan_back_sums_kernel(ScanArgs a, BackWs ws, int all_tiles) {
    using G = BackTile<LN, K>;
    __shared__ float2 su[G::RT][G::CW];
    __shared__ float sdp[G::RT][G::CW];
    __shared__ float sb[G::RT][G::NP], sc[G::RT][G::NP];
    const int tid = threadIdx.x, dim = a.cfg.dim, n_state = a.cfg.n_state, per_group = dim / a.cfg.n_group;
    const int tile = blockIdx.x % all_tiles, block = blockIdx.x / all_tiles;
    const int tiles = (per_group + G::CW - 1) / G::CW, group = tile / tiles, in_group = (tile % tiles) * G::CW;
    const int d0 = group * per_group + in_group, width = FULL ? G::CW : min(G::CW, per_group - in_group);
    const int2 item = a.rows.items[block];
    const int64_t begin = a.rows.begin[item.x] + ((int64_t)item.y << G::LG), end = a.rows.end[item.x];
    const int here = (int)min(end - begin, (int64_t)G::RT);
    if (here <= 0) return;
    const int lt = tid / (G::CW / G::EPT), lc = tid % (G::CW / G::EPT) * G::EPT, valid = width - lc;
    const int64_t r = begin + min(lt, here - 1);         // (rows behind the block are not walked)
    const auto u = load_part<T, G::EPT, FULL>(a.in.u, r, d0 + lc, valid), delta = load_part<T, G::EPT, FULL>(a.in.delta, r, d0 + lc, valid);
    const auto dy = load_part<T, G::EPT, FULL>(a.dy, r, d0 + lc, valid);
    Pack<T, G::EPT> z;
    if (a.in.z.data) z = load_part<T, G::EPT, FULL>(a.in.z, r, d0 + lc, valid);
#pragma unroll
    for (int j = 0; j < G::BC; ++j) {
        const int e = tid + 256 * j, t = e / G::NP, n = e % G::NP;
        if (t >= G::RT) break;
        const int64_t col = (int64_t)group * n_state + min(n, n_state - 1), at = begin + min(t, here - 1);
        const float b = (float)row_in<T>(a.in.b, at)[col], c = (float)row_in<T>(a.in.c, at)[col];
        sb[t][n] = n < n_state ? b : 0.f;
        sc[t][n] = n < n_state ? c : 0.f;
    }
    float raw[G::EPT], step[G::EPT], dp[G::EPT];
#pragma unroll
    for (int i = 0; i < G::EPT; ++i) {
        raw[i] = (float)delta.v[i] + (a.in.delta_bias && i < valid ? a.in.delta_bias[d0 + lc + i] : 0.f);
        dp[i] = (float)dy.v[i];
    }
    steps_of(a.cfg, raw, step);
    if (a.in.z.data) {
#pragma unroll
        for (int i = 0; i < G::EPT; ++i) dp[i] *= (float)z.v[i] * sigmoid((float)z.v[i]);
    }
#pragma unroll
    for (int i = 0; i < G::EPT; ++i) {                   // (neither rows behind the block nor channels behind the tile are walked)
        su[lt][lc + i] = make_float2(step[i], step[i] * (float)u.v[i]);
        sdp[lt][lc + i] = dp[i];
    }
    __syncthreads();
    const int ch = tid / LN, nq = (tid % LN) * K;
    if (ch >= width) return;
    const int64_t at = ((int64_t)block * dim + d0 + ch) * n_state + nq;
    float f[K] = {}, q[K], back[K] = {}, rate[K], sum = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        rate[k] = nq + k < n_state ? rate2(a.in.a[(int64_t)(d0 + ch) * n_state + nq + k]) : 0.f;
        q[k] = 1.f;
    }
#pragma unroll 4
    for (int t = 0; t < here; ++t) {
        const float2 s = su[t][ch];
        const float dp = sdp[t][ch];
        sum += s.x;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float e = __builtin_amdgcn_exp2f(s.x * rate[k]);
            f[k] = fmaf(e, f[k], s.y * sb[t][nq + k]);
            q[k] *= e;
            back[k] = fmaf(q[k], sc[t][nq + k] * dp, back[k]);
        }
    }
    // Decays that grow, by a rate above zero or a step below it, may take the product out of the range of 32 bits where no term is: the
    // sum is then formed row by row from the last, as the definition does, and a term of zero stays zero (but for a decay of NaN).
    bool lost = false;
#pragma unroll
    for (int k = 0; k < K; ++k) lost = lost || !(q[k] <= 3.4e38f);
    if (!a.cfg.softplus) {
        float least = 0.f, most = 0.f;
        for (int t = 0; t < here; ++t) {
            least = fminf(least, su[t][ch].x);
            most = fmaxf(most, su[t][ch].x);
        }
        lost = lost || (least < 0.f && most > 0.f);      // what underflows may grow again
    }
    if (lost) {
#pragma unroll
        for (int k = 0; k < K; ++k) back[k] = 0.f;
#pragma unroll 1
        for (int t = here - 1; t >= 0; --t) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const float e = __builtin_amdgcn_exp2f(su[t][ch].x * rate[k]), g = fmaf(sc[t][nq + k], sdp[t][ch], back[k]);
                back[k] = g == 0.f && e == e ? 0.f : e * g;
            }
        }
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (nq + k < n_state) ws.first[at + k] = f[k], ws.behind[at + k] = back[k];
    if (tid % LN == 0) ws.steps[(int64_t)block * dim + d0 + ch] = sum;
}

// Forward through a sequence's blocks for their first states, back for what comes in from behind.
template <int GROUPS> __global__ __launch_bounds__(kJoinStates<GROUPS> * GROUPS) void scan_back_join_kernel(ScanArgs a, BackWs ws) {
    __shared__ JoinShared<GROUPS> sh;
    const int64_t width = (int64_t)a.cfg.dim * a.cfg.n_state, i = (int64_t)blockIdx.x * kJoinStates<GROUPS> + threadIdx.x % kJoinStates<GROUPS>;
    const int seq = blockIdx.y, from = a.rows.first[seq], n = a.rows.first[seq + 1] - from;
    if (a.rows.end[seq] == a.rows.begin[seq]) return;    // (an empty sequence's block has no sums)
    const int64_t d = i / a.cfg.n_state;
    const float rate = i < width ? rate2(a.in.a[i]) : 0.f, h = a.state_in && i < width ? a.state_in[seq * width + i] : 0.f;
    join_blocks(sh, ws.first, ws.steps, width, i, a.cfg.dim, d, rate, h, from, 1, n, n);
    join_blocks(sh, ws.behind, ws.steps, width, i, a.cfg.dim, d, rate, 0.f, from + n - 1, -1, n, n);
}

// What a walker reads of a row: its channel's step, step u and dp, its states' b or c.  Rows are read one ahead of their use: the
// scheduler would otherwise put a row's reads right before it and wait for LDS at every row.
template <int K> struct RowIn {
    float2 s;
    float dp, v[K];
    template <int R, int CW, int NP>
    __device__ inline void load(const float2 (&su)[R][CW], const float (&sdp)[R][CW], const float (&sv)[R][NP], int t, int ch, int nq) {
        s = su[t][ch];
        dp = sdp[t][ch];
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = sv[t][nq + k];
    }
};
__device__ inline void stay_ahead() { __builtin_amdgcn_sched_barrier(0x2 | 0x4 | 0x200); }      // arithmetic and LDS writes may pass, reads not

template <class T, int LN, int K, bool FULL, bool SPARE>
__global__ __launch_bounds__(256, K <= 4 ? 2 : 1) void scan_back_kernel(ScanArgs a, BackWs ws, BackPlan plan, int64_t n_rows, bool joined) {
    using G = BackTile<LN, K>;
    constexpr int NS = G::RT / G::SUB, V = 2 * K;
    __shared__ float2 su[G::RT][G::CW];                  // (step, step u); behind a row's walk (sum g b, sum of e g h a)
    __shared__ float sdp[G::RT][G::CW];                  // dp; behind a row's walk sum c h
    __shared__ float sb[G::RT][G::NP], sc[G::RT][G::NP];
    __shared__ float sbc[4][G::RT][2 * G::NP];           // each wavefront's sums over its channels for db and dc
    __shared__ float sbias[G::CW], sskip[G::CW];
    __shared__ float sst[NS][256][K];                    // each lane's states before the stretches
    const int tid = threadIdx.x, dim = a.cfg.dim, n_state = a.cfg.n_state, per_group = dim / a.cfg.n_group;
    const int tile = blockIdx.x % plan.tiles, run = blockIdx.x / plan.tiles;
    const int tiles = plan.tiles / a.cfg.n_group, group = tile / tiles, in_group = (tile % tiles) * G::CW;
    const int d0 = group * per_group + in_group, width = FULL ? G::CW : min(G::CW, per_group - in_group);
    const int first_item = (int)((int64_t)a.rows.n_items * run / plan.runs), end_item = (int)((int64_t)a.rows.n_items * (run + 1) / plan.runs);

    const int ch = tid / LN, nq = (tid % LN) * K, wave = tid / 64;
    const bool walks = ch < width;
    float rate[K], da[K] = {};
#pragma unroll
    for (int k = 0; k < K; ++k) rate[k] = walks && nq + k < n_state ? rate2(a.in.a[(int64_t)(d0 + ch) * n_state + nq + k]) : 0.f;
    const int lt = tid / (G::CW / G::EPT), lc = tid % (G::CW / G::EPT) * G::EPT;
    if (tid < G::CW) {
        sbias[tid] = a.in.delta_bias && tid < width ? a.in.delta_bias[d0 + tid] : 0.f;
        sskip[tid] = a.in.skip && tid < width ? a.in.skip[d0 + tid] : 0.f;
    }
    float acc[kept<G::EPT>()] = {};                      // dskip and ddelta_bias, as sum_rows deals them
    const bool gate = a.in.z.data;
    __syncthreads();

    // A block's rows and what a lane reads of them.  A short block's rows are the last ones of its RT: the ones in front of them have steps,
    // inputs and gradients of zero and leave the first state as it is.  (Behind them they would meet the last row's state, which
    // is in no gradient by the rates: a number or not.)  The next block's are asked for behind the walk, when the states' registers are
    // free, and where it lies a block earlier.
    struct Block {
        int seq, here, pad;
        int64_t begin;
    };
    struct Data {
        Pack<T, G::EPT> u, delta, dy, z;
        T b[G::BC], c[G::BC];
        float first[K], behind[K];
    };
    auto locate = [&](int it) -> Block {
        if (it >= end_item) return {0, 0, 0, 0};
        const int2 item = a.rows.items[it];
        const int64_t begin = a.rows.begin[item.x] + ((int64_t)item.y << G::LG);
        const int here = (int)min(a.rows.end[item.x] - begin, (int64_t)G::RT);
        return {item.x, here, G::RT - here, begin};
    };
    auto fetch = [&](const Block& blk, int it, Data& v) {
        if (blk.here <= 0) return;
        const int64_t r = blk.begin + max(lt - blk.pad, 0);
        v.u = load_part<T, G::EPT, FULL>(a.in.u, r, d0 + lc, width - lc);
        v.delta = load_part<T, G::EPT, FULL>(a.in.delta, r, d0 + lc, width - lc);
        v.dy = load_part<T, G::EPT, FULL>(a.dy, r, d0 + lc, width - lc);
        if (gate) v.z = load_part<T, G::EPT, FULL>(a.in.z, r, d0 + lc, width - lc);
#pragma unroll
        for (int j = 0; j < G::BC; ++j) {
            const int e = tid + 256 * j, t = e / G::NP, n = e % G::NP;
            const bool there = t >= blk.pad && n < n_state;      // (what lies behind the tile is not kept either)
            const int64_t col = (int64_t)group * n_state + min(n, n_state - 1), at = blk.begin + min(max(t - blk.pad, 0), blk.here - 1);
            const T b = row_in<T>(a.in.b, at)[col], c = row_in<T>(a.in.c, at)[col];
            v.b[j] = there ? b : (T)0;
            v.c[j] = there ? c : (T)0;
        }
        // the state before the block, and what comes in from behind it: e g of the row behind
        const int64_t at = ((int64_t)it * dim + d0 + ch) * n_state + nq, in = ((int64_t)blk.seq * dim + d0 + ch) * n_state + nq;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const bool there = walks && nq + k < n_state;
            v.first[k] = !there ? 0.f : joined ? ws.first[at + k] : a.state_in ? a.state_in[in + k] : 0.f;
            v.behind[k] = there && joined ? ws.behind[at + k] : 0.f;
        }
    };
    Block blk = locate(first_item), next_blk;
    Data v, next_v;
    fetch(blk, first_item, v);
    for (int it = first_item; it < end_item; ++it, blk = next_blk, v = next_v) {
        next_blk = locate(it + 1);
        const int here = blk.here;
        if (here <= 0) {                                 // (an empty sequence's block)
            fetch(next_blk, it + 1, next_v);
            continue;
        }
        const int pad = blk.pad, first_stretch = pad / G::SUB, valid = lt >= pad ? width - lc : 0;
        const int64_t begin = blk.begin, r = begin + lt - pad;
        const Pack<T, G::EPT> u = v.u, delta = v.delta, dy = v.dy, z = v.z;
#pragma unroll
        for (int j = 0; j < G::BC; ++j) {
            const int e = tid + 256 * j;
            if (G::RT * G::NP % 256 == 0 || e < G::RT * G::NP) {
                (&sb[0][0])[e] = (float)v.b[j];
                (&sc[0][0])[e] = (float)v.c[j];
            }
        }
        float carried[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            sst[first_stretch][tid][k] = v.first[k];
            carried[k] = v.behind[k];
        }
        float raw[G::EPT], step[G::EPT], dp[G::EPT];
#pragma unroll
        for (int i = 0; i < G::EPT; ++i) {
            raw[i] = (float)delta.v[i] + sbias[lc + i];
            dp[i] = (float)dy.v[i];
        }
        steps_of(a.cfg, raw, step);
        if (gate) {
#pragma unroll
            for (int i = 0; i < G::EPT; ++i) dp[i] *= (float)z.v[i] * sigmoid((float)z.v[i]);
        }
#pragma unroll
        for (int i = 0; i < G::EPT; ++i) {
            // (rows in front of the block are walked with steps and dp of zero)
            step[i] = i < valid ? step[i] : 0.f;
            su[lt][lc + i] = make_float2(step[i], i < valid ? step[i] * (float)u.v[i] : 0.f);
            sdp[lt][lc + i] = i < valid ? dp[i] : 0.f;
        }
        __syncthreads();
        // states before the later stretches
        {
            float st[K];
#pragma unroll
            for (int k = 0; k < K; ++k) st[k] = v.first[k];
#pragma unroll 1
            for (int s = first_stretch + 1; s < NS; ++s) {
#pragma unroll
                for (int j = 0; j < G::SUB; ++j) {
                    const int t = (s - 1) * G::SUB + j;
                    const float2 x = su[t][ch];
#pragma unroll
                    for (int k = 0; k < K; ++k) st[k] = fmaf(__builtin_amdgcn_exp2f(x.x * rate[k]), st[k], x.y * sb[t][nq + k]);
                }
#pragma unroll
                for (int k = 0; k < K; ++k) sst[s][tid][k] = SPARE && nq + k >= n_state ? 0.f : st[k];
            }
        }
#pragma unroll 1
        for (int s = NS - 1; s >= first_stretch; --s) {
            float h[G::SUB + 1][K], e[G::SUB][K];
#pragma unroll
            for (int k = 0; k < K; ++k) h[0][k] = sst[s][tid][k];
            RowIn<K> next;
            next.load(su, sdp, sb, s * G::SUB, ch, nq);
#pragma unroll
            for (int j = 0; j < G::SUB; ++j) {
                const RowIn<K> x = next;
                if (j + 1 < G::SUB) next.load(su, sdp, sb, s * G::SUB + j + 1, ch, nq);
                stay_ahead();
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    e[j][k] = __builtin_amdgcn_exp2f(x.s.x * rate[k]);
                    h[j + 1][k] = fmaf(e[j][k], h[j][k], x.s.y * x.v[k]);
                    if (SPARE && nq + k >= n_state) e[j][k] = h[j + 1][k] = 0.f;
                }
            }
            float of_gb[4] = {}, of_eh[4] = {}, of_p[4] = {};
            RowIn<K> next_c;
            next.load(su, sdp, sb, (s + 1) * G::SUB - 1, ch, nq);
            next_c.load(su, sdp, sc, (s + 1) * G::SUB - 1, ch, nq);
#pragma unroll
            for (int j = G::SUB - 1; j >= 0; --j) {
                const int t = s * G::SUB + j;
                const RowIn<K> x = next, xc = next_c;
                if (j > 0) {
                    next.load(su, sdp, sb, t - 1, ch, nq);
                    next_c.load(su, sdp, sc, t - 1, ch, nq);
                }
                stay_ahead();
                float gb = 0.f, eha = 0.f, p = 0.f, w[V];
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const float c = xc.v[k];
                    float g = fmaf(c, x.dp, carried[k]);
                    if (SPARE && nq + k >= n_state) g = 0.f;
                    carried[k] = e[j][k] * g;
                    const float eh = carried[k] * h[j][k];
                    p = fmaf(c, h[j + 1][k], p);
                    gb = fmaf(g, x.v[k], gb);
                    eha = fmaf(eh, rate[k], eha);
                    da[k] = fmaf(eh, x.s.x, da[k]);
                    w[k] = g * x.s.y;
                    w[K + k] = x.dp * h[j + 1][k];
                }
                // lane q of a channel keeps every LN-th row; the rows' steps are not read again
                constexpr int kTurns = LN < G::SUB ? LN : G::SUB;
                if constexpr (LN == 4) {
                    of_gb[j % 4] = gb;
                    of_eh[j % 4] = eha;
                    of_p[j % 4] = p;
                    if (j % 4 == 0) {
                        su[t + tid % LN][ch] = make_float2(quad_sums(of_gb), quad_sums(of_eh));
                        sdp[t + tid % LN][ch] = quad_sums(of_p);
                    }
                } else {
                    gb = lanes_sum<LN>(gb);
                    eha = lanes_sum<LN>(eha);
                    p = lanes_sum<LN>(p);
                    const bool mine = j % kTurns == tid % LN;
                    of_gb[0] = mine ? gb : of_gb[0];
                    of_eh[0] = mine ? eha : of_eh[0];
                    of_p[0] = mine ? p : of_p[0];
                    if (j % kTurns == 0 && tid % LN < kTurns) {
                        su[t + tid % LN][ch] = make_float2(of_gb[0], of_eh[0]);
                        sdp[t + tid % LN][ch] = of_p[0];
                    }
                }
                // sums over the wavefront's channels (bits log2 LN .. 5 of the lane): a quarter of the values to each 16 lanes
                halve<5, V>(w);
                halve<4, V / 2>(w);
#pragma unroll
                for (int i = 0; i < V / 4; ++i) {
                    if (LN <= 8) w[i] = dpp_add<0x128>(w[i]);              // lanes eight apart
                    if (LN <= 4) w[i] = dpp_add<0x124>(w[i]);              // four apart (those eight apart are equal now)
                }
                const int lane = tid % 64, quarter = ((lane >> 5) * 2 + (lane >> 4 & 1)) * (V / 4);
                if (LN <= 8 && V >= 8) {                 // half of them from lanes with bit 3
                    const bool up = lane & 8;
#pragma unroll
                    for (int i = 0; i < V / 8; ++i) {
                        const int val = quarter + i + (up ? V / 8 : 0);
                        sbc[wave][t][val / K * G::NP + nq + val % K] = up ? w[i + V / 8] : w[i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < V / 4; ++i) {
                        const int val = quarter + i;
                        sbc[wave][t][val / K * G::NP + nq + val % K] = w[i];
                    }
                }
            }
        }
        __syncthreads();
        fetch(next_blk, it + 1, next_v);
        float par[2 * G::EPT];                           // the row's dskip, then its ddelta_bias
        Pack<T, G::EPT> du, dd, dz;
        float dstep[G::EPT], gb[G::EPT];
#pragma unroll
        for (int i = 0; i < G::EPT; ++i) {
            const float2 x = su[lt][lc + i];
            gb[i] = x.x;
            dstep[i] = fmaf((float)u.v[i], x.x, x.y * 0.693147180559945309f);      // (the rates are those of powers of two)
            dp[i] = (float)dy.v[i];
        }
        if (a.cfg.softplus) {
#pragma unroll
            for (int i = 0; i < G::EPT; ++i) dstep[i] *= sigmoid((float)delta.v[i] + sbias[lc + i]);
        }
        if (gate) {
#pragma unroll
            for (int i = 0; i < G::EPT; ++i) {
                const float zi = (float)z.v[i], sg = sigmoid(zi);
                dz.v[i] = (T)(dp[i] * fmaf(sskip[lc + i], (float)u.v[i], sdp[lt][lc + i]) * sg * (1.f + zi * (1.f - sg)));
                dp[i] *= zi * sg;
            }
        }
#pragma unroll
        for (int i = 0; i < G::EPT; ++i) {
            du.v[i] = (T)fmaf(step[i], gb[i], sskip[lc + i] * dp[i]);
            dd.v[i] = (T)dstep[i];
            par[i] = i < valid ? dp[i] * (float)u.v[i] : 0.f;
            par[G::EPT + i] = i < valid ? dstep[i] : 0.f;
        }
        if (lt >= pad) {
            if (a.grad.du.data) store_part<T, G::EPT, FULL>(a.grad.du, r, d0 + lc, du, valid);
            if (a.grad.ddelta.data) store_part<T, G::EPT, FULL>(a.grad.ddelta, r, d0 + lc, dd, valid);
            if (a.grad.dz.data) store_part<T, G::EPT, FULL>(a.grad.dz, r, d0 + lc, dz, valid);
        }
        sum_rows<G::CW / G::EPT, G::EPT>(par);
#pragma unroll
        for (int i = 0; i < kept<G::EPT>(); ++i) acc[i] += par[i];
        float* const bc = ws.bc + ((int64_t)tile * n_rows + begin) * 2 * n_state;
        for (int e = tid; e < here * 2 * G::NP; e += 256) {
            const int row = e / (2 * G::NP), t = row + pad, at = e % (2 * G::NP), n = at % G::NP;
            if (n < n_state) bc[row * 2 * n_state + (at < G::NP ? n : n_state + n)] = (sbc[0][t][at] + sbc[1][t][at]) + (sbc[2][t][at] + sbc[3][t][at]);
        }
        __syncthreads();
    }
    if (!ws.par) return;
    float* const par = ws.par + (int64_t)run * dim * (n_state + 2);
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (walks && nq + k < n_state) par[(int64_t)(d0 + ch) * n_state + nq + k] = da[k];
    // each wavefront's sums, then theirs
    float* const sums = &sdp[0][0];                      // [4][2][CW]
    if (tid % (2 * G::CW / G::EPT) < G::CW / G::EPT) {
#pragma unroll
        for (int i = 0; i < kept<G::EPT>(); ++i) {
            const int val = kept_from<G::EPT>(tid % 64) + i;
            sums[(wave * 2 + val / G::EPT) * G::CW + lc + val % G::EPT] = acc[i];
        }
    }
    __syncthreads();
    if (tid >= width) return;
#pragma unroll
    for (int j = 0; j < 2; ++j)
        par[(int64_t)dim * (n_state + j) + d0 + tid] = (sums[j * G::CW + tid] + sums[(2 + j) * G::CW + tid]) + (sums[(4 + j) * G::CW + tid] + sums[(6 + j) * G::CW + tid]);
}

// db and dc: sums over the tiles of a group, a group of threads per block of rows.
template <class T>
__global__ __launch_bounds__(256) void scan_bc_kernel(ScanArgs a, BackWs ws, BackPlan plan, int64_t n_rows) {
    const int n_state = a.cfg.n_state, n_group = a.cfg.n_group, tiles = plan.tiles / n_group, width = 2 * n_state * n_group;
    const int2 item = a.rows.items[blockIdx.x];
    const int64_t begin = a.rows.begin[item.x] + ((int64_t)item.y << a.rows.lg);
    const int n = (int)min(a.rows.end[item.x] - begin, (int64_t)1 << a.rows.lg) * width;
    for (int i = threadIdx.x; i < n; i += 256) {
        const int64_t r = begin + i / width;
        const int group = (i % width) / (2 * n_state), k = (i % width) % (2 * n_state);
        float acc = 0.f;
        constexpr int kAhead = 8;                        // tiles whose sums are on their way together
        for (int t = 0; t < tiles; t += kAhead) {
            float v[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) v[j] = t + j < tiles ? ws.bc[((int64_t)(group * tiles + t + j) * n_rows + r) * 2 * n_state + k] : 0.f;
#pragma unroll
            for (int j = 0; j < kAhead; ++j) acc += v[j];
        }
        const aug_rows& out = k < n_state ? a.grad.db : a.grad.dc;
        if (out.data) row_out<T>(out, r)[group * n_state + (k < n_state ? k : k - n_state)] = (T)acc;
    }
}

}  // namespace

template <class F> void with_groups(bool eight, F f) {
    if (eight) f(std::integral_constant<int, 8>());
    else f(std::integral_constant<int, 1>());
}

// Calls f with whether lanes have states to spare.
template <class F> hipError_t with_spare(bool spare, F f) { return spare ? f(std::true_type()) : f(std::false_type()); }

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
int back_lanes_of(int n_state) { return n_state <= 16 ? 4 : n_state <= 64 ? 8 : 16; }
int scan_tiles(const aug_scan_cfg& cfg, bool backward) {
    const int cw = 256 / (backward ? back_lanes_of(cfg.n_state) : lanes_of(cfg.n_state));
    return cfg.n_group * ((cfg.dim / cfg.n_group + cw - 1) / cw);
}

int scan_lg_block(const aug_scan_cfg& cfg, int n_seq, const int64_t* begin, const int64_t* lengths, int n_cu, bool backward) {
    if (backward) return cfg.n_state <= 64 ? 5 : 4;      // BackTile
    // Sixteen states: a compute unit with several groups takes some 75 ns for a row of one, a group by itself 136 ns (the latency of its chain), so
    // that a whole sequence takes no less than its length of those.  In blocks the walk is done nearly twice (end states, then outputs),
    // some 143 ns a row, with two launches more.  (Four sequences of 4000 rows, 2048 channels: whole 501 us, in blocks 235; 32 of 800, 1024
    // channels: 132 and 193; 16 of 800: 102 and 110.)  The other numbers of states follow the same rule, by their own tiles: 4 states 960 and 135,
    // 190 and 109, 190 and 76; 32 states 741 and 379, 201 and 311, 152 and 177; 128 states 1105 and 1340, 666 and 1059, 365 and 605.  It is wrong
    // by a fifth where 64 states leave it few long sequences (the first of these: taken whole 826, in blocks 666) and by a tenth for 64 of
    // 800 rows with 4 states (whole 223, in blocks 198).
    int64_t rows = 0, longest = 0;
    for (int i = 0; i < n_seq; ++i) {
        const int64_t len = lengths ? lengths[i] : begin[i + 1] - begin[i];
        rows += len;
        longest = longest > len ? longest : len;
    }
    const int64_t tiles = scan_tiles(cfg, false), filled = rows * tiles / n_cu;      // rows per compute unit
    if (longest <= filled + 96) return kWholeLg;
    int lg = 10;
    while (lg > 6 && (rows >> lg) * tiles < 8 * (int64_t)n_cu) --lg;
    return lg;
}
// The gradients' lanes: at least four per channel, so that a block's elements are eight to a lane at most.
template <class F> hipError_t with_back_lanes(int n_state, F f) {
    using std::integral_constant;
    if (n_state <= 8) return f(integral_constant<int, 4>(), integral_constant<int, 2>());
    if (n_state <= 16) return f(integral_constant<int, 4>(), integral_constant<int, 4>());
    if (n_state <= 32) return f(integral_constant<int, 8>(), integral_constant<int, 4>());
    if (n_state <= 64) return f(integral_constant<int, 8>(), integral_constant<int, 8>());
    return f(integral_constant<int, 16>(), integral_constant<int, 8>());
}
BackPlan back_plan(const aug_scan_cfg& cfg, int n_items, int n_cu) {
    BackPlan p;
    p.tiles = scan_tiles(cfg, true);
    const int64_t runs = (8 * (int64_t)n_cu + p.tiles - 1) / p.tiles;
    p.runs = (int)(runs < n_items ? runs : n_items);
    return p;
}
int scan_abreast(const aug_scan_cfg& cfg, int n_cu) {
    const int n = n_cu / scan_tiles(cfg, false);
    return n < 1 ? 1 : n;
}
size_t scan_workspace(const aug_scan_cfg& cfg, int n_items, int64_t n_rows, int n_cu, bool backward) {
    if (!backward) return 4 * (size_t)n_items * cfg.dim * (cfg.n_state + 1);      // first states, steps' sums
    const BackPlan p = back_plan(cfg, n_items, n_cu);
    return 4 * ((size_t)n_items * cfg.dim * (2 * cfg.n_state + 1) + (size_t)p.tiles * n_rows * 2 * cfg.n_state + (size_t)p.runs * cfg.dim * (cfg.n_state + 2));
}

hipError_t launch_scan(hipStream_t s, const ScanArgs& a, int n_cu) {
    const int tiles = scan_tiles(a.cfg, false);
    return with_type(a.cfg.dtype, [&](auto t) {
        return with_lanes(a.cfg.n_state, [&](auto ln, auto k) {
            return with_full(a.cfg.dim / a.cfg.n_group % (256 / ln.value) == 0, [&](auto full) {
                using T = decltype(t);
                const dim3 grid((unsigned)(tiles * a.rows.n_items));
                float* const first_state = static_cast<float*>(a.ws);
                float* const step_sum = first_state + (int64_t)a.rows.n_items * a.cfg.dim * a.cfg.n_state;
                if (a.rows.lg == kWholeLg) {
                    return with_spare(a.cfg.n_state < ln.value * k.value, [&](auto spare) {
                        scan_kernel<T, ln.value, k.value, kWhole, full.value, spare.value><<<grid, dim3(256), 0, s>>>(a, tiles, nullptr, nullptr);
                        return hipGetLastError();
                    });
                }
                scan_kernel<T, ln.value, k.value, kSums, full.value, false><<<grid, dim3(256), 0, s>>>(a, tiles, first_state, step_sum);
                hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
                const int64_t width = (int64_t)a.cfg.dim * a.cfg.n_state;
                with_groups(join_in_groups(width, a.rows.n_seq, a.rows.n_items, n_cu), [&](auto g) {
                    constexpr int n = kJoinStates<g.value>;
                    scan_join_kernel<g.value><<<dim3((unsigned)((width + n - 1) / n), (unsigned)a.rows.n_seq), dim3(n * g.value), 0, s>>>(a, first_state, step_sum);
                });
                e = hipGetLastError();
                if (e != hipSuccess) return e;
                return with_spare(a.cfg.n_state < ln.value * k.value, [&](auto spare) {
                    scan_kernel<T, ln.value, k.value, kResume, full.value, spare.value><<<grid, dim3(256), 0, s>>>(a, tiles, first_state, step_sum);
                    return hipGetLastError();
                });
            });
        });
    });
}

hipError_t launch_scan_step(hipStream_t s, int n_seq, const ScanArgs& a, int n_cu) {
    // as many streams to a group as leave eight groups to a compute unit
    const int64_t tiles = scan_tiles(a.cfg, false), each = n_seq * tiles / (8 * (int64_t)n_cu);
    const int streams = each < 1 ? 1 : each > 16 ? 16 : (int)each;
    return with_type(a.cfg.dtype, [&](auto t) {
        return with_lanes(a.cfg.n_state, [&](auto ln, auto k) {
            scan_step_kernel<decltype(t), ln.value, k.value>
                <<<dim3((unsigned)tiles, (unsigned)((n_seq + streams - 1) / streams)), dim3(256), 0, s>>>(a, n_seq, streams);
            return hipGetLastError();
        });
    });
}

hipError_t launch_scan_backward(hipStream_t s, const ScanArgs& a, int64_t n_rows, int n_cu) {
    const BackPlan plan = back_plan(a.cfg, a.rows.n_items, n_cu);
    BackWs ws = back_ws(a.cfg, a.ws, a.rows.n_items, n_rows, plan.tiles);
    const int64_t dim = a.cfg.dim, width = dim * a.cfg.n_state, stride = width + 2 * dim;
    if (!a.grad.da && !a.grad.dskip && !a.grad.ddelta_bias) ws.par = nullptr;
    const bool joined = a.rows.n_items > a.rows.n_seq;   // a sequence of more than one block
    hipError_t e = with_type(a.cfg.dtype, [&](auto t) {
        return with_back_lanes(a.cfg.n_state, [&](auto ln, auto k) {
            using T = decltype(t);
            hipError_t e = with_full(a.cfg.dim / a.cfg.n_group % (256 / ln.value) == 0, [&](auto full) {
                if (joined) {
                    scan_back_sums_kernel<T, ln.value, k.value, full.value><<<dim3((unsigned)(plan.tiles * a.rows.n_items)), dim3(256), 0, s>>>(a, ws, plan.tiles);
                    hipError_t e = hipGetLastError();
                    if (e != hipSuccess) return e;
                    with_groups(join_in_groups(width, a.rows.n_seq, a.rows.n_items, n_cu), [&](auto g) {
                        constexpr int n = kJoinStates<g.value>;
                        scan_back_join_kernel<g.value><<<dim3((unsigned)((width + n - 1) / n), (unsigned)a.rows.n_seq), dim3(n * g.value), 0, s>>>(a, ws);
                    });
                    e = hipGetLastError();
                    if (e != hipSuccess) return e;
                }
                return with_spare(a.cfg.n_state < ln.value * k.value, [&](auto spare) {
                    scan_back_kernel<T, ln.value, k.value, full.value, spare.value><<<dim3((unsigned)(plan.tiles * plan.runs)), dim3(256), 0, s>>>(a, ws, plan, n_rows, joined);
                    return hipGetLastError();
                });
            });
            if (e != hipSuccess || (!a.grad.db.data && !a.grad.dc.data)) return e;
            scan_bc_kernel<T><<<dim3((unsigned)a.rows.n_items), dim3(256), 0, s>>>(a, ws, plan, n_rows);
            return hipGetLastError();
        });
    });
    if (e == hipSuccess && ws.par) e = launch_sum_partials(s, ws.par, plan.runs, stride, {{{a.grad.da, width}, {a.grad.dskip, dim}, {a.grad.ddelta_bias, dim}}});
    return e;
}

}  // namespace aug
