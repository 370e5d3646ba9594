// The API layer of the operators on feature rows on a host runtime (that of out_of_memory.cpp): what it refuses, with nothing
// launched, and that after a call that ran out of memory the tables are what the context says.  Built by test_rows_api.py.
#define main out_of_memory_main
#include "out_of_memory.cpp"
#undef main
#include "../../paper_1912_11040_amd/csrc/rows_api.hip"

static int g_launches = 0, g_tables = 0;
static bool g_capturing = false;
static int g_device = 0;
static const int64_t *g_begin, *g_lengths;
static int g_n_seq;

extern "C" hipError_t hipGetDevice(int* d) { *d = g_device; return hipSuccess; }

namespace aug {
static int64_t end_of(int i) { return g_lengths ? g_begin[i] + g_lengths[i] : g_begin[i + 1]; }
hipError_t launch_row_tables(hipStream_t, const RowTableArgs& a) {
    ++g_tables;
    for (int i = 0; i <= a.n_seq; ++i) {
        if (a.begin) a.d_begin[i] = a.begin[i], a.d_end[i] = a.end[i];
        if (a.whole) {
            if (i < a.n_seq) a.items[a.first[i]] = make_int2(i, 0);
            continue;
        }
        a.d_first[i] = a.first[i];
        for (int j = 0; i < a.n_seq && j < a.first[i + 1] - a.first[i]; ++j) a.items[a.first[i] + j] = make_int2(i, j);
    }
    return hipSuccess;
}
static void check_blocks(const RowBlocks& b) {
    ++g_launches;
    EXPECT(b.n_seq == g_n_seq);
    std::vector<int> seen(b.n_seq, 0);
    for (int i = 0; i < b.n_seq; ++i) EXPECT(b.begin[i] == g_begin[i] && b.end[i] == end_of(i));
    for (int j = 0; j < b.n_items; ++j) {
        const int2 it = b.items[j];
        if (it.x < 0 || it.x >= b.n_seq) { EXPECT(!"a block of no sequence"); return; }
        EXPECT(it.y == 0 || ((int64_t)it.y << b.lg) < end_of(it.x) - g_begin[it.x]);
        ++seen[it.x];
    }
    for (int i = 0; i < b.n_seq; ++i) {
        const int64_t len = end_of(i) - g_begin[i];
        EXPECT(seen[i] == (len ? (int)((len + ((int64_t)1 << b.lg) - 1) >> b.lg) : 1));
    }
}
hipError_t launch_sum_partials(hipStream_t, const float*, int, int64_t, const SumOuts&) { ++g_launches; return hipSuccess; }
hipError_t launch_norm(hipStream_t, const NormArgs&, int) { ++g_launches; return hipSuccess; }
int norm_partials(int64_t n, int, int) { return (int)(n < 512 ? n : 512); }
hipError_t launch_norm_backward(hipStream_t, const NormBackArgs&, int) { ++g_launches; return hipSuccess; }
int short_conv_tiles(const aug_short_conv_cfg& c, bool) { return (c.dim + 255) / 256; }
int short_conv_lg_block(const aug_short_conv_cfg&, bool backward) { return backward ? 7 : 6; }
int short_conv_partials(const aug_short_conv_cfg&, int n, int) { return n; }
hipError_t launch_short_conv(hipStream_t, const ShortConvArgs& a) { check_blocks(a.rows); return hipSuccess; }
hipError_t launch_short_conv_backward(hipStream_t, const ShortConvArgs& a, int) { check_blocks(a.rows); return hipSuccess; }
hipError_t launch_short_conv_step(hipStream_t, int, const ShortConvArgs&) { ++g_launches; return hipSuccess; }
int scan_tiles(const aug_scan_cfg& c, bool) { return (c.dim + 63) / 64; }
int scan_abreast(const aug_scan_cfg&, int) { return 3; }
int scan_lg_block(const aug_scan_cfg&, int, const int64_t*, const int64_t*, int, bool backward) { return backward ? 5 : kWholeLg; }
size_t scan_workspace(const aug_scan_cfg& c, int n_items, int64_t, int, bool) { return (size_t)n_items * c.dim * c.n_state * 4; }
hipError_t launch_scan(hipStream_t, const ScanArgs& a, int) { check_blocks(a.rows); return hipSuccess; }
hipError_t launch_scan_backward(hipStream_t, const ScanArgs& a, int64_t, int) { check_blocks(a.rows); return hipSuccess; }
hipError_t launch_scan_step(hipStream_t, int, const ScanArgs&, int) { ++g_launches; return hipSuccess; }
}  // namespace aug

// Addresses far apart that nothing here follows.
static char* place(int i) { return reinterpret_cast<char*>((uintptr_t)(i + 1) << 44); }
static float* floats(int i) { return reinterpret_cast<float*>(place(i)); }
static aug_rows rows(int i, int64_t ld = 64) { return {place(i), ld}; }

#define REFUSED(code, expr)                                                                                        \
    do {                                                                                                           \
        const int l0 = g_launches + g_tables, rc = (expr);                                                         \
        if (rc != (code) || g_launches + g_tables != l0 || !aug_last_error(ctx)[0]) {                              \
            ++g_faults;                                                                                            \
            printf("line %d: %s gave %d (%s), %d launches\n", __LINE__, #expr, rc, aug_last_error(ctx), g_launches + g_tables - l0); \
        }                                                                                                          \
    } while (0)
#define ACCEPTED(expr)                                                                                             \
    do {                                                                                                           \
        const int rc = (expr);                                                                                     \
        if (rc != AUG_OK) { ++g_faults; printf("line %d: %s gave %d (%s)\n", __LINE__, #expr, rc, aug_last_error(ctx)); } \
    } while (0)

static void norm(aug_ctx* ctx) {
    const aug_norm_cfg ok{AUG_BF16, 64, 1e-6f, 32};
    const aug_rows x = rows(0), r = rows(1), s = rows(2), y = rows(3), q = rows(4), none{nullptr, 0};
    auto call = [&](const aug_norm_cfg& c, int64_t n, const aug_rows* px, const aug_rows* pr, const aug_rows* ps, const aug_rows* py,
                    const aug_rows* pq, float* scale) { return aug_rms_norm_batch(ctx, n, &c, px, pr, floats(5), ps, py, pq, scale, floats(7)); };
    ACCEPTED(call(ok, 8, &x, &r, &s, &y, &q, floats(6)));
    ACCEPTED(call(ok, 8, &x, nullptr, &none, nullptr, &q, floats(6)));
    ACCEPTED(call(ok, 8, &x, &r, &x, &r, nullptr, nullptr));           // in place of both
    ACCEPTED(call(ok, 0, &none, &none, &none, &none, &none, nullptr));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 8, nullptr, &r, &s, &y, nullptr, nullptr));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, -1, &x, &r, &s, &y, nullptr, nullptr));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 8, &x, &r, &s, &y, &q, nullptr));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 8, &x, &r, &x, &x, nullptr, nullptr));      // two outputs in one place
    const aug_rows shifted{place(0) + 16, 64}, narrow{place(3), 63}, other{place(0), 128};
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 8, &x, &r, &s, &shifted, nullptr, nullptr));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 8, &x, &r, &s, &other, nullptr, nullptr));  // x's place with another ld
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 8, &x, &r, &s, &narrow, nullptr, nullptr));
    const aug_rows vast{place(3), (int64_t)1 << 46};
    REFUSED(AUG_ERR_UNSUPPORTED, call(ok, 8, &x, &r, &s, &vast, nullptr, nullptr));
    REFUSED(AUG_ERR_UNSUPPORTED, call(ok, (int64_t)1 << 41, &x, &r, &s, &y, nullptr, nullptr));
    const aug_rows left{place(8), 128}, right{place(8) + 128, 128};
    ACCEPTED(call(ok, 8, &left, &r, &s, &right, nullptr, nullptr));    // the two halves of a matrix
    aug_norm_cfg c = ok;
    for (int qb : {8, 24, 1024, -16}) { c.q_block = qb; REFUSED(AUG_ERR_INVALID_ARG, call(c, 8, &x, &r, &s, &y, nullptr, nullptr)); }
    c = ok; c.dtype = 3; REFUSED(AUG_ERR_INVALID_ARG, call(c, 8, &x, &r, &s, &y, nullptr, nullptr));
    c = ok; c.dim = 0; REFUSED(AUG_ERR_INVALID_ARG, call(c, 8, &x, &r, &s, &y, nullptr, nullptr));
    c = ok; c.dim = AUG_MAX_NORM_DIM + 1; REFUSED(AUG_ERR_UNSUPPORTED, call(c, 8, &x, &r, &s, &y, nullptr, nullptr));
    for (float eps : {-1.f, NAN, INFINITY}) { c = ok; c.eps = eps; REFUSED(AUG_ERR_INVALID_ARG, call(c, 8, &x, &r, &s, &y, nullptr, nullptr)); }
    REFUSED(AUG_ERR_INVALID_ARG, aug_rms_norm_batch(ctx, 8, nullptr, &x, &r, nullptr, &s, &y, nullptr, nullptr, nullptr));

    auto back = [&](int64_t n, const aug_rows* ps, const float* rstd, const aug_rows* dy, const aug_rows* dx, float* dw) {
        return aug_rms_norm_backward_batch(ctx, n, &ok, ps, floats(5), rstd, dy, &r, dx, dw); };
    ACCEPTED(back(8, &x, floats(6), &s, &s, floats(7)));
    ACCEPTED(back(0, &none, nullptr, &none, &none, floats(7)));
    REFUSED(AUG_ERR_INVALID_ARG, back(8, &x, nullptr, &s, &y, floats(7)));
    REFUSED(AUG_ERR_INVALID_ARG, back(8, &x, floats(6), nullptr, &y, floats(7)));
    REFUSED(AUG_ERR_INVALID_ARG, back(8, &x, floats(6), &s, &y, floats(5)));          // the weight's gradient onto the weight
    REFUSED(AUG_ERR_INVALID_ARG, back(8, &x, floats(6), &s, &shifted, floats(7)));
}

static int64_t off[] = {0, 5, 5, 75, 80}, lens[] = {4, 0, 70, 5};
static void batch(const int64_t* begin, const int64_t* lengths, int n) { g_begin = begin, g_lengths = lengths, g_n_seq = n; }

static void conv(aug_ctx* ctx) {
    const aug_short_conv_cfg ok{AUG_F16, 64, 4, 1};
    const aug_rows x = rows(0), y = rows(3), dy = rows(4), none{nullptr, 0};
    auto call = [&](const aug_short_conv_cfg& c, int n, const int64_t* o, const int64_t* l, const aug_rows* px, void* in, void* out, const aug_rows* py) {
        batch(o, l, n);
        return aug_short_conv_batch(ctx, n, o, l, &c, px, floats(5), floats(6), in, out, py); };
    ACCEPTED(call(ok, 4, off, nullptr, &x, place(7), place(8), &y));
    ACCEPTED(call(ok, 4, off, lens, &x, place(7), place(7), &y));
    ACCEPTED(call(ok, 4, off, nullptr, &x, nullptr, nullptr, &y));
    ACCEPTED(call(ok, 0, off, nullptr, &none, nullptr, nullptr, &none));
    int64_t bad_off[] = {0, 5, 4, 75, 80}, start[] = {1, 5, 5, 75, 80}, neg[] = {4, -1, 70, 5}, more[] = {6, 0, 70, 5}, vast[] = {0, (int64_t)1 << 30},
            rows41[] = {0, (int64_t)1 << 41};
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 4, bad_off, nullptr, &x, nullptr, nullptr, &y));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 4, start, nullptr, &x, nullptr, nullptr, &y));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 4, off, neg, &x, nullptr, nullptr, &y));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 4, off, more, &x, nullptr, nullptr, &y));
    REFUSED(AUG_ERR_UNSUPPORTED, call(ok, 1, vast, nullptr, &x, nullptr, nullptr, &y));
    REFUSED(AUG_ERR_UNSUPPORTED, call(ok, 1, rows41, nullptr, &x, nullptr, nullptr, &y));
    REFUSED(AUG_ERR_UNSUPPORTED, call(ok, AUG_MAX_UTT + 1, off, nullptr, &x, nullptr, nullptr, &y));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, -1, off, nullptr, &x, nullptr, nullptr, &y));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 4, nullptr, nullptr, &x, nullptr, nullptr, &y));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 4, off, nullptr, &none, nullptr, nullptr, &y));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 4, off, nullptr, &x, nullptr, nullptr, nullptr));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 4, off, nullptr, &x, nullptr, nullptr, &x));          // rows need those before them
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, 4, off, nullptr, &x, place(7), place(7) + 2, &y));
    int64_t many[] = {0, ((int64_t)1 << 30) - 1};
    aug_short_conv_cfg c = ok; c.dim = 512;
    const aug_rows wx = rows(0, 512), wy = rows(9, 512);
    REFUSED(AUG_ERR_UNSUPPORTED, call(c, 1, many, nullptr, &wx, nullptr, nullptr, &wy));         // 2^24 blocks, two groups each
    c = ok; c.taps = 0; REFUSED(AUG_ERR_INVALID_ARG, call(c, 4, off, nullptr, &x, nullptr, nullptr, &y));
    c = ok; c.taps = AUG_MAX_TAPS + 1; REFUSED(AUG_ERR_UNSUPPORTED, call(c, 4, off, nullptr, &x, nullptr, nullptr, &y));
    c = ok; c.dim = AUG_MAX_DIM + 1; REFUSED(AUG_ERR_UNSUPPORTED, call(c, 4, off, nullptr, &x, nullptr, nullptr, &y));
    c = ok; c.dtype = -1; REFUSED(AUG_ERR_INVALID_ARG, call(c, 4, off, nullptr, &x, nullptr, nullptr, &y));
    auto back = [&](const aug_rows* pdy, const aug_rows* dx, float* dw, float* db) {
        batch(off, nullptr, 4);
        return aug_short_conv_backward_batch(ctx, 4, off, nullptr, &ok, &x, floats(5), floats(6), place(7), pdy, dx, dw, db); };
    ACCEPTED(back(&dy, &y, floats(8), floats(9)));
    ACCEPTED(back(&dy, nullptr, nullptr, floats(9)));
    ACCEPTED(back(&dy, nullptr, nullptr, nullptr));
    REFUSED(AUG_ERR_INVALID_ARG, back(&dy, &dy, floats(8), floats(9)));               // rows need dy of those behind them
    REFUSED(AUG_ERR_INVALID_ARG, back(nullptr, &y, floats(8), floats(9)));
    REFUSED(AUG_ERR_INVALID_ARG, back(&dy, &y, floats(8), floats(8) + 3));
    auto step = [&](int n, void* in, void* out, const aug_rows* py) { return aug_short_conv_step(ctx, n, &ok, &x, floats(5), nullptr, in, out, py); };
    ACCEPTED(step(8, place(7), place(7), &x));
    REFUSED(AUG_ERR_INVALID_ARG, step(8, nullptr, place(7), &y));
    REFUSED(AUG_ERR_INVALID_ARG, step(8, place(7), nullptr, &y));
    REFUSED(AUG_ERR_UNSUPPORTED, step(AUG_MAX_UTT + 1, place(7), place(8), &y));
}

static void scan(aug_ctx* ctx) {
    const aug_scan_cfg ok{AUG_F32, 64, 16, 2, 1};
    const aug_scan_in in{rows(0), rows(1), rows(2), rows(3), rows(4), floats(5), floats(6), floats(7)};
    const aug_rows y = rows(8), dy = rows(9), none{nullptr, 0};
    auto call = [&](const aug_scan_cfg& c, const aug_scan_in& i, const int64_t* l, float* si, float* so, const aug_rows* py) {
        batch(off, l, 4);
        return aug_scan_batch(ctx, 4, off, l, &c, &i, si, so, py); };
    ACCEPTED(call(ok, in, nullptr, floats(10), floats(11), &y));
    ACCEPTED(call(ok, in, lens, floats(10), floats(10), &y));
    aug_scan_in i = in; i.z = none; i.skip = nullptr; i.delta_bias = nullptr;
    ACCEPTED(call(ok, i, nullptr, nullptr, nullptr, &y));
    i = in; i.a = nullptr; REFUSED(AUG_ERR_INVALID_ARG, call(ok, i, nullptr, nullptr, nullptr, &y));
    i = in; i.u = none; REFUSED(AUG_ERR_INVALID_ARG, call(ok, i, nullptr, nullptr, nullptr, &y));
    i = in; i.b.ld = 31; REFUSED(AUG_ERR_INVALID_ARG, call(ok, i, nullptr, nullptr, nullptr, &y));
    for (const aug_rows* m : {&in.u, &in.delta, &in.z, &in.b}) REFUSED(AUG_ERR_INVALID_ARG, call(ok, in, nullptr, nullptr, nullptr, m));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, in, nullptr, floats(10), floats(10) + 1, &y));
    REFUSED(AUG_ERR_INVALID_ARG, call(ok, in, nullptr, nullptr, floats(5), &y));
    aug_scan_cfg c = ok; c.n_group = 3; REFUSED(AUG_ERR_INVALID_ARG, call(c, in, nullptr, nullptr, nullptr, &y));
    c = ok; c.n_state = 0; REFUSED(AUG_ERR_INVALID_ARG, call(c, in, nullptr, nullptr, nullptr, &y));
    c = ok; c.n_state = AUG_MAX_STATE + 1; REFUSED(AUG_ERR_UNSUPPORTED, call(c, in, nullptr, nullptr, nullptr, &y));
    c = ok; c.dtype = 9; REFUSED(AUG_ERR_INVALID_ARG, call(c, in, nullptr, nullptr, nullptr, &y));
    const aug_scan_grad all{rows(10), rows(11), rows(12), rows(13), rows(14), floats(15), floats(16), floats(17)};
    auto back = [&](const aug_scan_in& si, const aug_rows* pdy, const aug_scan_grad& g) {
        batch(off, nullptr, 4);
        return aug_scan_backward_batch(ctx, 4, off, nullptr, &ok, &si, nullptr, pdy, &g); };
    ACCEPTED(back(in, &dy, all));
    ACCEPTED(back(in, &dy, aug_scan_grad{}));
    REFUSED(AUG_ERR_INVALID_ARG, back(in, nullptr, all));
    i = in; i.z = none; REFUSED(AUG_ERR_INVALID_ARG, back(i, &dy, all));               // dz without a gate
    aug_scan_grad g = all; g.du = in.u; REFUSED(AUG_ERR_INVALID_ARG, back(in, &dy, g));
    g = all; g.dskip = g.ddelta_bias; REFUSED(AUG_ERR_INVALID_ARG, back(in, &dy, g));
    g = all; g.dc.ld = 3; REFUSED(AUG_ERR_INVALID_ARG, back(in, &dy, g));
    REFUSED(AUG_ERR_INVALID_ARG, aug_scan_backward_batch(ctx, 4, off, nullptr, &ok, &in, nullptr, &dy, nullptr));
    auto step = [&](const aug_scan_in& si, float* hi, float* ho, const aug_rows* py) { return aug_scan_step(ctx, 8, &ok, &si, hi, ho, py); };
    ACCEPTED(step(in, floats(10), floats(10), &in.u));
    ACCEPTED(step(in, floats(10), floats(11), &in.z));
    REFUSED(AUG_ERR_INVALID_ARG, step(in, floats(10), floats(11), &in.b));
    REFUSED(AUG_ERR_INVALID_ARG, step(in, nullptr, floats(11), &y));
}

// Calls with other sequences in turn, one of them out of memory at each of its allocations: the tables stay true, and a call with the
// sequences of the one before it builds none.
static int out_of_memory() {
    std::vector<int64_t> large{0};
    for (int i = 0; i < 5000; ++i) large.push_back(large.back() + 30 + i % 200);
    const aug_short_conv_cfg cc{AUG_F32, 64, 4, 1};
    const aug_scan_cfg sc{AUG_F32, 64, 16, 1, 1};
    const aug_scan_in in{rows(0), rows(1), rows(2), rows(3), rows(4), floats(5), nullptr, nullptr};
    const aug_rows y = rows(8), x = rows(0), dy = rows(9);
    const aug_scan_grad g{rows(10), rows(11), rows(12), rows(13), rows(14), floats(15), floats(16), floats(17)};
    auto call = [&](aug_ctx* ctx, int entry, const int64_t* o, int n) {
        batch(o, nullptr, n);
        switch (entry) {
            case 0: return aug_short_conv_batch(ctx, n, o, nullptr, &cc, &x, floats(5), nullptr, nullptr, nullptr, &y);
            case 1: return aug_short_conv_backward_batch(ctx, n, o, nullptr, &cc, &x, floats(5), nullptr, nullptr, &dy, &y, floats(8) + (1 << 30), nullptr);
            case 2: return aug_scan_batch(ctx, n, o, nullptr, &sc, &in, nullptr, nullptr, &y);
            default: return aug_scan_backward_batch(ctx, n, o, nullptr, &sc, &in, nullptr, &dy, &g);
        }
    };
    int refused = 0;
    for (int first = 0; first < 4; ++first)
        for (int second = 0; second < 4; ++second)
            for (int k = 0;; ++k) {
                aug_ctx* ctx = nullptr;
                EXPECT(aug_create(&ctx, 0, nullptr) == AUG_OK);
                ACCEPTED(call(ctx, first, off, 4));
                g_until_failure = k;
                const int rc = call(ctx, second, large.data(), 5000);
                g_until_failure = -1;
                EXPECT(rc == AUG_OK || rc == AUG_ERR_NOMEM);
                refused += rc == AUG_ERR_NOMEM;
                ACCEPTED(call(ctx, first, off, 4));
                const int t = g_tables;
                ACCEPTED(call(ctx, first, off, 4));
                EXPECT(g_tables == t);                   // the same sequences: launches of the operator only
                ACCEPTED(call(ctx, second, large.data(), 5000));
                ACCEPTED(call(ctx, first, large.data(), 5000));
                ACCEPTED(call(ctx, second, large.data(), 5000));
                aug_destroy(ctx);
                if (rc == AUG_OK) break;
            }
    return refused;
}

int main() {
    aug_ctx* ctx = nullptr;
    EXPECT(aug_create(&ctx, 0, nullptr) == AUG_OK);
    norm(ctx);
    conv(ctx);
    scan(ctx);
    aug_destroy(ctx);
    EXPECT(aug_scan_batch(nullptr, 0, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) == AUG_ERR_INVALID_ARG);
    const int refused = out_of_memory();
    printf("%d launches, %d calls out of memory, %d faults\n", g_launches, refused, g_faults);
    return g_faults || refused < 32;
}
