// C ABI of the operators on feature rows: argument checks, the tables that cut sequences into blocks, workspace,
// launches.  No arithmetic of the operators lives here.

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "api_common.h"
#include "rows_internal.h"

namespace {

using aug::fail;
using aug::fail_hip;
using aug::grow;
using aug::mark;
using aug::RowBlocks;

// The caller's current device, put back at the end of the call; nothing is thrown across the boundary.
template <class F>
int guarded(aug_ctx* ctx, F body) {
    int before = -1;
    if (hipGetDevice(&before) != hipSuccess) (void)hipGetLastError();
    int rc = aug::enter(ctx);
    try {
        if (rc == AUG_OK) rc = body();
    } catch (const std::bad_alloc&) {
        rc = AUG_ERR_NOMEM;
    }
    if (ctx && before >= 0 && before != ctx->device && hipSetDevice(before) != hipSuccess) (void)hipGetLastError();
    return rc;
}

int element_bytes(int dtype) { return dtype == AUG_F32 ? 4 : 2; }

int check_dtype(aug_ctx* ctx, int dtype) {
    return dtype == AUG_F32 || dtype == AUG_BF16 || dtype == AUG_F16 ? AUG_OK : fail(ctx, AUG_ERR_INVALID_ARG, "unknown element type %d", dtype);
}

// The memory that a call reads and writes: `rows` stretches of `width` bytes, `pitch` apart.
struct Spans {
    struct Span {
        const char* name;
        uintptr_t at;
        int64_t pitch, width, rows;
        int out;
        int in_place;                // an output that may be this span, a bit per span
    };
    Span s[24];
    int n = 0;
    int add(const char* name, const void* p, int64_t pitch, int64_t width, int64_t rows, int out, int in_place) {
        if (!p || width <= 0 || rows <= 0 || n == 24) return 0;
        s[n] = {name, reinterpret_cast<uintptr_t>(p), rows > 1 ? pitch : width, width, rows, out, in_place};
        return 1 << n++;
    }
    static bool overlap(const Span& a, const Span& b) {
        const uintptr_t ea = a.at + (uintptr_t)((a.rows - 1) * a.pitch + a.width), eb = b.at + (uintptr_t)((b.rows - 1) * b.pitch + b.width);
        if (ea <= b.at || eb <= a.at) return false;
        const int64_t pitch = a.rows > 1 ? a.pitch : b.pitch;
        if (pitch == (b.rows > 1 ? b.pitch : a.pitch) && (a.rows > 1 || b.rows > 1)) {      // columns of one matrix
            const int64_t d = (int64_t)(a.at >= b.at ? (a.at - b.at) % (uintptr_t)pitch : (pitch - (int64_t)((b.at - a.at) % (uintptr_t)pitch)) % pitch);
            if (d >= b.width && d + a.width <= pitch) return false;
        }
        return true;
    }
    int check(aug_ctx* ctx) const {
        for (int i = 0; i < n; ++i)
            for (int j = 0; j < n; ++j) {
                if (i == j || !s[i].out || (s[j].out && j < i)) continue;
                const bool same = s[i].at == s[j].at && s[i].pitch == s[j].pitch && s[i].width == s[j].width;
                if (same && ((s[i].in_place >> j) & 1)) continue;
                if (overlap(s[i], s[j])) return fail(ctx, AUG_ERR_INVALID_ARG, "%s overlaps %s", s[i].name, s[j].name);
            }
        return AUG_OK;
    }
};

// A matrix argument: null only where it is optional or has no elements.
int check_rows(aug_ctx* ctx, const char* name, const aug_rows* m, int64_t n_rows, int64_t width, bool needed) {
    if (!m || !m->data) return needed && n_rows > 0 && width > 0 ? fail(ctx, AUG_ERR_INVALID_ARG, "%s is null", name) : AUG_OK;
    if (m->ld < width) return fail(ctx, AUG_ERR_INVALID_ARG, "ld of %s is less than its width", name);
    if (n_rows > 0 && m->ld > ((int64_t)1 << 48) / n_rows) return fail(ctx, AUG_ERR_UNSUPPORTED, "%s is too large", name);
    return AUG_OK;
}

aug_rows of(const aug_rows* m) { return m ? *m : aug_rows{nullptr, 0}; }

// ---- sequences ----

int check_sequences(aug_ctx* ctx, int n_seq, const int64_t* offsets, const int64_t* lengths) {
    if (n_seq < 0) return fail(ctx, AUG_ERR_INVALID_ARG, "n_seq is negative");
    if (n_seq > AUG_MAX_UTT) return fail(ctx, AUG_ERR_UNSUPPORTED, "more than %d sequences in one call", AUG_MAX_UTT);
    if (!offsets) return fail(ctx, AUG_ERR_INVALID_ARG, "row_offsets is null");
    if (offsets[0] != 0) return fail(ctx, AUG_ERR_INVALID_ARG, "row_offsets[0] must be 0");
    for (int i = 0; i < n_seq; ++i) {
        if (offsets[i + 1] < offsets[i]) return fail(ctx, AUG_ERR_INVALID_ARG, "row_offsets not ascending at sequence %d", i);
        if (offsets[i + 1] > ((int64_t)1 << 40)) return fail(ctx, AUG_ERR_UNSUPPORTED, "too many rows in one call");
        const int64_t has = offsets[i + 1] - offsets[i], len = lengths ? lengths[i] : has;
        if (len < 0 || len > has) return fail(ctx, AUG_ERR_INVALID_ARG, "row_lengths[%d] is negative or more than the sequence's rows", i);
        if (len >= ((int64_t)1 << 30)) return fail(ctx, AUG_ERR_UNSUPPORTED, "sequence %d is 2^30 rows or longer", i);
    }
    return AUG_OK;
}

// The sequences of a call between their checks and the launch that builds their tables.
struct Sequences {
    aug_ctx* ctx;
    int n_seq;
    const int64_t *offsets, *lengths;
    int64_t n_rows = 0;                  // rows up to the last sequence's end
    int64_t total = 0;                   // rows of the sequences
    RowBlocks blocks;
    size_t order = 0;                    // the table of whole sequences
    bool new_rows = false, new_table = false;

    Sequences(aug_ctx* c, int n, const int64_t* o, const int64_t* l) : ctx(c), n_seq(n), offsets(o), lengths(l) {
        for (int i = 0; i < n; ++i) {
            total += end(i) - o[i];
            if (end(i) > o[i]) n_rows = end(i);
        }
    }
    int64_t end(int i) const { return lengths ? offsets[i] + lengths[i] : offsets[i + 1]; }

    // Cut into blocks of 1 << lg rows, each of which `tiles` work groups share; left whole, `abreast` of them are taken side by side.
    // Memory is found here, nothing is launched.
    int plan(int lg, int tiles, int abreast = 1) {
        aug::RowTables& t = aug::whole(ctx).rows;
        const size_t n = (size_t)n_seq + 1;
        bool same = t.begin.size() == n && !memcmp(t.begin.data(), offsets, n * sizeof(int64_t));
        for (int i = 0; same && i < n_seq; ++i) same = t.end[i] == end(i);
        int64_t items = 0;
        for (int i = 0; i < n_seq; ++i) items += blocks_of(i, lg);
        if (items * tiles >= (int64_t)1 << 24) return fail(ctx, AUG_ERR_UNSUPPORTED, "too many blocks of rows and channels in one call");
        blocks.n_seq = n_seq;
        blocks.lg = lg;
        blocks.n_items = (int)items;
        new_rows = n_seq > 0 && !same;
        const bool whole = lg == aug::kWholeLg;
        if (whole) {
            if (abreast >= n_seq) abreast = 0;
            for (order = 0; order < t.orders.size() && t.orders[order].abreast != abreast;) ++order;
            if (order == t.orders.size()) {
                t.orders.emplace_back();
                t.orders[order].abreast = abreast;
            }
        }
        const bool there = whole ? t.orders[order].there : t.n_items[lg] > 0;
        new_table = n_seq > 0 && (new_rows || !there);
        if (new_table) {
            hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
            if (hipStreamIsCapturing(ctx->stream, &st) != hipSuccess) (void)hipGetLastError();
            if (st != hipStreamCaptureStatusNone)
                return fail(ctx, AUG_ERR_UNSUPPORTED, "the tables for these rows are not there: they cannot be built while the stream is "
                            "being captured (run the same call once before capturing it)");
            if (new_rows) {              // (the record is true again once the tables are launched)
                t.forget();
                AUG_TRY(grow(ctx, t.d_begin, n * sizeof(int64_t), "row offsets buffer"));
                AUG_TRY(grow(ctx, t.d_end, n * sizeof(int64_t), "row ends buffer"));
            }
            if (!whole) AUG_TRY(grow(ctx, t.d_first[lg], n * sizeof(int), "row block prefix table"));
            AUG_TRY(grow(ctx, whole ? t.orders[order].d_items : t.d_items[lg], (size_t)items * sizeof(int2), "row block table"));
            AUG_TRY(aug::ring_reserve(ctx, aug::ring_bytes(n)));
        }
        blocks.begin = t.d_begin.as<int64_t>();
        blocks.end = t.d_end.as<int64_t>();
        blocks.first = whole ? nullptr : t.d_first[lg].as<int>();
        blocks.items = (whole ? t.orders[order].d_items : t.d_items[lg]).as<int2>();
        return AUG_OK;
    }

    int launch() {
        if (!new_table) return AUG_OK;
        aug::RowTables& t = aug::whole(ctx).rows;
        aug::HostRing& r = ctx->ring;
        const size_t n = (size_t)n_seq + 1, i64 = n * sizeof(int64_t);
        if (new_rows) {
            t.end.resize(n);
            t.begin.reserve(n);
        }
        const int slot = r.next;
        if (slot % aug::HostRing::kPerEvent == 0) AUG_HIP(hipEventSynchronize(r.done[slot / aug::HostRing::kPerEvent]), "staging event wait");
        unsigned char* const h = r.host + (size_t)slot * r.bytes;
        unsigned char* const d = r.device + (size_t)slot * r.bytes;
        const bool whole = blocks.lg == aug::kWholeLg;
        aug::RowTableArgs ta{};
        ta.n_seq = n_seq;
        ta.whole = whole;
        ta.d_begin = t.d_begin.as<int64_t>();
        ta.d_end = t.d_end.as<int64_t>();
        ta.d_first = whole ? nullptr : t.d_first[blocks.lg].as<int>();
        ta.items = (whole ? t.orders[order].d_items : t.d_items[blocks.lg]).as<int2>();
        if (new_rows) {
            memcpy(h, offsets, i64);
            for (int i = 0; i < n_seq; ++i) t.end[i] = end(i);
            t.end[n_seq] = offsets[n_seq];
            memcpy(h + i64, t.end.data(), i64);
            ta.begin = reinterpret_cast<const int64_t*>(d);
            ta.end = reinterpret_cast<const int64_t*>(d + i64);
        }
        int* const first = reinterpret_cast<int*>(h + 2 * i64);
        int at = 0;
        if (whole) {
            place(first, t.orders[order].abreast);
        } else {
            for (int i = 0; i < n_seq; ++i) {
                first[i] = at;
                at += (int)blocks_of(i, blocks.lg);
            }
            first[n_seq] = at;
        }
        ta.first = reinterpret_cast<const int*>(d + 2 * i64);
        AUG_HIP(aug::launch_row_tables(ctx->stream, ta), "row tables kernel");
        if (new_rows) t.begin.assign(offsets, offsets + n);
        if (whole) t.orders[order].there = true;
        else t.n_items[blocks.lg] = at;
        return aug::packing_launched(ctx);
    }

  private:
    // Places of whole sequences: the long ones first, `abreast` of them (0: all) side by side in turn forth and back, so that a compute
    // unit's sequences add up alike.  (64 sequences of 98 to 1598 rows in the order they came in: the unluckiest had half as many rows again as the mean.)
    void place(int* at, int abreast) const {
        if (!abreast) abreast = n_seq;
        std::vector<int> by_length(n_seq);
        for (int i = 0; i < n_seq; ++i) by_length[i] = i;
        std::sort(by_length.begin(), by_length.end(), [&](int i, int j) {
            const int64_t a = end(i) - offsets[i], b = end(j) - offsets[j];
            return a != b ? a > b : i < j;
        });
        for (int p = 0; p < n_seq; ++p) {
            const int turn = p / abreast, from = turn * abreast, to = std::min(from + abreast, n_seq);
            at[by_length[p]] = turn % 2 ? to - 1 - (p - from) : p;
        }
    }
    int64_t blocks_of(int i, int lg) const {
        const int64_t len = end(i) - offsets[i];
        return len > 0 ? (len + ((int64_t)1 << lg) - 1) >> lg : 1;
    }
};

// ---- checks of the three operators ----

int check_norm(aug_ctx* ctx, int64_t n_rows, const aug_norm_cfg* cfg) {
    if (!cfg) return fail(ctx, AUG_ERR_INVALID_ARG, "norm config is null");
    AUG_TRY(check_dtype(ctx, cfg->dtype));
    if (n_rows < 0) return fail(ctx, AUG_ERR_INVALID_ARG, "n_rows is negative");
    if (n_rows > ((int64_t)1 << 40)) return fail(ctx, AUG_ERR_UNSUPPORTED, "too many rows in one call");
    if (cfg->dim < 1) return fail(ctx, AUG_ERR_INVALID_ARG, "dim must be positive");
    if (cfg->dim > AUG_MAX_NORM_DIM) return fail(ctx, AUG_ERR_UNSUPPORTED, "dim is more than %d", AUG_MAX_NORM_DIM);
    return AUG_OK;
}

int check_short_conv(aug_ctx* ctx, const aug_short_conv_cfg* cfg) {
    if (!cfg) return fail(ctx, AUG_ERR_INVALID_ARG, "short convolution config is null");
    AUG_TRY(check_dtype(ctx, cfg->dtype));
    if (cfg->dim < 1 || cfg->taps < 1) return fail(ctx, AUG_ERR_INVALID_ARG, "dim and taps must be positive");
    if (cfg->dim > AUG_MAX_DIM || cfg->taps > AUG_MAX_TAPS)
        return fail(ctx, AUG_ERR_UNSUPPORTED, "more than %d channels or %d taps", AUG_MAX_DIM, AUG_MAX_TAPS);
    return AUG_OK;
}

int check_scan(aug_ctx* ctx, const aug_scan_cfg* cfg, const aug_scan_in* in, int64_t n_rows) {
    if (!cfg || !in) return fail(ctx, AUG_ERR_INVALID_ARG, "scan config or input is null");
    AUG_TRY(check_dtype(ctx, cfg->dtype));
    if (cfg->dim < 1 || cfg->n_state < 1 || cfg->n_group < 1) return fail(ctx, AUG_ERR_INVALID_ARG, "dim, n_state and n_group must be positive");
    if (cfg->dim > AUG_MAX_DIM || cfg->n_state > AUG_MAX_STATE)
        return fail(ctx, AUG_ERR_UNSUPPORTED, "more than %d channels or %d states", AUG_MAX_DIM, AUG_MAX_STATE);
    if (cfg->dim % cfg->n_group) return fail(ctx, AUG_ERR_INVALID_ARG, "n_group does not divide dim");
    const int64_t bc = (int64_t)cfg->n_group * cfg->n_state;
    AUG_TRY(check_rows(ctx, "u", &in->u, n_rows, cfg->dim, true));
    AUG_TRY(check_rows(ctx, "delta", &in->delta, n_rows, cfg->dim, true));
    AUG_TRY(check_rows(ctx, "b", &in->b, n_rows, bc, true));
    AUG_TRY(check_rows(ctx, "c", &in->c, n_rows, bc, true));
    AUG_TRY(check_rows(ctx, "z", &in->z, n_rows, cfg->dim, false));
    if (!in->a) return fail(ctx, AUG_ERR_INVALID_ARG, "a is null");
    return AUG_OK;
}

// The spans of the scan's inputs; the bits of u, delta and z.
int add_scan_in(Spans& sp, const aug_scan_cfg& cfg, const aug_scan_in& in, int64_t n_rows) {
    const int64_t e = element_bytes(cfg.dtype), w = cfg.dim * e, bc = (int64_t)cfg.n_group * cfg.n_state * e;
    int bits = sp.add("u", in.u.data, in.u.ld * e, w, n_rows, 0, 0);
    bits |= sp.add("delta", in.delta.data, in.delta.ld * e, w, n_rows, 0, 0);
    bits |= sp.add("z", in.z.data, in.z.ld * e, w, n_rows, 0, 0);
    sp.add("b", in.b.data, in.b.ld * e, bc, n_rows, 0, 0);
    sp.add("c", in.c.data, in.c.ld * e, bc, n_rows, 0, 0);
    sp.add("a", in.a, 0, 4 * (int64_t)cfg.dim * cfg.n_state, 1, 0, 0);
    sp.add("skip", in.skip, 0, 4 * (int64_t)cfg.dim, 1, 0, 0);
    sp.add("delta_bias", in.delta_bias, 0, 4 * (int64_t)cfg.dim, 1, 0, 0);
    return bits;
}

}  // namespace

extern "C" {

int aug_rms_norm_batch(aug_ctx* ctx, int64_t n_rows, const aug_norm_cfg* cfg, const aug_rows* x, const aug_rows* residual,
                       const float* weight, const aug_rows* sum_out, const aug_rows* y_out, const aug_rows* q_out,
                       float* scale_out, float* rstd_out) {
    return guarded(ctx, [&]() -> int {
        AUG_TRY(check_norm(ctx, n_rows, cfg));
        if (!(cfg->eps >= 0.f) || !std::isfinite(cfg->eps)) return fail(ctx, AUG_ERR_INVALID_ARG, "eps must be a number >= 0");
        const int qb = cfg->q_block;
        if (qb != 0 && (qb < 16 || qb > 512 || (qb & (qb - 1)))) return fail(ctx, AUG_ERR_INVALID_ARG, "q_block must be 0 or a power of two in 16..512");
        aug::NormArgs a{n_rows, *cfg, of(x), of(residual), of(sum_out), of(y_out), of(q_out), weight, scale_out, rstd_out};
        AUG_TRY(check_rows(ctx, "x", &a.x, n_rows, cfg->dim, true));
        AUG_TRY(check_rows(ctx, "residual", &a.residual, n_rows, cfg->dim, false));
        AUG_TRY(check_rows(ctx, "sum_out", &a.sum, n_rows, cfg->dim, false));
        AUG_TRY(check_rows(ctx, "y_out", &a.y, n_rows, cfg->dim, false));
        AUG_TRY(check_rows(ctx, "q_out", &a.q, n_rows, cfg->dim, false));
        if (a.q.data && !scale_out && n_rows > 0) return fail(ctx, AUG_ERR_INVALID_ARG, "q_out needs scale_out");
        if (n_rows == 0) return AUG_OK;
        const int64_t e = element_bytes(cfg->dtype), w = cfg->dim * e;
        const int64_t n_scales = qb ? (cfg->dim + qb - 1) / qb : 1;
        Spans sp;
        int in = sp.add("x", a.x.data, a.x.ld * e, w, n_rows, 0, 0);
        in |= sp.add("residual", a.residual.data, a.residual.ld * e, w, n_rows, 0, 0);
        sp.add("weight", weight, 0, 4 * (int64_t)cfg->dim, 1, 0, 0);
        sp.add("sum_out", a.sum.data, a.sum.ld * e, w, n_rows, 1, in);
        sp.add("y_out", a.y.data, a.y.ld * e, w, n_rows, 1, in);
        sp.add("q_out", a.q.data, a.q.ld, cfg->dim, n_rows, 1, 0);
        if (a.q.data) sp.add("scale_out", scale_out, 0, 4 * n_rows * n_scales, 1, 1, 0);
        sp.add("rstd_out", rstd_out, 0, 4 * n_rows, 1, 1, 0);
        AUG_TRY(sp.check(ctx));
        AUG_TRY(mark(ctx, -1));
        AUG_HIP(aug::launch_norm(ctx->stream, a, ctx->n_cu), "norm kernel");
        return mark(ctx, AUG_STAGE_NORM);
    });
}

int aug_rms_norm_backward_batch(aug_ctx* ctx, int64_t n_rows, const aug_norm_cfg* cfg, const aug_rows* sum, const float* weight,
                                const float* rstd, const aug_rows* dy, const aug_rows* dsum, const aug_rows* dx_out,
                                float* dweight_out) {
    return guarded(ctx, [&]() -> int {
        AUG_TRY(check_norm(ctx, n_rows, cfg));
        aug::NormBackArgs a{n_rows, cfg->dtype, cfg->dim, of(sum), of(dy), of(dsum), of(dx_out), weight, rstd, dweight_out, nullptr};
        AUG_TRY(check_rows(ctx, "sum", &a.sum, n_rows, cfg->dim, true));
        AUG_TRY(check_rows(ctx, "dy", &a.dy, n_rows, cfg->dim, true));
        AUG_TRY(check_rows(ctx, "dsum", &a.dsum, n_rows, cfg->dim, false));
        AUG_TRY(check_rows(ctx, "dx_out", &a.dx, n_rows, cfg->dim, false));
        if (!rstd && n_rows > 0) return fail(ctx, AUG_ERR_INVALID_ARG, "rstd is null");
        const int64_t e = element_bytes(cfg->dtype), w = cfg->dim * e;
        Spans sp;
        int in = sp.add("sum", a.sum.data, a.sum.ld * e, w, n_rows, 0, 0);
        in |= sp.add("dy", a.dy.data, a.dy.ld * e, w, n_rows, 0, 0);
        in |= sp.add("dsum", a.dsum.data, a.dsum.ld * e, w, n_rows, 0, 0);
        sp.add("weight", weight, 0, 4 * (int64_t)cfg->dim, 1, 0, 0);
        sp.add("rstd", rstd, 0, 4 * n_rows, 1, 0, 0);
        sp.add("dx_out", a.dx.data, a.dx.ld * e, w, n_rows, 1, in);
        sp.add("dweight_out", dweight_out, 0, 4 * (int64_t)cfg->dim, 1, 1, 0);
        AUG_TRY(sp.check(ctx));
        if (n_rows == 0) {
            if (dweight_out) AUG_HIP(aug::launch_sum_partials(ctx->stream, nullptr, 0, 0, {{{dweight_out, cfg->dim}, {}, {}}}), "gradient sum kernel");
            return AUG_OK;
        }
        if (!a.dx.data && !dweight_out) return AUG_OK;
        if (dweight_out) {
            AUG_TRY(grow(ctx, aug::whole(ctx).seq_ws, 4 * (size_t)aug::norm_partials(n_rows, cfg->dim, ctx->n_cu) * cfg->dim, "gradient workspace"));
            a.partial = aug::whole(ctx).seq_ws.as<float>();
        }
        AUG_TRY(mark(ctx, -1));
        AUG_HIP(aug::launch_norm_backward(ctx->stream, a, ctx->n_cu), "norm gradient kernels");
        return mark(ctx, AUG_STAGE_NORM);
    });
}

int aug_short_conv_batch(aug_ctx* ctx, int n_seq, const int64_t* row_offsets, const int64_t* row_lengths,
                         const aug_short_conv_cfg* cfg, const aug_rows* x, const float* weight, const float* bias,
                         const void* state_in, void* state_out, const aug_rows* y_out) {
    return guarded(ctx, [&]() -> int {
        AUG_TRY(check_sequences(ctx, n_seq, row_offsets, row_lengths));
        AUG_TRY(check_short_conv(ctx, cfg));
        Sequences seq(ctx, n_seq, row_offsets, row_lengths);
        aug::ShortConvArgs a{};
        a.cfg = *cfg;
        a.x = of(x);
        a.y = of(y_out);
        a.weight = weight;
        a.bias = bias;
        a.state_in = state_in;
        a.state_out = state_out;
        AUG_TRY(check_rows(ctx, "x", &a.x, seq.n_rows, cfg->dim, true));
        AUG_TRY(check_rows(ctx, "y_out", &a.y, seq.n_rows, cfg->dim, true));
        if (!weight) return fail(ctx, AUG_ERR_INVALID_ARG, "weight is null");
        const int64_t e = element_bytes(cfg->dtype), w = cfg->dim * e, held = (int64_t)n_seq * (cfg->taps - 1) * w;
        Spans sp;
        sp.add("x", a.x.data, a.x.ld * e, w, seq.n_rows, 0, 0);
        sp.add("weight", weight, 0, 4 * (int64_t)cfg->dim * cfg->taps, 1, 0, 0);
        sp.add("bias", bias, 0, 4 * (int64_t)cfg->dim, 1, 0, 0);
        const int st = sp.add("state_in", state_in, 0, held, 1, 0, 0);
        sp.add("state_out", state_out, 0, held, 1, 1, st);
        sp.add("y_out", a.y.data, a.y.ld * e, w, seq.n_rows, 1, 0);
        AUG_TRY(sp.check(ctx));
        if (n_seq == 0 || (seq.total == 0 && !state_out)) return AUG_OK;
        AUG_TRY(seq.plan(aug::short_conv_lg_block(*cfg, false), aug::short_conv_tiles(*cfg, false)));
        AUG_TRY(seq.launch());
        a.rows = seq.blocks;
        AUG_TRY(mark(ctx, -1));
        AUG_HIP(aug::launch_short_conv(ctx->stream, a), "short convolution kernel");
        return mark(ctx, AUG_STAGE_SHORT_CONV);
    });
}

int aug_short_conv_backward_batch(aug_ctx* ctx, int n_seq, const int64_t* row_offsets, const int64_t* row_lengths,
                                  const aug_short_conv_cfg* cfg, const aug_rows* x, const float* weight, const float* bias,
                                  const void* state_in, const aug_rows* dy, const aug_rows* dx_out, float* dweight_out,
                                  float* dbias_out) {
    return guarded(ctx, [&]() -> int {
        AUG_TRY(check_sequences(ctx, n_seq, row_offsets, row_lengths));
        AUG_TRY(check_short_conv(ctx, cfg));
        Sequences seq(ctx, n_seq, row_offsets, row_lengths);
        aug::ShortConvArgs a{};
        a.cfg = *cfg;
        a.x = of(x);
        a.dy = of(dy);
        a.dx = of(dx_out);
        a.weight = weight;
        a.bias = bias;
        a.state_in = state_in;
        a.dweight = dweight_out;
        a.dbias = dbias_out;
        AUG_TRY(check_rows(ctx, "x", &a.x, seq.n_rows, cfg->dim, true));
        AUG_TRY(check_rows(ctx, "dy", &a.dy, seq.n_rows, cfg->dim, true));
        AUG_TRY(check_rows(ctx, "dx_out", &a.dx, seq.n_rows, cfg->dim, false));
        if (!weight) return fail(ctx, AUG_ERR_INVALID_ARG, "weight is null");
        const int64_t e = element_bytes(cfg->dtype), w = cfg->dim * e;
        Spans sp;
        sp.add("x", a.x.data, a.x.ld * e, w, seq.n_rows, 0, 0);
        sp.add("dy", a.dy.data, a.dy.ld * e, w, seq.n_rows, 0, 0);
        sp.add("weight", weight, 0, 4 * (int64_t)cfg->dim * cfg->taps, 1, 0, 0);
        sp.add("bias", bias, 0, 4 * (int64_t)cfg->dim, 1, 0, 0);
        sp.add("state_in", state_in, 0, (int64_t)n_seq * (cfg->taps - 1) * w, 1, 0, 0);
        sp.add("dx_out", a.dx.data, a.dx.ld * e, w, seq.n_rows, 1, 0);
        sp.add("dweight_out", dweight_out, 0, 4 * (int64_t)cfg->dim * cfg->taps, 1, 1, 0);
        sp.add("dbias_out", dbias_out, 0, 4 * (int64_t)cfg->dim, 1, 1, 0);
        AUG_TRY(sp.check(ctx));
        if (!a.dx.data && !dweight_out && !dbias_out) return AUG_OK;
        if (seq.total == 0) {
            const aug::SumOuts zeros{{{dweight_out, (int64_t)cfg->dim * cfg->taps}, {dbias_out, cfg->dim}, {}}};
            AUG_HIP(aug::launch_sum_partials(ctx->stream, nullptr, 0, 0, zeros), "gradient sum kernel");
            return AUG_OK;
        }
        AUG_TRY(seq.plan(aug::short_conv_lg_block(*cfg, true), aug::short_conv_tiles(*cfg, true)));
        if (dweight_out || dbias_out) {
            const size_t n = (size_t)aug::short_conv_partials(*cfg, seq.blocks.n_items, ctx->n_cu);
            AUG_TRY(grow(ctx, aug::whole(ctx).seq_ws, 4 * n * cfg->dim * (cfg->taps + 1), "gradient workspace"));
            a.partial = aug::whole(ctx).seq_ws.as<float>();
        }
        AUG_TRY(seq.launch());
        a.rows = seq.blocks;
        AUG_TRY(mark(ctx, -1));
        AUG_HIP(aug::launch_short_conv_backward(ctx->stream, a, ctx->n_cu), "short convolution gradient kernels");
        return mark(ctx, AUG_STAGE_SHORT_CONV);
    });
}

int aug_short_conv_step(aug_ctx* ctx, int n_seq, const aug_short_conv_cfg* cfg, const aug_rows* x, const float* weight,
                        const float* bias, const void* state_in, void* state_out, const aug_rows* y_out) {
    return guarded(ctx, [&]() -> int {
        if (n_seq < 0) return fail(ctx, AUG_ERR_INVALID_ARG, "n_seq is negative");
        if (n_seq > AUG_MAX_UTT) return fail(ctx, AUG_ERR_UNSUPPORTED, "more than %d sequences in one call", AUG_MAX_UTT);
        AUG_TRY(check_short_conv(ctx, cfg));
        aug::ShortConvArgs a{};
        a.cfg = *cfg;
        a.x = of(x);
        a.y = of(y_out);
        a.weight = weight;
        a.bias = bias;
        a.state_in = state_in;
        a.state_out = state_out;
        AUG_TRY(check_rows(ctx, "x", &a.x, n_seq, cfg->dim, true));
        AUG_TRY(check_rows(ctx, "y_out", &a.y, n_seq, cfg->dim, true));
        if (!weight) return fail(ctx, AUG_ERR_INVALID_ARG, "weight is null");
        if (n_seq > 0 && cfg->taps > 1 && (!state_in || !state_out)) return fail(ctx, AUG_ERR_INVALID_ARG, "state_in or state_out is null");
        if (n_seq == 0) return AUG_OK;
        const int64_t e = element_bytes(cfg->dtype), w = cfg->dim * e, held = (int64_t)n_seq * (cfg->taps - 1) * w;
        Spans sp;
        const int in = sp.add("x", a.x.data, a.x.ld * e, w, n_seq, 0, 0);
        sp.add("weight", weight, 0, 4 * (int64_t)cfg->dim * cfg->taps, 1, 0, 0);
        sp.add("bias", bias, 0, 4 * (int64_t)cfg->dim, 1, 0, 0);
        const int st = sp.add("state_in", state_in, 0, held, 1, 0, 0);
        sp.add("state_out", state_out, 0, held, 1, 1, st);
        sp.add("y_out", a.y.data, a.y.ld * e, w, n_seq, 1, in);
        AUG_TRY(sp.check(ctx));
        AUG_TRY(mark(ctx, -1));
        AUG_HIP(aug::launch_short_conv_step(ctx->stream, n_seq, a), "short convolution kernel");
        return mark(ctx, AUG_STAGE_SHORT_CONV);
    });
}

int aug_scan_batch(aug_ctx* ctx, int n_seq, const int64_t* row_offsets, const int64_t* row_lengths, const aug_scan_cfg* cfg,
                   const aug_scan_in* in, const float* state_in, float* state_out, const aug_rows* y_out) {
    return guarded(ctx, [&]() -> int {
        AUG_TRY(check_sequences(ctx, n_seq, row_offsets, row_lengths));
        Sequences seq(ctx, n_seq, row_offsets, row_lengths);
        AUG_TRY(check_scan(ctx, cfg, in, seq.n_rows));
        aug::ScanArgs a{};
        a.cfg = *cfg;
        a.in = *in;
        a.y = of(y_out);
        a.state_in = state_in;
        a.state_out = state_out;
        AUG_TRY(check_rows(ctx, "y_out", &a.y, seq.n_rows, cfg->dim, true));
        const int64_t e = element_bytes(cfg->dtype), held = 4 * (int64_t)n_seq * cfg->dim * cfg->n_state;
        Spans sp;
        add_scan_in(sp, *cfg, *in, seq.n_rows);
        const int st = sp.add("state_in", state_in, 0, held, 1, 0, 0);
        sp.add("state_out", state_out, 0, held, 1, 1, st);
        sp.add("y_out", a.y.data, a.y.ld * e, cfg->dim * e, seq.n_rows, 1, 0);
        AUG_TRY(sp.check(ctx));
        if (n_seq == 0 || (seq.total == 0 && !state_out)) return AUG_OK;
        AUG_TRY(seq.plan(aug::scan_lg_block(*cfg, n_seq, row_offsets, row_lengths, ctx->n_cu, false), aug::scan_tiles(*cfg, false),
                         aug::scan_abreast(*cfg, ctx->n_cu)));
        if (seq.blocks.lg != aug::kWholeLg) {        // whole sequences need none
            AUG_TRY(grow(ctx, aug::whole(ctx).seq_ws, aug::scan_workspace(*cfg, seq.blocks.n_items, seq.n_rows, ctx->n_cu, false), "scan workspace"));
            a.ws = aug::whole(ctx).seq_ws.ptr;
        }
        AUG_TRY(seq.launch());
        a.rows = seq.blocks;
        AUG_TRY(mark(ctx, -1));
        AUG_HIP(aug::launch_scan(ctx->stream, a, ctx->n_cu), "scan kernels");
        return mark(ctx, AUG_STAGE_SCAN);
    });
}

int aug_scan_backward_batch(aug_ctx* ctx, int n_seq, const int64_t* row_offsets, const int64_t* row_lengths,
                            const aug_scan_cfg* cfg, const aug_scan_in* in, const float* state_in, const aug_rows* dy,
                            const aug_scan_grad* out) {
    return guarded(ctx, [&]() -> int {
        AUG_TRY(check_sequences(ctx, n_seq, row_offsets, row_lengths));
        Sequences seq(ctx, n_seq, row_offsets, row_lengths);
        AUG_TRY(check_scan(ctx, cfg, in, seq.n_rows));
        if (!out) return fail(ctx, AUG_ERR_INVALID_ARG, "the gradients' struct is null");
        aug::ScanArgs a{};
        a.cfg = *cfg;
        a.in = *in;
        a.dy = of(dy);
        a.state_in = state_in;
        a.grad = *out;
        const aug_scan_grad& g = a.grad;
        const int64_t bc = (int64_t)cfg->n_group * cfg->n_state, e = element_bytes(cfg->dtype);
        AUG_TRY(check_rows(ctx, "dy", &a.dy, seq.n_rows, cfg->dim, true));
        if (g.dz.data && !in->z.data) return fail(ctx, AUG_ERR_INVALID_ARG, "dz without a gate");
        const struct { const char* name; const aug_rows* m; int64_t width; } mats[] = {
            {"du", &g.du, cfg->dim}, {"ddelta", &g.ddelta, cfg->dim}, {"db", &g.db, bc}, {"dc", &g.dc, bc}, {"dz", &g.dz, cfg->dim}};
        Spans sp;
        add_scan_in(sp, *cfg, *in, seq.n_rows);
        sp.add("state_in", state_in, 0, 4 * (int64_t)n_seq * cfg->dim * cfg->n_state, 1, 0, 0);
        sp.add("dy", a.dy.data, a.dy.ld * e, cfg->dim * e, seq.n_rows, 0, 0);
        bool any = g.da || g.dskip || g.ddelta_bias;
        for (const auto& m : mats) {
            AUG_TRY(check_rows(ctx, m.name, m.m, seq.n_rows, m.width, false));
            sp.add(m.name, m.m->data, m.m->ld * e, m.width * e, seq.n_rows, 1, 0);
            any = any || m.m->data;
        }
        sp.add("da", g.da, 0, 4 * (int64_t)cfg->dim * cfg->n_state, 1, 1, 0);
        sp.add("dskip", g.dskip, 0, 4 * (int64_t)cfg->dim, 1, 1, 0);
        sp.add("ddelta_bias", g.ddelta_bias, 0, 4 * (int64_t)cfg->dim, 1, 1, 0);
        AUG_TRY(sp.check(ctx));
        if (!any) return AUG_OK;
        if (seq.total == 0) {
            const aug::SumOuts zeros{{{g.da, (int64_t)cfg->dim * cfg->n_state}, {g.dskip, cfg->dim}, {g.ddelta_bias, cfg->dim}}};
            AUG_HIP(aug::launch_sum_partials(ctx->stream, nullptr, 0, 0, zeros), "gradient sum kernel");
            return AUG_OK;
        }
        AUG_TRY(seq.plan(aug::scan_lg_block(*cfg, n_seq, row_offsets, row_lengths, ctx->n_cu, true), aug::scan_tiles(*cfg, true)));
        AUG_TRY(grow(ctx, aug::whole(ctx).seq_ws, aug::scan_workspace(*cfg, seq.blocks.n_items, seq.n_rows, ctx->n_cu, true), "scan workspace"));
        a.ws = aug::whole(ctx).seq_ws.ptr;
        AUG_TRY(seq.launch());
        a.rows = seq.blocks;
        AUG_TRY(mark(ctx, -1));
        AUG_HIP(aug::launch_scan_backward(ctx->stream, a, seq.n_rows, ctx->n_cu), "scan gradient kernels");
        return mark(ctx, AUG_STAGE_SCAN);
    });
}

int aug_scan_step(aug_ctx* ctx, int n_seq, const aug_scan_cfg* cfg, const aug_scan_in* in, const float* state_in,
                  float* state_out, const aug_rows* y_out) {
    return guarded(ctx, [&]() -> int {
        if (n_seq < 0) return fail(ctx, AUG_ERR_INVALID_ARG, "n_seq is negative");
        if (n_seq > AUG_MAX_UTT) return fail(ctx, AUG_ERR_UNSUPPORTED, "more than %d sequences in one call", AUG_MAX_UTT);
        AUG_TRY(check_scan(ctx, cfg, in, n_seq));
        aug::ScanArgs a{};
        a.cfg = *cfg;
        a.in = *in;
        a.y = of(y_out);
        a.state_in = state_in;
        a.state_out = state_out;
        AUG_TRY(check_rows(ctx, "y_out", &a.y, n_seq, cfg->dim, true));
        if (n_seq == 0) return AUG_OK;
        if (!state_in || !state_out) return fail(ctx, AUG_ERR_INVALID_ARG, "state_in or state_out is null");
        const int64_t e = element_bytes(cfg->dtype), held = 4 * (int64_t)n_seq * cfg->dim * cfg->n_state;
        Spans sp;
        const int bits = add_scan_in(sp, *cfg, *in, n_seq);
        const int st = sp.add("state_in", state_in, 0, held, 1, 0, 0);
        sp.add("state_out", state_out, 0, held, 1, 1, st);
        sp.add("y_out", a.y.data, a.y.ld * e, cfg->dim * e, n_seq, 1, bits);
        AUG_TRY(sp.check(ctx));
        AUG_TRY(mark(ctx, -1));
        AUG_HIP(aug::launch_scan_step(ctx->stream, n_seq, a, ctx->n_cu), "scan kernel");
        return mark(ctx, AUG_STAGE_SCAN);
    });
}

}  // extern "C"
