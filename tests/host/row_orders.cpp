// The order in which whole sequences are taken, on the host runtime of out_of_memory.cpp: it is that of the number of sequences that the call
// takes side by side, whatever calls came before it, and a call whose order is there builds none.  Built by test_row_orders.py.
#define main out_of_memory_main
#include "out_of_memory.cpp"
#undef main
#include "../../paper_1912_11040_amd/csrc/rows_api.hip"

static int g_tables = 0, g_launches = 0;
static std::vector<int> g_order;         // of the last scan's sequences

extern "C" hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }

namespace aug {
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
hipError_t launch_sum_partials(hipStream_t, const float*, int, int64_t, const SumOuts&) { return hipSuccess; }
hipError_t launch_norm(hipStream_t, const NormArgs&, int) { return hipSuccess; }
int norm_partials(int64_t, int, int) { return 1; }
hipError_t launch_norm_backward(hipStream_t, const NormBackArgs&, int) { return hipSuccess; }
int short_conv_tiles(const aug_short_conv_cfg&, bool) { return 1; }
int short_conv_lg_block(const aug_short_conv_cfg&, bool) { return 6; }
int short_conv_partials(const aug_short_conv_cfg&, int n, int) { return n; }
hipError_t launch_short_conv(hipStream_t, const ShortConvArgs&) { return hipSuccess; }
hipError_t launch_short_conv_backward(hipStream_t, const ShortConvArgs&, int) { return hipSuccess; }
hipError_t launch_short_conv_step(hipStream_t, int, const ShortConvArgs&) { return hipSuccess; }
int scan_tiles(const aug_scan_cfg&, bool) { return 1; }
int scan_abreast(const aug_scan_cfg& c, int) { return c.dim; }       // what the tests vary
int scan_lg_block(const aug_scan_cfg& c, int, const int64_t*, const int64_t*, int, bool backward) { return backward || c.n_state > 16 ? 5 : kWholeLg; }
size_t scan_workspace(const aug_scan_cfg&, int, int64_t, int, bool) { return 64; }
hipError_t launch_scan(hipStream_t, const ScanArgs& a, int) {
    ++g_launches;
    g_order.clear();
    for (int i = 0; i < a.rows.n_items; ++i) g_order.push_back(a.rows.items[i].x);
    return hipSuccess;
}
hipError_t launch_scan_backward(hipStream_t, const ScanArgs&, int64_t, int) { return hipSuccess; }
hipError_t launch_scan_step(hipStream_t, int, const ScanArgs&, int) { return hipSuccess; }
}  // namespace aug

static char* place(int i) { return reinterpret_cast<char*>((uintptr_t)(i + 1) << 44); }

// By length, the longest first, equal ones as they came, every second `abreast` of them backwards.
static std::vector<int> expected(const std::vector<int64_t>& off, int abreast) {
    const int n = (int)off.size() - 1;
    std::vector<int> v;
    for (int i = 0; i < n; ++i) v.push_back(i);
    std::stable_sort(v.begin(), v.end(), [&](int i, int j) { return off[i + 1] - off[i] > off[j + 1] - off[j]; });
    for (int from = abreast; from < n; from += 2 * abreast) std::reverse(v.begin() + from, v.begin() + std::min(from + abreast, n));
    return v;
}

int main() {
    const std::vector<int64_t> a{0, 7, 7, 40, 45, 46, 99, 106, 130}, b{0, 30, 31, 90, 90, 91, 97};
    aug_ctx* ctx = nullptr;
    EXPECT(aug_create(&ctx, 0, nullptr) == AUG_OK);
    auto scan = [&](const std::vector<int64_t>& off, int abreast, int n_state = 16) {
        const aug_scan_cfg c{AUG_F32, abreast, n_state, 1, 1};
        auto m = [](int i) { return aug_rows{place(i), 4096}; };
        const aug_scan_in in{m(0), m(1), m(2), m(3), m(4), reinterpret_cast<float*>(place(5)), nullptr, nullptr};
        const aug_rows y = m(8);
        const int rc = aug_scan_batch(ctx, (int)off.size() - 1, off.data(), nullptr, &c, &in, nullptr, nullptr, &y);
        if (rc != AUG_OK) { ++g_faults; printf("%s\n", aug_last_error(ctx)); }
    };
    for (int turn = 0; turn < 3; ++turn)
        for (const auto* off : {&a, &b}) {
            for (int abreast : {3, 2, 1, 100, 3, 2, 8, 100}) {
                scan(*off, abreast);
                EXPECT(g_order == expected(*off, abreast));
            }
            const int t = g_tables;
            for (int abreast : {2, 100, 1, 3}) scan(*off, abreast);
            EXPECT(g_tables == t);                       // each number's order is still there
            scan(*off, 3, 32);                           // in blocks between them
            scan(*off, 2);
            EXPECT(g_order == expected(*off, 2) && g_tables == t + 1);
        }
    // an order whose memory is not there leaves the others as they were
    scan(a, 3);
    g_until_failure = 0;
    {
        const aug_scan_cfg c{AUG_F32, 5, 16, 1, 1};
        auto m = [](int i) { return aug_rows{place(i), 4096}; };
        const aug_scan_in in{m(0), m(1), m(2), m(3), m(4), reinterpret_cast<float*>(place(5)), nullptr, nullptr};
        const aug_rows y = m(8);
        EXPECT(aug_scan_batch(ctx, 8, a.data(), nullptr, &c, &in, nullptr, nullptr, &y) == AUG_ERR_NOMEM);
    }
    g_until_failure = -1;
    const int t = g_tables;
    scan(a, 3);
    EXPECT(g_order == expected(a, 3) && g_tables == t);
    scan(a, 5);
    EXPECT(g_order == expected(a, 5) && g_tables == t + 1);
    aug_destroy(ctx);
    printf("%d scans, %d tables, %d faults\n", g_launches, g_tables, g_faults);
    return g_faults != 0;
}
