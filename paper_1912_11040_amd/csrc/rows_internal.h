// The operators on feature rows: what the C ABI hands to their launchers (which check nothing).
#pragma once

#include "aug_internal.h"

namespace aug {

// The sequences of the last call on feature rows and, per power of two of rows, the table that cuts them into blocks of so many
// (an empty sequence has one block).  Kept apart from Packing: a step of training alternates between the two.
struct RowTables {
    std::vector<int64_t> begin;          // n_seq + 1, as given
    std::vector<int64_t> end;            // n_seq + 1: end of each sequence (the last entry counts for nothing)
    static constexpr int kTables = 30;   // blocks of 1 .. 2^29 rows
    int n_items[kTables] = {};           // blocks; 0: the table is not there
    DeviceBuffer d_begin, d_end;         // int64 [n_seq+1]
    DeviceBuffer d_first[kTables];       // int [n_seq+1]: blocks of the sequences before i
    DeviceBuffer d_items[kTables];       // int2 [n_items]: (sequence, block of it)
    // Whole sequences: a table per number of them that calls take side by side (0: all of them), which its order depends on.
    struct Order {
        int abreast = 0;
        bool there = false;
        DeviceBuffer d_items;            // int2 [n_seq]
    };
    std::vector<Order> orders;
    void forget() {
        begin.clear();
        for (int& n : n_items) n = 0;
        for (Order& o : orders) o.there = false;
    }
};

// What aug_create makes: the waveform path's context with the row operators' share of it.
struct Context : aug_ctx {
    RowTables rows;
    DeviceBuffer seq_ws;                 // partial sums of gradients; states and sums per block of the scan
};
inline Context& whole(aug_ctx* ctx) { return *static_cast<Context*>(ctx); }

// The sequences of a call, cut into blocks of 1 << lg rows.
struct RowBlocks {
    int n_seq = 0, lg = 0, n_items = 0;
    const int64_t* begin = nullptr;      // device [n_seq+1]
    const int64_t* end = nullptr;        // device [n_seq+1]
    const int* first = nullptr;          // device [n_seq+1]: blocks of the sequences before i
    const int2* items = nullptr;         // device [n_items]: (sequence, block of it)
};

constexpr int kWholeLg = RowTables::kTables;      // blocks of whole sequences, which are shorter than 2^30 rows

// The device's tables of a batch of sequences from what the host left in pinned memory: begin and end (null: they are there already)
// and the exclusive prefix sum of the blocks, n_seq + 1 entries each.  With `whole`, a block per sequence, `first` gives instead the
// place of each sequence in the table of blocks.
struct RowTableArgs {
    int n_seq;
    bool whole;
    const int64_t *begin, *end;
    const int* first;
    int64_t *d_begin, *d_end;
    int* d_first;
    int2* items;
};
hipError_t launch_row_tables(hipStream_t s, const RowTableArgs& a);

// Sums of the columns of partial [n_partial][stride] into up to three arrays that follow one another in a row of it (null: not wanted).
// The terms of a column are added in an order that depends on n_partial only.
struct SumOuts {
    struct Out {
        float* out;
        int64_t width;
    } part[3];
};
hipError_t launch_sum_partials(hipStream_t s, const float* partial, int n_partial, int64_t stride, const SumOuts& outs);

struct NormArgs {
    int64_t n_rows;
    aug_norm_cfg cfg;
    aug_rows x, residual, sum, y, q;     // data null: not there
    const float* weight;
    float* scale;
    float* rstd;
};
hipError_t launch_norm(hipStream_t s, const NormArgs& a, int n_cu);

struct NormBackArgs {
    int64_t n_rows;
    int dtype, dim;
    aug_rows sum, dy, dsum, dx;
    const float* weight;
    const float* rstd;
    float* dweight;
    float* partial;                      // [norm_partials][dim], used with dweight
};
int norm_partials(int64_t n_rows, int dim, int n_cu);
hipError_t launch_norm_backward(hipStream_t s, const NormBackArgs& a, int n_cu);

struct ShortConvArgs {
    RowBlocks rows;
    aug_short_conv_cfg cfg;
    aug_rows x, y;
    const float* weight;
    const float* bias;
    const void* state_in;
    void* state_out;
    // gradients
    aug_rows dy, dx;
    float* dweight;
    float* dbias;
    float* partial;                      // [short_conv_partials][dim * (taps + 1)]: by the weight, then by the bias
};
int short_conv_tiles(const aug_short_conv_cfg& cfg, bool backward);            // groups of threads across a row
int short_conv_lg_block(const aug_short_conv_cfg& cfg, bool backward);       // rows of a block, as a power of two
int short_conv_partials(const aug_short_conv_cfg& cfg, int n_items, int n_cu);
hipError_t launch_short_conv(hipStream_t s, const ShortConvArgs& a);
hipError_t launch_short_conv_backward(hipStream_t s, const ShortConvArgs& a, int n_cu);
hipError_t launch_short_conv_step(hipStream_t s, int n_seq, const ShortConvArgs& a);

struct ScanArgs {
    RowBlocks rows;
    aug_scan_cfg cfg;
    aug_scan_in in;
    const float* state_in;
    float* state_out;
    aug_rows y;
    // gradients
    aug_rows dy;
    aug_scan_grad grad;
    void* ws;
};
// Rows of a block as a power of two, kWholeLg: sequences are not cut; of those, how many a row of work groups across the chip takes.
int scan_lg_block(const aug_scan_cfg& cfg, int n_seq, const int64_t* begin, const int64_t* lengths, int n_cu, bool backward);
int scan_tiles(const aug_scan_cfg& cfg, bool backward);      // groups of threads across a row
int scan_abreast(const aug_scan_cfg& cfg, int n_cu);
size_t scan_workspace(const aug_scan_cfg& cfg, int n_items, int64_t n_rows, int n_cu, bool backward);     // bytes
hipError_t launch_scan(hipStream_t s, const ScanArgs& a, int n_cu);
hipError_t launch_scan_backward(hipStream_t s, const ScanArgs& a, int64_t n_rows, int n_cu);
hipError_t launch_scan_step(hipStream_t s, int n_seq, const ScanArgs& a, int n_cu);

}  // namespace aug
