// What the operators on feature rows share: the tables that cut sequences into blocks, and sums of partial sums.

#include "rows_internal.h"

namespace aug {
namespace {

// Threads per sequence, as for the packing of utterances: more when one sequence may own all the blocks.
__host__ __device__ inline int lanes_per_sequence(int n_seq) { return n_seq < 32 ? 256 : 16; }

__global__ __launch_bounds__(256) void row_tables_kernel(RowTableArgs a) {
    const int lanes = lanes_per_sequence(a.n_seq), at = blockIdx.x * 256 + threadIdx.x, i = at / lanes, l = at % lanes;
    if (i > a.n_seq) return;
    if (l == 0 && a.begin) {
        a.d_begin[i] = a.begin[i];
        a.d_end[i] = a.end[i];
    }
    if (a.whole) {
        if (l == 0 && i < a.n_seq) a.items[a.first[i]] = make_int2(i, 0);
        return;
    }
    const int from = a.first[i];
    if (l == 0) a.d_first[i] = from;
    if (i == a.n_seq) return;
    for (int j = l; j < a.first[i + 1] - from; j += lanes) a.items[from + j] = make_int2(i, j);
}

// Sixteen columns to a group, every sixteenth row a lane's, eight rows' loads on their way at once: few columns of many rows are bound by
// latency (512 rows of 1001: 64 columns and four rows side by side took 12 us, so 5; one row after another 38 for 128 rows).
constexpr int kColumns = 16, kAbreast = 16;
__global__ __launch_bounds__(kColumns * kAbreast) void sum_partials_kernel(const float* partial, int n_partial, int64_t stride, SumOuts outs) {
    __shared__ float part[kAbreast][kColumns];
    const int lane = threadIdx.x % kColumns, group = threadIdx.x / kColumns;
    const int64_t c = (int64_t)blockIdx.x * kColumns + lane, width = outs.part[0].width + outs.part[1].width + outs.part[2].width;
    constexpr int kAhead = 8;
    float acc = 0.f;
    for (int p = group; p < n_partial; p += kAbreast * kAhead) {
        float v[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) v[j] = c < width && p + kAbreast * j < n_partial ? partial[(int64_t)(p + kAbreast * j) * stride + c] : 0.f;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) acc += v[j];
    }
    part[group][lane] = acc;
    __syncthreads();
    if (group || c >= width) return;
    float sum = 0.f;
#pragma unroll
    for (int g = 0; g < kAbreast; ++g) sum += part[g][lane];
    int64_t at = c;
    for (const SumOuts::Out& o : outs.part) {
        if (at >= 0 && at < o.width && o.out) o.out[at] = sum;
        at -= o.width;
    }
}

}  // namespace

hipError_t launch_row_tables(hipStream_t s, const RowTableArgs& a) {
    const int64_t threads = ((int64_t)a.n_seq + 1) * lanes_per_sequence(a.n_seq);
    row_tables_kernel<<<dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_sum_partials(hipStream_t s, const float* partial, int n_partial, int64_t stride, const SumOuts& outs) {
    const int64_t width = outs.part[0].width + outs.part[1].width + outs.part[2].width;
    if (width <= 0) return hipSuccess;
    sum_partials_kernel<<<dim3((unsigned)((width + kColumns - 1) / kColumns)), dim3(kColumns * kAbreast), 0, s>>>(partial, n_partial, stride, outs);
    return hipGetLastError();
}

}  // namespace aug
