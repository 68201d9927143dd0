// The bias of every offset on a grid from a table by buckets of distance, and
// the table's gradient.
//
//   bias[h][dy][dx] = table[h][by(dy)][bx(dx)],  dtable[h][a][b] = the sum of dbias where by = a, bx = b
//
// The offsets of a bucket are a run along either axis (the edges rise, and the
// middle bucket lies around 0), so a cell of the table is a rectangle of the
// plane.  Forward: a block writes one row of the plane of some heads; bound by
// its writes.  Backward: a wave sums the runs of one row, a second kernel the
// rows of each cell; every sum has a fixed order.
//
// Measured, replayed from a graph: 8 heads of 64 x 64, bf16, 3.1 us for 258 KB;
// 16 of 128 x 128, fp32, 6.3 us for 4.2 MB and 9.0 backward in two launches: the
// launches bound them (alone in a trace the first takes 3.9 us, the last two 9.9).

#include "scram_rows.h"

namespace scram {
namespace {

struct BiasParams {
    const void* from;
    void* to;
    float* rows;  // [heads, 2 H - 1, nx] sums of the runs of each row
    int heads, H, W;
    int my, mx;
    int ey[SCRAM_BIAS_MAX_EDGES], ex[SCRAM_BIAS_MAX_EDGES];
};

// #{k : e_k <= t}
__device__ __forceinline__ int edges_up_to(const int* e, int m, int t)
{
    int lo = 0, hi = m;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (e[mid] <= t) lo = mid + 1; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int bucket_of(const int* e, int m, int t)
{
    const int k = edges_up_to(e, m, t < 0 ? -t : t);
    return t < 0 ? m - k : m + k;
}

// First and last offset of bucket b (an axis of 2 n - 1 offsets); last < first: none.
__device__ __forceinline__ void bucket_run(const int* e, int m, int n, int b, int& first, int& last)
{
    if (b == m) {
        last = (m ? min(e[0], n) : n) - 1;
        first = -last;
        return;
    }
    const int k = b < m ? m - b : b - m;                      // edges up to its distances: e[k - 1] ..
    const int near = e[k - 1], far = min(k < m ? e[k] : n, n) - 1;
    first = b < m ? -far : near;
    last = b < m ? -near : far;
}

template <typename T>
__global__ __launch_bounds__(kBlock) void relative_bias_kernel(BiasParams p)
{
    __shared__ int ex[SCRAM_BIAS_MAX_EDGES];
    if (static_cast<int>(threadIdx.x) < p.mx) ex[threadIdx.x] = p.ex[threadIdx.x];
    __syncthreads();
    const int ny = 2 * p.my + 1, nx = 2 * p.mx + 1;
    const int64_t height = 2 * int64_t(p.H) - 1, width = 2 * int64_t(p.W) - 1;
    for (int64_t row = blockIdx.x; row < height; row += gridDim.x) {
        const int by = bucket_of(p.ey, p.my, static_cast<int>(row) - p.H + 1);
        for (int64_t x = threadIdx.x; x < width; x += kBlock) {
            const int bx = bucket_of(ex, p.mx, static_cast<int>(x) - p.W + 1);
            const T* from = static_cast<const T*>(p.from) + by * nx + bx;
            T* to = static_cast<T*>(p.to) + row * width + x;
            for (int h = blockIdx.y; h < p.heads; h += gridDim.y)
                to[h * height * width] = from[static_cast<int64_t>(h) * ny * nx];
        }
    }
}

// A wave takes a row of the plane: eight lanes a bucket.
template <typename T>
__global__ __launch_bounds__(kBlock) void relative_rows_kernel(BiasParams p)
{
    __shared__ int ex[SCRAM_BIAS_MAX_EDGES];
    if (static_cast<int>(threadIdx.x) < p.mx) ex[threadIdx.x] = p.ex[threadIdx.x];
    __syncthreads();
    const int nx = 2 * p.mx + 1, lane = threadIdx.x & 7;
    const int64_t height = 2 * int64_t(p.H) - 1, width = 2 * int64_t(p.W) - 1, all = height * p.heads;
    for (int64_t row = blockIdx.x * 4ll + (threadIdx.x >> 6); row < all; row += gridDim.x * 4ll) {
        const T* const from = static_cast<const T*>(p.from) + row * width + p.W - 1;
        for (int b = (threadIdx.x & 63) >> 3; b < nx; b += 8) {
            int first, last;
            bucket_run(ex, p.mx, p.W, b, first, last);
            float x = 0.f;
            for (int64_t i = static_cast<int64_t>(first) + lane; i <= last; i += 8) x += to_float(from[i]);
            for (int m = 1; m < 8; m <<= 1) x += __shfl_xor(x, m);
            if (lane == 0) p.rows[row * nx + b] = x;
        }
    }
}

// A thread of 16 takes a share of the rows of one cell's column.
template <typename T>
__global__ __launch_bounds__(kBlock) void relative_cells_kernel(BiasParams p)
{
    const int ny = 2 * p.my + 1, nx = 2 * p.mx + 1, lane = threadIdx.x & 15;
    const int64_t height = 2 * int64_t(p.H) - 1, all = static_cast<int64_t>(p.heads) * ny * nx;
    for (int64_t cell = blockIdx.x * 16ll + (threadIdx.x >> 4); cell < all; cell += gridDim.x * 16ll) {
        const int64_t h = cell / (ny * nx);
        const int a = static_cast<int>(cell / nx % ny), b = static_cast<int>(cell % nx);
        int first, last;
        bucket_run(p.ey, p.my, p.H, a, first, last);
        const float* const from = p.rows + (h * height + p.H - 1) * nx + b;
        float x = 0.f;
        for (int64_t i = static_cast<int64_t>(first) + lane; i <= last; i += 16) x += from[i * nx];
        for (int m = 1; m < 16; m <<= 1) x += __shfl_xor(x, m);
        if (lane == 0) static_cast<T*>(p.to)[cell] = from_float<T>(x);
    }
}

BiasParams bias_params(const BiasCall& c)
{
    BiasParams p{};
    p.heads = c.heads;
    p.H = c.H;
    p.W = c.W;
    p.my = c.edges[0];
    p.mx = c.edges[1];
    for (int k = 0; k < p.my; ++k) p.ey[k] = c.edge[0][k];
    for (int k = 0; k < p.mx; ++k) p.ex[k] = c.edge[1][k];
    return p;
}

}  // namespace

hipError_t launch_relative_bias(const BiasCall& c, const void* table, void* bias, hipStream_t stream)
{
    BiasParams p = bias_params(c);
    p.from = table;
    p.to = bias;
    const int64_t height = 2 * int64_t(c.H) - 1;
    const uint32_t rows = static_cast<uint32_t>(height < (1 << 16) ? height : 1 << 16);
    const dim3 grid(rows, static_cast<uint32_t>(c.heads < 64 ? c.heads : 64));
    if (c.dtype == SCRAM_BF16)
        hipLaunchKernelGGL(relative_bias_kernel<uint16_t>, grid, dim3(kBlock), 0, stream, p);
    else
        hipLaunchKernelGGL(relative_bias_kernel<float>, grid, dim3(kBlock), 0, stream, p);
    return hipGetLastError();
}

size_t relative_bias_backward_workspace_bytes(const BiasCall& c)
{
    return size_t(c.heads) * (2 * size_t(c.H) - 1) * (2 * size_t(c.edges[1]) + 1) * sizeof(float);
}

hipError_t launch_relative_bias_backward(const BiasCall& c, const void* dbias, void* dtable, void* workspace, hipStream_t stream)
{
    BiasParams p = bias_params(c);
    p.from = dbias;
    p.to = dtable;
    p.rows = static_cast<float*>(workspace);
    const int64_t rows = (2 * int64_t(c.H) - 1) * c.heads, cells = int64_t(c.heads) * (2 * p.my + 1) * (2 * p.mx + 1);
    auto blocks = [](int64_t n) { return dim3(static_cast<uint32_t>(n < (1 << 20) ? n : 1 << 20)); };
    auto run = [&](auto type) {
        using T = decltype(type);
        hipLaunchKernelGGL(relative_rows_kernel<T>, blocks((rows + 3) / 4), dim3(kBlock), 0, stream, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(relative_cells_kernel<T>, blocks((cells + 15) / 16), dim3(kBlock), 0, stream, p);
        return hipGetLastError();
    };
    return c.dtype == SCRAM_BF16 ? run(uint16_t{}) : run(float{});
}

}  // namespace scram
