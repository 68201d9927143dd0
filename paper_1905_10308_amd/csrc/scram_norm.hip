// Layer norm of rows of C channels, forward and backward.
//
//   mu = mean x, r = (mean (x - mu)^2 + eps)^-1/2, xh = (x - mu) r, y = xh w + b
//   g = dy w:  dx = r (g - mean g - xh mean(g xh)),  dw = sum_rows dy xh,  db = sum_rows dy
//
// A row stays in registers between its passes, so every input is read once:
// bound by memory.  A row is held by `lanes` threads (a power of two), V
// neighbouring channels a chunk and up to 16 channels a thread; several rows
// share a wave, or several waves a row.  Sums are fp32: the two of the forward
// pass are of the row and then of its centred values, so that a row's offset
// costs no accuracy.
//
// The weights' gradients: a block keeps those of its rows in registers,
// adds them up over its threads once at its end and writes one row of parts;
// a second kernel adds up the parts, in a fixed order.

#include "scram_device.h"

namespace scram {
namespace {

constexpr int kNormThreads = 1024;  // most threads of a block
constexpr int kPerThread = 16;      // most channels of a thread

struct NormParams {
    const void* X;
    const void* dY;
    const void* weight;  // nullable
    const void* bias;    // nullable
    int weight_f32;
    void* out;           // Y or dX
    const float* mean_in;
    const float* rstd_in;
    float* mean;         // nullable
    float* rstd;
    float* parts;        // [blocks, 2, C]
    int64_t rows;
    int C, lanes;
    float eps;
};

template <typename T, int V>
using vec = T __attribute__((ext_vector_type(V)));

template <typename T>
__device__ __forceinline__ float norm_float(T x)
{
    if constexpr (std::is_same<T, float>::value)
        return x;
    else
        return __uint_as_float(static_cast<uint32_t>(x) << 16);
}

template <typename T>
__device__ __forceinline__ T norm_round(float x)
{
    if constexpr (std::is_same<T, float>::value)
        return x;
    else
        return static_cast<T>(f32_to_bf16_rne(x));
}

// Element i of a weight vector of either type.
__device__ __forceinline__ float norm_weight(const void* w, int f32, int i)
{
    return f32 ? static_cast<const float*>(w)[i] : norm_float(static_cast<const uint16_t*>(w)[i]);
}

// Sums of N values over the `lanes` threads of a row, on all of them.  Rows of several waves pass through LDS, in one of
// two halves in turn so that one barrier per sum is enough.
template <int N, bool WIDE>
__device__ __forceinline__ void row_sum(float (&x)[N], int lanes, float (*lds)[kNormThreads / 64][N], int& half)
{
    for (int m = 1; m < (WIDE ? 64 : lanes); m <<= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += __shfl_xor(x[i], m);
    if constexpr (WIDE) {
        const int wave = threadIdx.x >> 6, waves = lanes >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) lds[half][wave][i] = x[i];
        __syncthreads();
        const int w0 = wave & ~(waves - 1);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = lds[half][w0][i];
        for (int w = 1; w < waves; ++w)
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] += lds[half][w0 + w][i];
        half ^= 1;
    }
}

// Every thread of a block takes part in every row of its loop (the sums of wide rows hold barriers); rows past the end
// are neither read nor written.
template <typename T, int V, int NC, bool WIDE>
__global__ __launch_bounds__(WIDE ? kNormThreads : kBlock) void norm_kernel(NormParams p)
{
    using Vec = vec<T, V>;
    __shared__ float s_sum[2][kNormThreads / 64][1];
    int half = 0;
    const int lane = threadIdx.x & (p.lanes - 1);
    const int slots = blockDim.x / p.lanes, slot = threadIdx.x / p.lanes;
    const int chunks = p.C / V;
    const float inv_c = 1.f / static_cast<float>(p.C);
    float w[NC][V], b[NC][V];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int at = min(lane + c * p.lanes, chunks - 1) * V + j;
            w[c][j] = p.weight ? norm_weight(p.weight, p.weight_f32, at) : 1.f;
            b[c][j] = p.bias ? norm_weight(p.bias, p.weight_f32, at) : 0.f;
        }
    for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * slots; r0 < p.rows; r0 += static_cast<int64_t>(gridDim.x) * slots) {
        const int64_t row = r0 + slot;
        const bool live = row < p.rows;
        const T* const x = static_cast<const T*>(p.X) + row * p.C;
        float v[NC][V];
        float sum[1] = {0.f};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = lane + c * p.lanes;
            Vec a = {};
            if (live && at < chunks) a = reinterpret_cast<const Vec*>(x)[at];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                v[c][j] = norm_float(static_cast<T>(a[j]));
                sum[0] += v[c][j];
            }
        }
        row_sum<1, WIDE>(sum, p.lanes, s_sum, half);
        const float mean = sum[0] * inv_c;
        sum[0] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const bool in = lane + c * p.lanes < chunks;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                v[c][j] -= mean;
                sum[0] = in ? fmaf(v[c][j], v[c][j], sum[0]) : sum[0];
            }
        }
        row_sum<1, WIDE>(sum, p.lanes, s_sum, half);
        const float rstd = 1.f / sqrtf(sum[0] * inv_c + p.eps);
        if (!live) continue;
        T* const y = static_cast<T*>(p.out) + row * p.C;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = lane + c * p.lanes;
            Vec a;
#pragma unroll
            for (int j = 0; j < V; ++j) a[j] = norm_round<T>(fmaf(v[c][j] * rstd, w[c][j], b[c][j]));
            if (at < chunks) reinterpret_cast<Vec*>(y)[at] = a;
        }
        if (lane == 0 && p.mean) {
            p.mean[row] = mean;
            p.rstd[row] = rstd;
        }
    }
}

template <typename T, typename TG, int V, int NC, bool WIDE>
__global__ __launch_bounds__(WIDE ? kNormThreads : kBlock) void norm_backward_kernel(NormParams p)
{
    using Vec = vec<T, V>;
    using VecG = vec<TG, V>;
    __shared__ float s_sum[2][kNormThreads / 64][2];
    __shared__ float s_part[WIDE ? kNormThreads : kBlock];
    int half = 0;
    const int lane = threadIdx.x & (p.lanes - 1);
    const int slots = blockDim.x / p.lanes, slot = threadIdx.x / p.lanes;
    const int chunks = p.C / V;
    const float inv_c = 1.f / static_cast<float>(p.C);
    float w[NC][V], dw[NC][V], db[NC][V];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int at = min(lane + c * p.lanes, chunks - 1) * V + j;
            w[c][j] = p.weight ? norm_weight(p.weight, p.weight_f32, at) : 1.f;
            dw[c][j] = db[c][j] = 0.f;
        }
    for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * slots; r0 < p.rows; r0 += static_cast<int64_t>(gridDim.x) * slots) {
        const int64_t row = r0 + slot;
        const bool live = row < p.rows;
        float xh[NC][V], g[NC][V];
        float sum[2] = {0.f, 0.f};
        const float mean = live ? p.mean_in[row] : 0.f, rstd = live ? p.rstd_in[row] : 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = lane + c * p.lanes;
            Vec a = {};
            VecG d = {};
            const bool in = live && at < chunks;
            if (in) {
                a = reinterpret_cast<const Vec*>(static_cast<const T*>(p.X) + row * p.C)[at];
                d = reinterpret_cast<const VecG*>(static_cast<const TG*>(p.dY) + row * p.C)[at];
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float dy = norm_float(static_cast<TG>(d[j]));
                xh[c][j] = in ? (norm_float(static_cast<T>(a[j])) - mean) * rstd : 0.f;
                dw[c][j] = fmaf(dy, xh[c][j], dw[c][j]);
                db[c][j] += dy;
                g[c][j] = dy * w[c][j];
                sum[0] += g[c][j];
                sum[1] = fmaf(g[c][j], xh[c][j], sum[1]);
            }
        }
        row_sum<2, WIDE>(sum, p.lanes, s_sum, half);
        const float mg = sum[0] * inv_c, mx = sum[1] * inv_c;
        if (!live) continue;
        TG* const dx = static_cast<TG*>(p.out) + row * p.C;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int at = lane + c * p.lanes;
            VecG d;
#pragma unroll
            for (int j = 0; j < V; ++j) d[j] = norm_round<TG>(rstd * (g[c][j] - mg - xh[c][j] * mx));
            if (at < chunks) reinterpret_cast<VecG*>(dx)[at] = d;
        }
    }
    // the block's parts: over the threads that hold the same channels
    float* const parts = p.parts + static_cast<size_t>(blockIdx.x) * 2 * p.C;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                __syncthreads();
                s_part[threadIdx.x] = k ? db[c][j] : dw[c][j];
                __syncthreads();
                const int at = lane + c * p.lanes;
                if (slot == 0 && at < chunks) {
                    float x = 0.f;
                    for (int i = 0; i < slots; ++i) x += s_part[lane + i * p.lanes];
                    parts[static_cast<size_t>(k) * p.C + at * V + j] = x;
                }
            }
}

// dweight, dbias: the sum of the blocks' parts, 32 columns a block, 32 threads a column.
__global__ __launch_bounds__(1024) void norm_parts_kernel(const float* parts, int blocks, int C, float* dweight, float* dbias)
{
    __shared__ float s[32][33];
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), first = threadIdx.x >> 5;
    float x = 0.f;
    if (col < 2 * C)
        for (int i = first; i < blocks; i += 32) x += parts[static_cast<size_t>(i) * 2 * C + col];
    s[first][threadIdx.x & 31] = x;
    __syncthreads();
    if (first == 0 && col < 2 * C) {
        x = 0.f;
        for (int i = 0; i < 32; ++i) x += s[i][threadIdx.x & 31];
        (col < C ? dweight : dbias)[col < C ? col : col - C] = x;
    }
}

// How a row is held: V channels a chunk (the most, up to 16 bytes of X, that divide the row and to which the tensors are
// aligned), `chunks` chunks of a row over `lanes` threads, one chunk a thread where a block has enough.
struct NormPlan {
    int v, lanes;
    bool many;  // several chunks a thread
};

NormPlan norm_plan(const NormCall& c, const void* out)
{
    const int elem = c.dtype == SCRAM_BF16 ? 2 : 4;
    const int grad = c.dY ? (c.grad_dtype == SCRAM_BF16 ? 2 : 4) : elem;
    auto fits = [&](int n) {
        return c.channels % n == 0 && reinterpret_cast<uintptr_t>(c.X) % (n * elem) == 0 &&
               reinterpret_cast<uintptr_t>(out) % (n * grad) == 0 && reinterpret_cast<uintptr_t>(c.dY) % (n * grad) == 0;
    };
    NormPlan plan{16 / elem, 1, false};
    while (plan.v > 1 && !fits(plan.v)) plan.v /= 2;
    const int chunks = c.channels / plan.v;
    // one chunk a thread up to a wave's width, then up to 16 channels a thread, then more waves
    plan.many = chunks > 64;
    while (plan.lanes < 64 && plan.lanes < chunks) plan.lanes *= 2;
    while (plan.many && plan.lanes * (kPerThread / plan.v) < chunks) plan.lanes *= 2;
    return plan;
}

int norm_threads(const NormPlan& plan) { return plan.lanes > 256 ? plan.lanes : 256; }

// Blocks of the backward pass: each writes a row of parts.
int64_t norm_backward_blocks(int64_t rows) { return rows < 512 ? rows : 512; }

NormParams norm_params(const NormCall& c, const NormPlan& plan)
{
    NormParams p{};
    p.X = c.X;
    p.dY = c.dY;
    p.weight = c.weight;
    p.bias = c.bias;
    p.weight_f32 = c.weight_dtype == SCRAM_F32 ? 1 : 0;
    p.rows = c.rows;
    p.C = c.channels;
    p.lanes = plan.lanes;
    p.eps = c.eps;
    return p;
}

// f(V, NC, WIDE) for a plan of type T
template <typename T, typename F>
hipError_t norm_dispatch(const NormPlan& plan, F&& f)
{
    using std::integral_constant;
    auto with = [&](auto v) {
        constexpr int V = decltype(v)::value;
        if (!plan.many) return f(v, integral_constant<int, 1>{}, std::false_type{});
        if (plan.lanes <= 64) return f(v, integral_constant<int, kPerThread / V>{}, std::false_type{});
        return f(v, integral_constant<int, kPerThread / V>{}, std::true_type{});
    };
    if constexpr (sizeof(T) == 2)
        if (plan.v == 8) return with(integral_constant<int, 8>{});
    if (plan.v == 4) return with(integral_constant<int, 4>{});
    if (plan.v == 2) return with(integral_constant<int, 2>{});
    return with(integral_constant<int, 1>{});
}

}  // namespace

hipError_t launch_norm(const NormCall& c, void* Y, float* mean, float* rstd, hipStream_t stream)
{
    const NormPlan plan = norm_plan(c, Y);
    NormParams p = norm_params(c, plan);
    p.out = Y;
    p.mean = mean;
    p.rstd = rstd;
    const int threads = norm_threads(plan);
    const int64_t slots = threads / plan.lanes, want = (c.rows + slots - 1) / slots;
    const dim3 grid(static_cast<uint32_t>(want < 8192 ? want : 8192));
    auto run = [&](auto type) {
        using T = decltype(type);
        return norm_dispatch<T>(plan, [&](auto v, auto nc, auto wide) {
            hipLaunchKernelGGL((norm_kernel<T, decltype(v)::value, decltype(nc)::value, decltype(wide)::value>), grid, dim3(threads), 0,
                               stream, p);
            return hipGetLastError();
        });
    };
    return c.dtype == SCRAM_BF16 ? run(uint16_t{}) : run(float{});
}

size_t norm_backward_workspace_bytes(int64_t rows, int channels)
{
    return static_cast<size_t>(norm_backward_blocks(rows)) * 2 * channels * sizeof(float);
}

hipError_t launch_norm_backward(const NormCall& c, const float* mean, const float* rstd, void* dX, float* dweight,
                                float* dbias, void* workspace, hipStream_t stream)
{
    const NormPlan plan = norm_plan(c, dX);
    NormParams p = norm_params(c, plan);
    p.out = dX;
    p.mean_in = mean;
    p.rstd_in = rstd;
    p.parts = static_cast<float*>(workspace);
    const int threads = norm_threads(plan);
    const uint32_t blocks = static_cast<uint32_t>(norm_backward_blocks(c.rows));
    auto run = [&](auto type, auto grad) {
        using T = decltype(type);
        using TG = decltype(grad);
        return norm_dispatch<T>(plan, [&](auto v, auto nc, auto wide) {
            hipLaunchKernelGGL((norm_backward_kernel<T, TG, decltype(v)::value, decltype(nc)::value, decltype(wide)::value>),
                               dim3(blocks), dim3(threads), 0, stream, p);
            return hipGetLastError();
        });
    };
    const hipError_t e = c.dtype == SCRAM_F32        ? run(float{}, float{})
                         : c.grad_dtype == SCRAM_F32 ? run(uint16_t{}, float{})
                                                     : run(uint16_t{}, uint16_t{});
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(norm_parts_kernel, dim3((2 * c.channels + 31) / 32), dim3(1024), 0, stream, p.parts, static_cast<int>(blocks),
                       c.channels, dweight, dbias);
    return hipGetLastError();
}

}  // namespace scram
