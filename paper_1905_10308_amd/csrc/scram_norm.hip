// Layer norm of rows of C channels, forward and backward.
//
//   mu = mean x, r = (mean (x - mu)^2 + eps)^-1/2, xh = (x - mu) r, y = xh w + b
//   g = dy w:  dx = r (g - mean g - xh mean(g xh)),  dw = sum_rows dy xh,  db = sum_rows dy
//
// A row stays in registers between its passes, so every input is read once:
// bound by memory.  A row is held by `lanes` threads (a power of two), in
// chunks of 16 bytes of X, up to 16 channels a thread; several rows share a
// wave, or several waves a row.  Chunks are read and written whole wherever
// the row starts (memory takes vectors at any element's address), but for the
// last one of a row that does not end with a whole one.  Sums are fp32: the two of the forward
// pass are of the row and then of its centred values, so that a row's offset
// costs no accuracy.
//
// 262144 x 64 bf16: forward 14.7 us (67 MB and the statistics; 13.4 at a copy's
// rate), backward with fp32 gradients 41 us (33); 8192 x 4096 backward 51 (39).
//
// The weights' gradients: a block keeps those of its rows in registers,
// adds them up over its threads once at its end and writes one row of parts;
// a second kernel adds up the parts, in a fixed order.

#include "scram_rows.h"

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

// Sums of N values over the `lanes` threads of a row, on all of them.  Rows of several waves pass through LDS, in one of
// two halves in turn so that one barrier per sum is enough.
template <int N, bool WIDE, typename Lds>
__device__ __forceinline__ void row_sum(float (&x)[N], int lanes, Lds& lds, int& half)
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

// How many threads hold a row: a part of a wave, a chunk each; a wave; two or four waves; up to the whole block.
enum NormLayout { kNarrow = 0, kWave = 1, kWide = 2, kHuge = 3 };

constexpr int norm_threads(int layout) { return layout == kHuge ? kNormThreads : kBlock; }
constexpr bool norm_wide(int layout) { return layout >= kWide; }

// Rows per pass of a block's loop: their loads are in flight together, and wide rows share their barriers.  (262144 x 64,
// forward: a row at a time 26 us, four 16; 8192 x 4096 backward: one 57 us, two 50.)
constexpr int norm_rows(int layout, bool backward) { return layout == kHuge ? 1 : layout == kNarrow && !backward ? 4 : 2; }

// Channels at .. at + V - 1 of a row of C, those that it has, zeros after them.  TAIL: C is not a multiple of V.
template <bool TAIL, int V, typename T>
__device__ __forceinline__ vec<T, V> load_chunk(const T* row, int at, int C)
{
    return !TAIL || at + V <= C ? load_vec<T, V>(row + at) : load_part<T, V>(row + at, C % V);
}

template <bool TAIL, int V, typename T>
__device__ __forceinline__ void store_chunk(T* row, int at, int C, vec<T, V> x)
{
    if (!TAIL || at + V <= C)
        store_vec<T, V>(row + at, x);
    else
        store_part<T, V>(row + at, C % V, x);
}

// The thread's weights (or `none` without any).
template <bool TAIL, int V, int NC>
__device__ __forceinline__ void load_weights(const void* w, const NormParams& p, int lane, float none, float (&out)[NC][V])
{
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int at = (lane + c * p.lanes) * V;
        if (w != nullptr && at >= p.C) {
#pragma unroll
            for (int j = 0; j < V; ++j) out[c][j] = 0.f;
        } else if (w != nullptr && p.weight_f32) {
            const vec<float, V> x = load_chunk<TAIL, V>(static_cast<const float*>(w), at, p.C);
#pragma unroll
            for (int j = 0; j < V; ++j) out[c][j] = x[j];
        } else if (w != nullptr) {
            const vec<uint16_t, V> x = load_chunk<TAIL, V>(static_cast<const uint16_t*>(w), at, p.C);
#pragma unroll
            for (int j = 0; j < V; ++j) out[c][j] = to_float(static_cast<uint16_t>(x[j]));
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) out[c][j] = none;
        }
    }
}

// Every thread of a block takes part in every pass of its loop (the sums of wide rows hold barriers); rows past the end are
// neither read nor written.
template <typename T, int NC, int LAYOUT, bool TAIL>
__global__ __launch_bounds__(norm_threads(LAYOUT)) void norm_kernel(NormParams p)
{
    constexpr int V = kChunk<T>;
    using Vec = vec<T, V>;
    constexpr bool WIDE = norm_wide(LAYOUT);
    constexpr int R = norm_rows(LAYOUT, false);
    __shared__ float s_sum[2][WIDE ? norm_threads(LAYOUT) / 64 : 1][R];
    int half = 0;
    const int lane = threadIdx.x & (p.lanes - 1);
    const int slots = blockDim.x / p.lanes, slot = threadIdx.x / p.lanes;
    const float inv_c = 1.f / static_cast<float>(p.C);
    float w[NC][V], b[NC][V];
    load_weights<TAIL>(p.weight, p, lane, 1.f, w);
    load_weights<TAIL>(p.bias, p, lane, 0.f, b);
    const int64_t step = static_cast<int64_t>(slots) * R;
    for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * step; r0 < p.rows; r0 += static_cast<int64_t>(gridDim.x) * step) {
        const int64_t row = r0 + slot;  // and every slots-th row after it
        Vec a[R][NC];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const T* const x = static_cast<const T*>(p.X) + (row + k * slots) * p.C;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int at = (lane + c * p.lanes) * V;
                a[k][c] = Vec(T(0));
                if (row + k * slots < p.rows && at < p.C) a[k][c] = load_chunk<TAIL, V>(x, at, p.C);
            }
        }
        float mean[R], rstd[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            mean[k] = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int j = 0; j < V; ++j) mean[k] += to_float(static_cast<T>(a[k][c][j]));
        }
        row_sum<R, WIDE>(mean, p.lanes, s_sum, half);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            mean[k] *= inv_c;
            rstd[k] = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int left = p.C - (lane + c * p.lanes) * V;  // channels of the row from this chunk on
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float v = to_float(static_cast<T>(a[k][c][j])) - mean[k];
                    rstd[k] = (TAIL ? j : 0) < left ? fmaf(v, v, rstd[k]) : rstd[k];
                }
            }
        }
        row_sum<R, WIDE>(rstd, p.lanes, s_sum, half);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            rstd[k] = 1.f / sqrtf(rstd[k] * inv_c + p.eps);
            if (row + k * slots >= p.rows) continue;
            T* const y = static_cast<T*>(p.out) + (row + k * slots) * p.C;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int at = (lane + c * p.lanes) * V;
                Vec o;
#pragma unroll
                for (int j = 0; j < V; ++j)
                    o[j] = from_float<T>(fmaf((to_float(static_cast<T>(a[k][c][j])) - mean[k]) * rstd[k], w[c][j], b[c][j]));
                if (at < p.C) store_chunk<TAIL, V>(y, at, p.C, o);
            }
            if (lane == 0 && p.mean) {
                p.mean[row + k * slots] = mean[k];
                p.rstd[row + k * slots] = rstd[k];
            }
        }
    }
}

template <typename T, typename TG, int NC, int LAYOUT, bool TAIL>
__global__ __launch_bounds__(norm_threads(LAYOUT)) void norm_backward_kernel(NormParams p)
{
    constexpr int V = kChunk<T>;
    using Vec = vec<T, V>;
    using VecG = vec<TG, V>;
    constexpr bool WIDE = norm_wide(LAYOUT);
    constexpr int R = norm_rows(LAYOUT, true);
    __shared__ float s_sum[2][WIDE ? norm_threads(LAYOUT) / 64 : 1][2 * R];
    __shared__ float s_part[norm_threads(LAYOUT)];
    int half = 0;
    const int lane = threadIdx.x & (p.lanes - 1);
    const int slots = blockDim.x / p.lanes, slot = threadIdx.x / p.lanes;
    const float inv_c = 1.f / static_cast<float>(p.C);
    float w[NC][V], dw[NC][V], db[NC][V];
    load_weights<TAIL>(p.weight, p, lane, 1.f, w);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < V; ++j) dw[c][j] = db[c][j] = 0.f;
    const int64_t step = static_cast<int64_t>(slots) * R;
    for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * step; r0 < p.rows; r0 += static_cast<int64_t>(gridDim.x) * step) {
        const int64_t row = r0 + slot;
        Vec a[R][NC];
        VecG d[R][NC];
        float mean[R], rstd[R], sum[2 * R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int64_t at_row = row + k * slots;
            const bool live = at_row < p.rows;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int at = (lane + c * p.lanes) * V;
                a[k][c] = Vec(T(0));
                d[k][c] = VecG(TG(0));
                if (live && at < p.C) {
                    a[k][c] = load_chunk<TAIL, V>(static_cast<const T*>(p.X) + at_row * p.C, at, p.C);
                    d[k][c] = load_chunk<TAIL, V>(static_cast<const TG*>(p.dY) + at_row * p.C, at, p.C);
                }
            }
            mean[k] = live ? p.mean_in[at_row] : 0.f;
            rstd[k] = live ? p.rstd_in[at_row] : 0.f;
        }
        auto xhat = [&](int k, int c, int j) { return (to_float(static_cast<T>(a[k][c][j])) - mean[k]) * rstd[k]; };
#pragma unroll
        for (int k = 0; k < R; ++k) {
            sum[2 * k] = sum[2 * k + 1] = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                // past the end of the row dY is 0, but (0 - mean) rstd may be infinite: xh is 0 there
                const int left = p.C - (lane + c * p.lanes) * V;
                const float r = left > 0 ? rstd[k] : 0.f;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float dy = to_float(static_cast<TG>(d[k][c][j]));
                    const float xh = TAIL && j >= left ? 0.f : (to_float(static_cast<T>(a[k][c][j])) - mean[k]) * r;
                    dw[c][j] = fmaf(dy, xh, dw[c][j]);
                    db[c][j] += dy;
                    const float g = dy * w[c][j];
                    sum[2 * k] += g;
                    sum[2 * k + 1] = fmaf(g, xh, sum[2 * k + 1]);
                }
            }
        }
        row_sum<2 * R, WIDE>(sum, p.lanes, s_sum, half);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (row + k * slots >= p.rows) continue;
            const float mg = sum[2 * k] * inv_c, mx = sum[2 * k + 1] * inv_c;
            TG* const dx = static_cast<TG*>(p.out) + (row + k * slots) * p.C;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int at = (lane + c * p.lanes) * V;
                VecG o;
#pragma unroll
                for (int j = 0; j < V; ++j)
                    o[j] = from_float<TG>(rstd[k] * (to_float(static_cast<TG>(d[k][c][j])) * w[c][j] - mg - xhat(k, c, j) * mx));
                if (at < p.C) store_chunk<TAIL, V>(dx, at, p.C, o);
            }
        }
    }
    // the block's parts: over the threads that hold the same channels, first those of a wave
    float* const parts = p.parts + static_cast<size_t>(blockIdx.x) * 2 * p.C;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float x = k ? db[c][j] : dw[c][j];
                for (int m = p.lanes; m < 64; m <<= 1) x += __shfl_xor(x, m);
                const int group = p.lanes < 64 ? 64 : p.lanes;  // threads that hold different channels or a wave's sums
                if (slots > 1 && group < static_cast<int>(blockDim.x)) {
                    __syncthreads();
                    s_part[threadIdx.x] = x;
                    __syncthreads();
                    if (threadIdx.x < static_cast<uint32_t>(group))
                        for (int i = threadIdx.x + group; i < static_cast<int>(blockDim.x); i += group) x += s_part[i];
                }
                const int at = (lane + c * p.lanes) * V + j;
                if (slot == 0 && at < p.C) parts[static_cast<size_t>(k) * p.C + at] = x;
            }
}

// dweight, dbias: the sum of the blocks' parts, 32 columns a block, 32 threads a column.
__global__ __launch_bounds__(1024) void norm_parts_kernel(const float* parts, int blocks, int C, float* dweight, float* dbias)
{
    __shared__ float s[32][33];
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), first = threadIdx.x >> 5;
    float x = 0.f;
    if (col < 2 * C) {
#pragma unroll 8
        for (int i = first; i < blocks; i += 32) x += parts[static_cast<size_t>(i) * 2 * C + col];
    }
    s[first][threadIdx.x & 31] = x;
    __syncthreads();
    if (first == 0 && col < 2 * C) {
        x = 0.f;
        for (int i = 0; i < 32; ++i) x += s[i][threadIdx.x & 31];
        (col < C ? dweight : dbias)[col < C ? col : col - C] = x;
    }
}

// How a row is held: its chunks over `lanes` threads, one a thread up to a wave's width, then up to 16 channels a thread.
struct NormPlan {
    int lanes, layout;
};

NormPlan norm_plan(const NormCall& c)
{
    const int chunk = c.dtype == SCRAM_BF16 ? kChunk<uint16_t> : kChunk<float>;
    const int chunks = (c.channels + chunk - 1) / chunk;
    NormPlan plan{1, kNarrow};
    while (plan.lanes < 64 && plan.lanes < chunks) plan.lanes *= 2;
    if (chunks > 64) {
        while (plan.lanes * (kPerThread / chunk) < chunks) plan.lanes *= 2;
        plan.layout = plan.lanes <= 64 ? kWave : plan.lanes <= kBlock ? kWide : kHuge;
    }
    return plan;
}

int block_threads(const NormPlan& plan) { return plan.layout == kHuge ? plan.lanes : kBlock; }

// Blocks of the backward pass, each of which writes a row of parts: two per CU, or one where a row takes more than 256
// threads.  (8192 x 4096: 512 blocks 50 us, 256 64, 768 64; 2048 x 16384: 256 blocks 70, 512 94.)  Fewer rows than that leave
// blocks without one, whose parts are zeros (a call's kernels, with as many blocks as the rows fill beside it, bf16: 512 x 64
// 12 and 11 us, 2048 x 1024 16 and 14, 512 x 4096 22 and 16; 4096 rows and more the same).
int64_t norm_backward_blocks(int64_t rows, int channels)
{
    const int64_t most = channels > kPerThread * kBlock ? 256 : 512;
    return rows < most ? rows : most;
}

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

// f(NC, LAYOUT, TAIL) for a plan of type T
template <typename T, typename F>
hipError_t norm_dispatch(const NormPlan& plan, int channels, F&& f)
{
    using std::integral_constant;
    constexpr integral_constant<int, kPerThread / kChunk<T>> many{};
    auto with = [&](auto tail) {
        if (plan.layout == kNarrow) return f(integral_constant<int, 1>{}, integral_constant<int, kNarrow>{}, tail);
        if (plan.layout == kWave) return f(many, integral_constant<int, kWave>{}, tail);
        if (plan.layout == kWide) return f(many, integral_constant<int, kWide>{}, tail);
        return f(many, integral_constant<int, kHuge>{}, tail);
    };
    return channels % kChunk<T> ? with(std::true_type{}) : with(std::false_type{});
}

}  // namespace

hipError_t launch_norm(const NormCall& c, void* Y, float* mean, float* rstd, hipStream_t stream)
{
    const NormPlan plan = norm_plan(c);
    NormParams p = norm_params(c, plan);
    p.out = Y;
    p.mean = mean;
    p.rstd = rstd;
    const int threads = block_threads(plan);
    const int64_t slots = threads / plan.lanes, want = (c.rows + slots * 2 - 1) / (slots * 2);
    const dim3 grid(static_cast<uint32_t>(want < 4096 ? want : 4096));
    auto run = [&](auto type) {
        using T = decltype(type);
        return norm_dispatch<T>(plan, c.channels, [&](auto nc, auto layout, auto tail) {
            hipLaunchKernelGGL((norm_kernel<T, decltype(nc)::value, decltype(layout)::value, decltype(tail)::value>), grid, dim3(threads), 0,
                               stream, p);
            return hipGetLastError();
        });
    };
    return c.dtype == SCRAM_BF16 ? run(uint16_t{}) : run(float{});
}

size_t norm_backward_workspace_bytes(int64_t rows, int channels)
{
    return static_cast<size_t>(norm_backward_blocks(rows, channels)) * 2 * channels * sizeof(float);
}

hipError_t launch_norm_backward(const NormCall& c, const float* mean, const float* rstd, void* dX, float* dweight,
                                float* dbias, void* workspace, hipStream_t stream)
{
    const NormPlan plan = norm_plan(c);
    NormParams p = norm_params(c, plan);
    p.out = dX;
    p.mean_in = mean;
    p.rstd_in = rstd;
    p.parts = static_cast<float*>(workspace);
    const int threads = block_threads(plan);
    const uint32_t blocks = static_cast<uint32_t>(norm_backward_blocks(c.rows, c.channels));
    auto run = [&](auto type, auto grad) {
        using T = decltype(type);
        using TG = decltype(grad);
        return norm_dispatch<T>(plan, c.channels, [&](auto nc, auto layout, auto tail) {
            hipLaunchKernelGGL((norm_backward_kernel<T, TG, decltype(nc)::value, decltype(layout)::value, decltype(tail)::value>),
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
