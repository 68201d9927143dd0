// Group norm of images, channels last, with an activation, forward and backward.
//
// Over an image's pixels and a group's channels:
//   mu = mean x, r = (mean (x - mu)^2 + eps)^-1/2, xh = (x - mu) r, z = xh w + b, y = act(z)
//   dz = dy act'(z), g = dz w:  dx = r (g - mean g - xh mean(g xh)),  dw = sum dz xh,  db = sum dz
//
// Bound by memory: an image is read twice (statistics, then the result; the
// second time mostly from the caches) and written once.  An image is one run of
// pixels * C values, cut into super-rows of the smallest whole number of pixels
// that is a whole number of 16-byte chunks.  A thread stays at one chunk of the
// super-rows, so that the channels of its values never change, and whole
// vectors are read whatever C is.
//
// Statistics are not sums of squares: a thread takes the mean of a few values
// and the squares of what is left around it, and two such (count, mean, sum of
// squares around it) are joined exactly (Chan, Golub, LeVeque 1983), so that
// an image's offset costs no accuracy.

#include "scram_rows.h"

namespace scram {
namespace {

constexpr int kGroupBatch = 4;  // super-rows of a thread in flight together

struct GroupParams {
    const void* X;
    const void* dY;
    const void* weight;  // nullable
    const void* bias;    // nullable
    int weight_f32, silu;
    void* out;
    const float* mean_in;
    const float* rstd_in;
    float* mean;
    float* rstd;
    float* parts;        // of the blocks
    float* sums;         // backward: [images, 2, C] sum dz xh, sum dz
    float* means;        // backward: [images, groups, 2] mean g, mean g xh
    int64_t images, total;   // values of an image
    int64_t supers, per;     // super-rows of an image, of a block
    int C, groups, width;    // channels of a group
    int chunks, slots, columns;  // of a super-row; super-rows that a block takes at a time; blocks beside each other over its chunks
    int blocks;                  // of an image, one after another
    int pixels_super;
    float eps;
};

// Where a thread of unit u stands.
struct GroupPlace {
    int64_t image, first, last;  // its super-rows first, first + slots, .. below last
    int slot, chunk, block;
    bool active;
};

__device__ __forceinline__ GroupPlace group_place(const GroupParams& p, int64_t u)
{
    GroupPlace a;
    const int column = static_cast<int>(u % p.columns);
    a.block = static_cast<int>(u / p.columns % p.blocks);
    a.image = u / p.columns / p.blocks;
    const int across = min(p.chunks, kBlock);
    a.slot = threadIdx.x / across;
    a.chunk = column * kBlock + static_cast<int>(threadIdx.x) % across;
    a.active = a.slot < p.slots && a.chunk < p.chunks;
    a.first = a.block * p.per + a.slot;
    a.last = a.active ? min(p.supers, (a.block + 1) * p.per) : 0;
    return a;
}

template <int V>
__device__ __forceinline__ float channel_value(const void* w, int f32, int c, float none)
{
    if (w == nullptr) return none;
    return f32 ? static_cast<const float*>(w)[c] : to_float(static_cast<const uint16_t*>(w)[c]);
}

struct Moments {
    float n, mean, m2;
};

__device__ __forceinline__ Moments join(Moments a, Moments b)
{
    const float n = a.n + b.n;
    if (n == 0.f) return a;
    const float f = b.n / n, d = b.mean - a.mean;
    return Moments{n, fmaf(d, f, a.mean), a.m2 + b.m2 + d * d * (a.n * f)};
}

// Elements at `at` of an image's run of `total`, those that it has, zeros after them.
template <typename T, int V>
__device__ __forceinline__ vec<T, V> load_run(const T* image, int64_t at, int64_t total)
{
    return at + V <= total ? load_vec<T, V>(image + at)
                           : at < total ? load_part<T, V>(image + at, static_cast<int>(total - at)) : vec<T, V>(T(0));
}

template <typename T, int V>
__device__ __forceinline__ void store_run(T* image, int64_t at, int64_t total, vec<T, V> x)
{
    if (at + V <= total)
        store_vec<T, V>(image + at, x);
    else if (at < total)
        store_part<T, V>(image + at, static_cast<int>(total - at), x);
}

// Count, mean and squares around it of every place of the super-rows, over a block's super-rows.
template <typename T>
__global__ __launch_bounds__(kBlock) void group_stats_kernel(GroupParams p)
{
    constexpr int V = kChunk<T>, R = kGroupBatch;
    __shared__ float s_part[3][V][kBlock];
    const int64_t units = p.images * p.columns * p.blocks;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const GroupPlace a = group_place(p, u);
        const T* const image = static_cast<const T*>(p.X) + a.image * p.total;
        const int64_t step = static_cast<int64_t>(p.chunks) * V;
        Moments acc[V];
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = Moments{0.f, 0.f, 0.f};
        int64_t r = a.first;
        float n = 0.f;
        // batches of whole chunks
        for (; r + (R - 1) * static_cast<int64_t>(p.slots) < a.last &&
               (r + (R - 1) * static_cast<int64_t>(p.slots)) * step + a.chunk * V + V <= p.total;
             r += R * static_cast<int64_t>(p.slots)) {
            vec<T, V> x[R];
#pragma unroll
            for (int k = 0; k < R; ++k) x[k] = load_vec<T, V>(image + (r + k * static_cast<int64_t>(p.slots)) * step + a.chunk * V);
            const float next = n + R, f = R / next, nf = n * f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float m = 0.f, s = 0.f;
#pragma unroll
                for (int k = 0; k < R; ++k) m += to_float(static_cast<T>(x[k][j]));
                m *= 1.f / R;
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    const float d = to_float(static_cast<T>(x[k][j])) - m;
                    s = fmaf(d, d, s);
                }
                const float d = m - acc[j].mean;
                acc[j].mean = fmaf(d, f, acc[j].mean);
                acc[j].m2 += s + d * d * nf;
            }
            n = next;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j].n = n;
        for (; r < a.last; r += p.slots) {
            const int64_t at = r * step + a.chunk * V;
            const vec<T, V> x = load_run<T, V>(image, at, p.total);
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (at + j < p.total) acc[j] = join(acc[j], Moments{1.f, to_float(static_cast<T>(x[j])), 0.f});
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < V; ++j) {
            s_part[0][j][threadIdx.x] = acc[j].n;
            s_part[1][j][threadIdx.x] = acc[j].mean;
            s_part[2][j][threadIdx.x] = acc[j].m2;
        }
        __syncthreads();
        if (a.slot != 0 || !a.active) continue;
        float* const to = p.parts + 3 * ((a.image * p.blocks + a.block) * step + a.chunk * V);
        const int across = min(p.chunks, kBlock);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            for (int k = 1; k < p.slots; ++k) {
                const int t = static_cast<int>(threadIdx.x) + k * across;
                acc[j] = join(acc[j], Moments{s_part[0][j][t], s_part[1][j][t], s_part[2][j][t]});
            }
            to[3 * j] = acc[j].n;
            to[3 * j + 1] = acc[j].mean;
            to[3 * j + 2] = acc[j].m2;
        }
    }
}

// The statistics of a group of an image, from the blocks' parts.
__global__ __launch_bounds__(kBlock) void group_join_kernel(GroupParams p)
{
    __shared__ Moments s_part[kBlock / 64];
    const int64_t step = static_cast<int64_t>(p.C) * p.pixels_super;
    for (int64_t u = blockIdx.x; u < p.images * p.groups; u += gridDim.x) {
        const int64_t image = u / p.groups;
        const int c0 = static_cast<int>(u % p.groups) * p.width, each = p.width * p.pixels_super;
        Moments acc{0.f, 0.f, 0.f};
        for (int64_t i = threadIdx.x; i < static_cast<int64_t>(p.blocks) * each; i += kBlock) {
            const int b = static_cast<int>(i / each), e = static_cast<int>(i % each);
            const float* const at = p.parts + 3 * ((image * p.blocks + b) * step + e / p.width * static_cast<int64_t>(p.C) + c0 + e % p.width);
            acc = join(acc, Moments{at[0], at[1], at[2]});
        }
        for (int m = 1; m < 64; m <<= 1)
            acc = join(acc, Moments{__shfl_xor(acc.n, m), __shfl_xor(acc.mean, m), __shfl_xor(acc.m2, m)});
        __syncthreads();
        if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = acc;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kBlock / 64; ++w) acc = join(acc, s_part[w]);
            p.mean[u] = acc.mean;
            p.rstd[u] = 1.f / sqrtf(acc.m2 / acc.n + p.eps);
        }
    }
}

// z / (1 + exp(-z)), and its derivative
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f)); }
__device__ __forceinline__ float silu(float z) { return z * sigmoid(z); }
__device__ __forceinline__ float silu_slope(float z)
{
    const float s = sigmoid(z);
    return s * fmaf(z, 1.f - s, 1.f);
}

// What a thread knows of the channels of its chunk.
template <typename T, int V>
struct GroupChannels {
    float mean[V], rstd[V], w[V], b[V];
    int group[V];

    __device__ __forceinline__ void load(const GroupParams& p, const GroupPlace& a, const float* mean_in, const float* rstd_in)
    {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c = a.active ? (a.chunk * V + j) % p.C : 0;
            group[j] = c / p.width;
            mean[j] = mean_in[a.image * p.groups + group[j]];
            rstd[j] = rstd_in[a.image * p.groups + group[j]];
            w[j] = channel_value<V>(p.weight, p.weight_f32, c, 1.f);
            b[j] = channel_value<V>(p.bias, p.weight_f32, c, 0.f);
        }
    }
};

template <typename T>
__global__ __launch_bounds__(kBlock) void group_apply_kernel(GroupParams p)
{
    constexpr int V = kChunk<T>, R = kGroupBatch;
    const int64_t units = p.images * p.columns * p.blocks;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const GroupPlace a = group_place(p, u);
        const T* const from = static_cast<const T*>(p.X) + a.image * p.total;
        T* const to = static_cast<T*>(p.out) + a.image * p.total;
        const int64_t step = static_cast<int64_t>(p.chunks) * V;
        GroupChannels<T, V> ch;
        ch.load(p, a, p.mean, p.rstd);
        for (int64_t r = a.first; r < a.last; r += R * static_cast<int64_t>(p.slots)) {
            vec<T, V> x[R];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const int64_t row = r + k * static_cast<int64_t>(p.slots);
                x[k] = vec<T, V>(T(0));
                if (row < a.last) x[k] = load_run<T, V>(from, row * step + a.chunk * V, p.total);
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const int64_t row = r + k * static_cast<int64_t>(p.slots);
                vec<T, V> y;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float z = fmaf((to_float(static_cast<T>(x[k][j])) - ch.mean[j]) * ch.rstd[j], ch.w[j], ch.b[j]);
                    y[j] = from_float<T>(p.silu ? silu(z) : z);
                }
                if (row < a.last) store_run<T, V>(to, row * step + a.chunk * V, p.total, y);
            }
        }
    }
}

// Sums of dz xh and dz of every place of the super-rows, over a block's super-rows.
template <typename T, typename TG>
__global__ __launch_bounds__(kBlock) void group_sums_kernel(GroupParams p)
{
    constexpr int V = kChunk<T>, R = kGroupBatch;
    __shared__ float s_part[2][V][kBlock];
    const int64_t units = p.images * p.columns * p.blocks;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const GroupPlace a = group_place(p, u);
        const T* const image = static_cast<const T*>(p.X) + a.image * p.total;
        const TG* const grad = static_cast<const TG*>(p.dY) + a.image * p.total;
        const int64_t step = static_cast<int64_t>(p.chunks) * V;
        GroupChannels<T, V> ch;
        ch.load(p, a, p.mean_in, p.rstd_in);
        float dw[V], db[V];
#pragma unroll
        for (int j = 0; j < V; ++j) dw[j] = db[j] = 0.f;
        for (int64_t r = a.first; r < a.last; r += R * static_cast<int64_t>(p.slots)) {
            vec<T, V> x[R];
            vec<TG, V> d[R];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const int64_t row = r + k * static_cast<int64_t>(p.slots);
                x[k] = vec<T, V>(T(0));
                d[k] = vec<TG, V>(TG(0));
                if (row < a.last) {
                    x[k] = load_run<T, V>(image, row * step + a.chunk * V, p.total);
                    d[k] = load_run<TG, V>(grad, row * step + a.chunk * V, p.total);
                }
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const int64_t left = r + k * static_cast<int64_t>(p.slots) < a.last
                                         ? p.total - ((r + k * static_cast<int64_t>(p.slots)) * step + a.chunk * V) : 0;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float xh = (to_float(static_cast<T>(x[k][j])) - ch.mean[j]) * ch.rstd[j];
                    float dz = to_float(static_cast<TG>(d[k][j]));
                    if (p.silu) dz *= silu_slope(fmaf(xh, ch.w[j], ch.b[j]));
                    if (j < left) {  // (what stands in place of a value that is not there may be infinite)
                        dw[j] = fmaf(dz, xh, dw[j]);
                        db[j] += dz;
                    }
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < V; ++j) {
            s_part[0][j][threadIdx.x] = dw[j];
            s_part[1][j][threadIdx.x] = db[j];
        }
        __syncthreads();
        if (a.slot != 0 || !a.active) continue;
        float* const to = p.parts + 2 * ((a.image * p.blocks + a.block) * step + a.chunk * V);
        const int across = min(p.chunks, kBlock);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            for (int k = 1; k < p.slots; ++k) {
                dw[j] += s_part[0][j][threadIdx.x + k * across];
                db[j] += s_part[1][j][threadIdx.x + k * across];
            }
            to[2 * j] = dw[j];
            to[2 * j + 1] = db[j];
        }
    }
}

// An image's sums of each channel of a group, and from them the means that the group's dx takes off.
__global__ __launch_bounds__(kBlock) void group_means_kernel(GroupParams p)
{
    __shared__ float s_part[2][kBlock];
    const int64_t step = static_cast<int64_t>(p.C) * p.pixels_super;
    int across = 1;
    while (across < p.width && across < kBlock) across *= 2;
    const int lanes = kBlock / across, lane = threadIdx.x / across, entries = p.blocks * p.pixels_super;
    for (int64_t u = blockIdx.x; u < p.images * p.groups; u += gridDim.x) {
        const int64_t image = u / p.groups;
        const int g = static_cast<int>(u % p.groups);
        float g1 = 0.f, g2 = 0.f;
        for (int c0 = 0; c0 < p.width; c0 += across) {
            const int k = c0 + static_cast<int>(threadIdx.x) % across, c = g * p.width + k;
            float dw = 0.f, db = 0.f;
            if (k < p.width)
                for (int i = lane; i < entries; i += lanes) {
                    const float* const at =
                        p.parts + 2 * ((image * p.blocks + i / p.pixels_super) * step + i % p.pixels_super * static_cast<int64_t>(p.C) + c);
                    dw += at[0];
                    db += at[1];
                }
            __syncthreads();
            s_part[0][threadIdx.x] = dw;
            s_part[1][threadIdx.x] = db;
            __syncthreads();
            if (lane == 0 && k < p.width) {
                for (int l = 1; l < lanes; ++l) {
                    dw += s_part[0][threadIdx.x + l * across];
                    db += s_part[1][threadIdx.x + l * across];
                }
                p.sums[(image * 2) * p.C + c] = dw;
                p.sums[(image * 2 + 1) * p.C + c] = db;
                const float w = channel_value<1>(p.weight, p.weight_f32, c, 1.f);
                g1 = fmaf(w, db, g1);
                g2 = fmaf(w, dw, g2);
            }
        }
        __syncthreads();
        s_part[0][threadIdx.x] = g1;
        s_part[1][threadIdx.x] = g2;
        for (int m = kBlock / 2; m >= 1; m >>= 1) {
            __syncthreads();
            if (static_cast<int>(threadIdx.x) < m) {
                s_part[0][threadIdx.x] += s_part[0][threadIdx.x + m];
                s_part[1][threadIdx.x] += s_part[1][threadIdx.x + m];
            }
        }
        if (threadIdx.x == 0) {
            const float count = static_cast<float>(p.total / p.groups);
            p.means[2 * u] = s_part[0][0] / count;
            p.means[2 * u + 1] = s_part[1][0] / count;
        }
    }
}

template <typename T, typename TG>
__global__ __launch_bounds__(kBlock) void group_grad_kernel(GroupParams p)
{
    constexpr int V = kChunk<T>, R = kGroupBatch;
    const int64_t units = p.images * p.columns * p.blocks;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const GroupPlace a = group_place(p, u);
        const T* const image = static_cast<const T*>(p.X) + a.image * p.total;
        const TG* const grad = static_cast<const TG*>(p.dY) + a.image * p.total;
        TG* const to = static_cast<TG*>(p.out) + a.image * p.total;
        const int64_t step = static_cast<int64_t>(p.chunks) * V;
        GroupChannels<T, V> ch;
        ch.load(p, a, p.mean_in, p.rstd_in);
        float mg[V], mx[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            mg[j] = p.means[2 * (a.image * p.groups + ch.group[j])];
            mx[j] = p.means[2 * (a.image * p.groups + ch.group[j]) + 1];
        }
        for (int64_t r = a.first; r < a.last; r += R * static_cast<int64_t>(p.slots)) {
            vec<T, V> x[R];
            vec<TG, V> d[R];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const int64_t row = r + k * static_cast<int64_t>(p.slots);
                x[k] = vec<T, V>(T(0));
                d[k] = vec<TG, V>(TG(0));
                if (row < a.last) {
                    x[k] = load_run<T, V>(image, row * step + a.chunk * V, p.total);
                    d[k] = load_run<TG, V>(grad, row * step + a.chunk * V, p.total);
                }
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const int64_t row = r + k * static_cast<int64_t>(p.slots);
                vec<TG, V> y;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float xh = (to_float(static_cast<T>(x[k][j])) - ch.mean[j]) * ch.rstd[j];
                    float dz = to_float(static_cast<TG>(d[k][j]));
                    if (p.silu) dz *= silu_slope(fmaf(xh, ch.w[j], ch.b[j]));
                    y[j] = from_float<TG>(ch.rstd[j] * (dz * ch.w[j] - mg[j] - xh * mx[j]));
                }
                if (row < a.last) store_run<TG, V>(to, row * step + a.chunk * V, p.total, y);
            }
        }
    }
}

// dweight, dbias: the sum of the images' sums, 32 columns a block, 32 threads a column.
__global__ __launch_bounds__(1024) void group_parts_kernel(GroupParams p, float* dweight, float* dbias)
{
    __shared__ float s[32][33];
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), first = threadIdx.x >> 5;
    float x = 0.f;
    if (col < 2 * p.C)
        for (int64_t i = first; i < p.images; i += 32) x += p.sums[i * 2 * p.C + col];
    s[first][threadIdx.x & 31] = x;
    __syncthreads();
    if (first == 0 && col < 2 * p.C) {
        x = 0.f;
        for (int i = 0; i < 32; ++i) x += s[i][threadIdx.x & 31];
        (col < p.C ? dweight : dbias)[col < p.C ? col : col - p.C] = x;
    }
}

size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

GroupParams group_params(const GroupCall& c)
{
    GroupParams p{};
    p.X = c.X;
    p.dY = c.dY;
    p.weight = c.weight;
    p.bias = c.bias;
    p.weight_f32 = c.weight_dtype == SCRAM_F32 ? 1 : 0;
    p.silu = c.activation == SCRAM_ACT_SILU ? 1 : 0;
    p.images = c.images;
    p.total = c.pixels * c.channels;
    p.C = c.channels;
    p.groups = c.groups;
    p.width = c.channels / c.groups;
    p.eps = c.eps;
    const int V = c.dtype == SCRAM_BF16 ? kChunk<uint16_t> : kChunk<float>;
    int common = V;
    while (c.channels % common) common /= 2;
    p.chunks = c.channels / common;
    p.pixels_super = V / common;
    p.slots = p.chunks < kBlock ? kBlock / p.chunks : 1;
    p.columns = (p.chunks + kBlock - 1) / kBlock;
    p.supers = (c.pixels + p.pixels_super - 1) / p.pixels_super;
    // blocks of an image: some eight per CU over all images, with two batches at least for every thread
    const int64_t most = (p.supers + 2 * kGroupBatch * p.slots - 1) / (2 * kGroupBatch * p.slots);
    int64_t blocks = 2048 / (p.images < 2048 ? p.images * p.columns : 2048);
    blocks = blocks < 1 ? 1 : blocks > most ? most : blocks;
    p.per = (p.supers + blocks - 1) / blocks;
    p.blocks = static_cast<int>((p.supers + p.per - 1) / p.per);
    return p;
}

uint32_t group_grid(int64_t units) { return static_cast<uint32_t>(units < (1 << 20) ? units : 1 << 20); }

size_t group_parts_bytes(const GroupParams& p, int each)
{
    return round256(size_t(p.images) * p.blocks * p.C * p.pixels_super * each * sizeof(float));
}

}  // namespace

size_t group_norm_workspace_bytes(const GroupCall& c)
{
    const GroupParams p = group_params(c);
    return group_parts_bytes(p, 3) + round256(8 * size_t(p.images) * p.groups);
}

hipError_t launch_group_norm(const GroupCall& c, void* Y, float* mean, float* rstd, void* workspace, hipStream_t stream)
{
    GroupParams p = group_params(c);
    p.out = Y;
    p.parts = static_cast<float*>(workspace);
    p.mean = mean ? mean : reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + group_parts_bytes(p, 3));
    p.rstd = rstd ? rstd : p.mean + p.images * p.groups;
    const dim3 grid(group_grid(p.images * p.columns * p.blocks)), joins(group_grid(p.images * p.groups)), block(kBlock);
    auto run = [&](auto type) {
        using T = decltype(type);
        hipLaunchKernelGGL(group_stats_kernel<T>, grid, block, 0, stream, p);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(group_join_kernel, joins, block, 0, stream, p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        hipLaunchKernelGGL(group_apply_kernel<T>, grid, block, 0, stream, p);
        return hipGetLastError();
    };
    return c.dtype == SCRAM_BF16 ? run(uint16_t{}) : run(float{});
}

size_t group_norm_backward_workspace_bytes(const GroupCall& c)
{
    const GroupParams p = group_params(c);
    return group_parts_bytes(p, 2) + round256(8 * size_t(p.images) * p.C) + round256(8 * size_t(p.images) * p.groups);
}

hipError_t launch_group_norm_backward(const GroupCall& c, const float* mean, const float* rstd, void* dX, float* dweight,
                                      float* dbias, void* workspace, hipStream_t stream)
{
    GroupParams p = group_params(c);
    p.out = dX;
    p.mean_in = mean;
    p.rstd_in = rstd;
    unsigned char* const at = static_cast<unsigned char*>(workspace);
    p.parts = reinterpret_cast<float*>(at);
    p.sums = reinterpret_cast<float*>(at + group_parts_bytes(p, 2));
    p.means = reinterpret_cast<float*>(at + group_parts_bytes(p, 2) + round256(8 * size_t(p.images) * p.C));
    const dim3 grid(group_grid(p.images * p.columns * p.blocks)), joins(group_grid(p.images * p.groups)), block(kBlock);
    auto run = [&](auto type, auto grad) {
        using T = decltype(type);
        using TG = decltype(grad);
        hipLaunchKernelGGL((group_sums_kernel<T, TG>), grid, block, 0, stream, p);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(group_means_kernel, joins, block, 0, stream, p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        hipLaunchKernelGGL((group_grad_kernel<T, TG>), grid, block, 0, stream, p);
        return hipGetLastError();
    };
    const hipError_t e = c.dtype == SCRAM_F32        ? run(float{}, float{})
                         : c.grad_dtype == SCRAM_F32 ? run(uint16_t{}, float{})
                                                     : run(uint16_t{}, uint16_t{});
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(group_parts_kernel, dim3((2 * p.C + 31) / 32), dim3(1024), 0, stream, p, dweight, dbias);
    return hipGetLastError();
}

}  // namespace scram
