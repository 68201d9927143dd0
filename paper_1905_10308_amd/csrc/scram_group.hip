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
// and the squares of what is left around it, and (count, mean, squares around
// it) of two parts, or of many at once, are joined by their means' distances
// (Chan, Golub, LeVeque 1983), so that an image's offset costs no accuracy.
//
// Small groups are held in a block's registers and read once, in one launch.
//
// Measured, bf16, replayed from a graph: 4 images of 256 x 256, 128 channels
// 44.9 us, 67 MB each read and written (3.0 TB/s; a copy of them takes 20.0, 6.7
// TB/s, half of it from the caches as here); the gradients of 4 of 128 x 128,
// 256 channels 41.4 us.  Alone in a trace the kernels take 47.2 and 46.2 us.

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
    float* dweight;
    float* dbias;
    uint32_t weight_blocks;
    int64_t images, total;   // values of an image
    int64_t supers, per;     // super-rows of an image, of a block
    int C, groups, width;    // channels of a group
    int chunks, slots, columns;  // of a super-row; super-rows that a block takes at a time; blocks beside each other over its chunks
    int blocks;                  // of an image, one after another
    int pixels_super;
    float eps;
    Div div_width;
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

// What a difference of sums of squares leaves of them; not a number stays that (a maximum would hide it).
__device__ __forceinline__ float not_negative(float x) { return x < 0.f ? 0.f : x; }

// Sums of two values a thread over a block, on all its threads.
__device__ __forceinline__ float2 block_sum(float2 x, float2 (&lds)[kBlock / 64])
{
    for (int m = 1; m < 64; m <<= 1) {
        x.x += __shfl_xor(x.x, m);
        x.y += __shfl_xor(x.y, m);
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
    for (int w = 1; w < kBlock / 64; ++w) {
        x.x += lds[w].x;
        x.y += lds[w].y;
    }
    return x;
}

// What `count` places of a block's threads hold, summed over its slots: value(slot, place), two numbers, to use(place, sum).
// Threads share the slots of a place where there are fewer places than threads.
template <typename Value, typename Use>
__device__ __forceinline__ void over_slots(int count, int slots, float2 (&lds)[kBlock], Value&& value, Use&& use)
{
    const int share = count < kBlock ? kBlock / count : 1;
    const int part = share > 1 ? static_cast<int>(threadIdx.x) / count : 0;
    for (int place = share > 1 ? static_cast<int>(threadIdx.x) % count : static_cast<int>(threadIdx.x); place < count;
         place += share > 1 ? count : kBlock) {
        float2 x = make_float2(0.f, 0.f);
        if (part < share)
            for (int k = part; k < slots; k += share) {
                const float2 y = value(k, place);
                x.x += y.x;
                x.y += y.y;
            }
        if (share > 1) {
            __syncthreads();
            lds[threadIdx.x] = x;
            __syncthreads();
            x = lds[place];
            for (int k = 1; k < share; ++k) {
                x.x += lds[place + k * count].x;
                x.y += lds[place + k * count].y;
            }
        }
        if (part == 0) use(place, x);
        if (share > 1) return;
    }
}

// The super-rows of a thread that hold whole chunks: those below this one.
__device__ __forceinline__ int64_t whole_rows(const GroupParams& p, const GroupPlace& a, int64_t step, int V)
{
    const int64_t n = p.total - static_cast<int64_t>(a.chunk) * V - V;
    return n < 0 ? 0 : min(a.last, n / step + 1);
}

// Count, mean and squares around it of every place of the super-rows, over a block's super-rows.
template <typename T>
__global__ __launch_bounds__(kBlock) void group_stats_kernel(GroupParams p)
{
    constexpr int V = kChunk<T>, R = kGroupBatch;
    __shared__ float s_n[kBlock], s_mean[V][kBlock], s_m2[V][kBlock], s_all[V * kBlock];
    __shared__ float2 s_sum[kBlock];
    const int64_t units = p.images * p.columns * p.blocks;
    const int64_t step = static_cast<int64_t>(p.chunks) * V;
    const int across = min(p.chunks, kBlock);
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const GroupPlace a = group_place(p, u);
        const T* const image = static_cast<const T*>(p.X) + a.image * p.total + a.chunk * V;
        const int64_t whole = whole_rows(p, a, step, V), slots = p.slots;
        float mean[V], m2[V], n = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) mean[j] = m2[j] = 0.f;
        int64_t r = a.first;
        for (; r + (R - 1) * slots < whole; r += R * slots) {
            vec<T, V> x[R];
#pragma unroll
            for (int k = 0; k < R; ++k) x[k] = load_vec<T, V>(image + (r + k * slots) * step);
            const float f = R / (n + R), nf = n * f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float m = 0.f, q = 0.f;
#pragma unroll
                for (int k = 0; k < R; ++k) m += to_float(static_cast<T>(x[k][j]));
                m *= 1.f / R;
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    const float d = to_float(static_cast<T>(x[k][j])) - m;
                    q = fmaf(d, d, q);
                }
                const float d = m - mean[j];
                mean[j] = fmaf(d, f, mean[j]);
                m2[j] += fmaf(d * d, nf, q);
            }
            n += R;
        }
        for (; r < whole; r += slots) {
            const vec<T, V> x = load_vec<T, V>(image + r * step);
            n += 1.f;
            const float f = 1.f / n, nf = (n - 1.f) * f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = to_float(static_cast<T>(x[j])) - mean[j];
                mean[j] = fmaf(d, f, mean[j]);
                m2[j] = fmaf(d * d, nf, m2[j]);
            }
        }
        // the last super-row may end within a chunk: its places have a value more than the chunk's others
        const int more = r < a.last && a.active ? static_cast<int>(p.total - r * step - a.chunk * V) : 0;
        if (more > 0) {
            const vec<T, V> x = load_part<T, V>(image + r * step, more);
            const float f = 1.f / (n + 1.f), nf = n * f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = to_float(static_cast<T>(x[j])) - mean[j];
                mean[j] = j < more ? fmaf(d, f, mean[j]) : mean[j];
                m2[j] = j < more ? fmaf(d * d, nf, m2[j]) : m2[j];
            }
        }
        __syncthreads();
        s_n[threadIdx.x] = n + (more > 0 ? more * (1.f / 16.f) : 0.f);  // (a whole number and sixteenths: values of the last chunk)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            s_mean[j][threadIdx.x] = mean[j];
            s_m2[j][threadIdx.x] = m2[j];
        }
        __syncthreads();
        const int chunk0 = static_cast<int>(u % p.columns) * kBlock, count = min(across, p.chunks - chunk0) * V;
        float* const to = p.parts + 3 * ((a.image * p.blocks + a.block) * step + static_cast<int64_t>(chunk0) * V);
        // places lie chunk by chunk: place / V is the thread of slot 0, place % V the value of its chunk
        auto values = [&](int k, int place) {
            const float c = s_n[k * across + place / V], whole_n = floorf(c);
            return whole_n + (place % V < static_cast<int>((c - whole_n) * 16.f) ? 1.f : 0.f);
        };
        over_slots(count, p.slots, s_sum,
                   [&](int k, int place) {
                       const float c = values(k, place);
                       return make_float2(c, c * s_mean[place % V][k * across + place / V]);
                   },
                   [&](int place, float2 x) {
                       const float m = x.x > 0.f ? x.y / x.x : 0.f;
                       s_all[place] = m;
                       to[3 * place] = x.x;
                   });
        __syncthreads();
        over_slots(count, p.slots, s_sum,
                   [&](int k, int place) {
                       const int t = k * across + place / V;
                       const float d = s_mean[place % V][t] - s_all[place], cd = values(k, place) * d;
                       return make_float2(fmaf(cd, d, s_m2[place % V][t]), cd);
                   },
                   [&](int place, float2 x) {
                       // what the weighted sum's rounding left out of the mean
                       const float d = to[3 * place] > 0.f ? x.y / to[3 * place] : 0.f;
                       to[3 * place + 1] = s_all[place] + d;
                       to[3 * place + 2] = not_negative(fmaf(-x.y, d, x.x));
                   });
    }
}

// The statistics of a group of an image, from the blocks' parts.
__global__ __launch_bounds__(kBlock) void group_join_kernel(GroupParams p)
{
    __shared__ float2 s_part[kBlock / 64];
    const int64_t step = static_cast<int64_t>(p.C) * p.pixels_super;
    for (int64_t u = blockIdx.x; u < p.images * p.groups; u += gridDim.x) {
        const int64_t image = u / p.groups;
        const int c0 = static_cast<int>(u % p.groups) * p.width, each = p.width * p.pixels_super;
        const int64_t all = static_cast<int64_t>(p.blocks) * each;
        auto part = [&](int64_t i) {
            const int e = static_cast<int>(i % each);
            return p.parts + 3 * ((image * p.blocks + i / each) * step + e / p.width * static_cast<int64_t>(p.C) + c0 + e % p.width);
        };
        float2 x = make_float2(0.f, 0.f);
        for (int64_t i = threadIdx.x; i < all; i += kBlock) {
            const float* const at = part(i);
            x.x += at[0];
            x.y = fmaf(at[0], at[1], x.y);
        }
        x = block_sum(x, s_part);
        const float mean = x.y / x.x;
        float2 q = make_float2(0.f, 0.f);
        for (int64_t i = threadIdx.x; i < all; i += kBlock) {
            const float* const at = part(i);
            const float d = at[1] - mean;
            q.x += fmaf(at[0] * d, d, at[2]);
            q.y = fmaf(at[0], d, q.y);
        }
        q = block_sum(q, s_part);
        if (threadIdx.x == 0) {
            // what the weighted sum's rounding left out of the mean
            const float d = q.y / x.x;
            p.mean[u] = mean + d;
            p.rstd[u] = 1.f / sqrtf(not_negative(q.x / x.x - d * d) + p.eps);
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
    const int64_t step = static_cast<int64_t>(p.chunks) * V, slots = p.slots;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const GroupPlace a = group_place(p, u);
        const T* const from = static_cast<const T*>(p.X) + a.image * p.total + a.chunk * V;
        T* const to = static_cast<T*>(p.out) + a.image * p.total + a.chunk * V;
        const int64_t whole = whole_rows(p, a, step, V);
        GroupChannels<T, V> ch;
        ch.load(p, a, p.mean, p.rstd);
        auto result = [&](vec<T, V> x) {
            vec<T, V> y;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float z = fmaf((to_float(static_cast<T>(x[j])) - ch.mean[j]) * ch.rstd[j], ch.w[j], ch.b[j]);
                y[j] = from_float<T>(p.silu ? silu(z) : z);
            }
            return y;
        };
        int64_t r = a.first;
        for (; r + (R - 1) * slots < whole; r += R * slots) {
            vec<T, V> x[R];
#pragma unroll
            for (int k = 0; k < R; ++k) x[k] = load_vec<T, V>(from + (r + k * slots) * step);
#pragma unroll
            for (int k = 0; k < R; ++k) store_vec<T, V>(to + (r + k * slots) * step, result(x[k]));
        }
        for (; r < whole; r += slots) store_vec<T, V>(to + r * step, result(load_vec<T, V>(from + r * step)));
        const int more = r < a.last && a.active ? static_cast<int>(p.total - r * step - a.chunk * V) : 0;
        if (more > 0) store_part<T, V>(to + r * step, more, result(load_part<T, V>(from + r * step, more)));
    }
}

// Sums of dz xh and dz of every place of the super-rows, over a block's super-rows.
template <typename T, typename TG>
__global__ __launch_bounds__(kBlock) void group_sums_kernel(GroupParams p)
{
    constexpr int V = kChunk<T>, R = kGroupBatch;
    __shared__ float2 s_part[V][kBlock], s_sum[kBlock];
    const int64_t units = p.images * p.columns * p.blocks;
    const int64_t step = static_cast<int64_t>(p.chunks) * V, slots = p.slots;
    const int across = min(p.chunks, kBlock);
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const GroupPlace a = group_place(p, u);
        const T* const image = static_cast<const T*>(p.X) + a.image * p.total + a.chunk * V;
        const TG* const grad = static_cast<const TG*>(p.dY) + a.image * p.total + a.chunk * V;
        const int64_t whole = whole_rows(p, a, step, V);
        GroupChannels<T, V> ch;
        ch.load(p, a, p.mean_in, p.rstd_in);
        float dw[V], db[V];
#pragma unroll
        for (int j = 0; j < V; ++j) dw[j] = db[j] = 0.f;
        auto add = [&](vec<T, V> x, vec<TG, V> d, int n) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float xh = (to_float(static_cast<T>(x[j])) - ch.mean[j]) * ch.rstd[j];
                float dz = to_float(static_cast<TG>(d[j]));
                if (p.silu) dz *= silu_slope(fmaf(xh, ch.w[j], ch.b[j]));
                if (j < n) {  // (what stands in place of a value that is not there may be infinite)
                    dw[j] = fmaf(dz, xh, dw[j]);
                    db[j] += dz;
                }
            }
        };
        int64_t r = a.first;
        for (; r + (R - 1) * slots < whole; r += R * slots) {
            vec<T, V> x[R];
            vec<TG, V> d[R];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                x[k] = load_vec<T, V>(image + (r + k * slots) * step);
                d[k] = load_vec<TG, V>(grad + (r + k * slots) * step);
            }
#pragma unroll
            for (int k = 0; k < R; ++k) add(x[k], d[k], V);
        }
        for (; r < whole; r += slots) add(load_vec<T, V>(image + r * step), load_vec<TG, V>(grad + r * step), V);
        const int more = r < a.last && a.active ? static_cast<int>(p.total - r * step - a.chunk * V) : 0;
        if (more > 0) add(load_part<T, V>(image + r * step, more), load_part<TG, V>(grad + r * step, more), more);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < V; ++j) s_part[j][threadIdx.x] = make_float2(dw[j], db[j]);
        __syncthreads();
        const int chunk0 = static_cast<int>(u % p.columns) * kBlock, count = min(across, p.chunks - chunk0) * V;
        float* const to = p.parts + 2 * ((a.image * p.blocks + a.block) * step + static_cast<int64_t>(chunk0) * V);
        over_slots(count, p.slots, s_sum, [&](int k, int place) { return s_part[place % V][k * across + place / V]; },
                   [&](int place, float2 x) {
                       to[2 * place] = x.x;
                       to[2 * place + 1] = x.y;
                   });
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

// dweight, dbias: the sum of the images' sums, 32 columns a block, 8 threads a column.
__device__ __forceinline__ void group_weights(const GroupParams& p, int block)
{
    __shared__ float s[8][33];
    const int col = block * 32 + static_cast<int>(threadIdx.x & 31), first = threadIdx.x >> 5;
    float x = 0.f;
    if (col < 2 * p.C)
        for (int64_t i = first; i < p.images; i += 8) x += p.sums[i * 2 * p.C + col];
    s[first][threadIdx.x & 31] = x;
    __syncthreads();
    if (first == 0 && col < 2 * p.C) {
        for (int i = 1; i < 8; ++i) x += s[i][threadIdx.x & 31];
        (col < p.C ? p.dweight : p.dbias)[col < p.C ? col : col - p.C] = x;
    }
}

__global__ __launch_bounds__(kBlock) void group_weights_kernel(GroupParams p) { group_weights(p, blockIdx.x); }

// dx; the grid's last blocks add up the weights' gradients.
template <typename T, typename TG>
__global__ __launch_bounds__(kBlock) void group_grad_kernel(GroupParams p)
{
    constexpr int V = kChunk<T>, R = kGroupBatch;
    const int64_t units = p.images * p.columns * p.blocks;
    const uint32_t main = gridDim.x - p.weight_blocks;
    if (blockIdx.x >= main) return group_weights(p, blockIdx.x - main);
    for (int64_t u = blockIdx.x; u < units; u += main) {
        const GroupPlace a = group_place(p, u);
        const T* const image = static_cast<const T*>(p.X) + a.image * p.total + a.chunk * V;
        const TG* const grad = static_cast<const TG*>(p.dY) + a.image * p.total + a.chunk * V;
        TG* const to = static_cast<TG*>(p.out) + a.image * p.total + a.chunk * V;
        const int64_t step = static_cast<int64_t>(p.chunks) * V, slots = p.slots, whole = whole_rows(p, a, step, V);
        GroupChannels<T, V> ch;
        ch.load(p, a, p.mean_in, p.rstd_in);
        float mg[V], mx[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            mg[j] = p.means[2 * (a.image * p.groups + ch.group[j])];
            mx[j] = p.means[2 * (a.image * p.groups + ch.group[j]) + 1];
        }
        auto result = [&](vec<T, V> x, vec<TG, V> d) {
            vec<TG, V> y;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float xh = (to_float(static_cast<T>(x[j])) - ch.mean[j]) * ch.rstd[j];
                float dz = to_float(static_cast<TG>(d[j]));
                if (p.silu) dz *= silu_slope(fmaf(xh, ch.w[j], ch.b[j]));
                y[j] = from_float<TG>(ch.rstd[j] * (dz * ch.w[j] - mg[j] - xh * mx[j]));
            }
            return y;
        };
        int64_t r = a.first;
        for (; r + (R - 1) * slots < whole; r += R * slots) {
            vec<T, V> x[R];
            vec<TG, V> d[R];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                x[k] = load_vec<T, V>(image + (r + k * slots) * step);
                d[k] = load_vec<TG, V>(grad + (r + k * slots) * step);
            }
#pragma unroll
            for (int k = 0; k < R; ++k) store_vec<TG, V>(to + (r + k * slots) * step, result(x[k], d[k]));
        }
        for (; r < whole; r += slots)
            store_vec<TG, V>(to + r * step, result(load_vec<T, V>(image + r * step), load_vec<TG, V>(grad + r * step)));
        const int more = r < a.last && a.active ? static_cast<int>(p.total - r * step - a.chunk * V) : 0;
        if (more > 0)
            store_part<TG, V>(to + r * step, more,
                              result(load_part<T, V>(image + r * step, more), load_part<TG, V>(grad + r * step, more)));
    }
}

// Small groups: a block holds the values of one, kSmallEach a thread, in the order of the pixels.
constexpr int kSmallEach = 16;

// An image's group and the place of its value i of thread `threadIdx.x`.
struct SmallPlace {
    int64_t base;  // of the image, at the group's first channel
    int count, c0;

    __device__ __forceinline__ SmallPlace(const GroupParams& p, int64_t u)
    {
        c0 = static_cast<int>(u % p.groups) * p.width;
        base = u / p.groups * p.total + c0;
        count = static_cast<int>(p.total / p.C) * p.width;
    }
    __device__ __forceinline__ bool at(const GroupParams& p, int i, int64_t& where, int& c) const
    {
        const uint32_t e = i * kBlock + threadIdx.x;
        uint32_t pixel, k;
        divmod(e, p.div_width, pixel, k);
        where = base + static_cast<int64_t>(pixel) * p.C + k;
        c = c0 + static_cast<int>(k);
        return static_cast<int>(e) < count;
    }
};

template <typename T>
__global__ __launch_bounds__(kBlock) void group_small_kernel(GroupParams p)
{
    __shared__ float2 s_part[kBlock / 64];
    for (int64_t u = blockIdx.x; u < p.images * p.groups; u += gridDim.x) {
        const SmallPlace a(p, u);
        const T* const from = static_cast<const T*>(p.X);
        float x[kSmallEach];
        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kSmallEach; ++i) {
            int64_t where;
            int c;
            x[i] = 0.f;
            if (i * kBlock < a.count && a.at(p, i, where, c)) x[i] = to_float(from[where]);
            sum.x += x[i];
        }
        const float n = static_cast<float>(a.count);
        const float near = block_sum(sum, s_part).x / n;
        sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kSmallEach; ++i) {
            const float d = i * kBlock + static_cast<int>(threadIdx.x) < a.count ? x[i] - near : 0.f;
            sum.x += d;
            sum.y = fmaf(d, d, sum.y);
        }
        sum = block_sum(sum, s_part);
        const float d = sum.x / n, mean = near + d;  // (what the first sum's rounding left out)
        const float rstd = 1.f / sqrtf(not_negative(sum.y / n - d * d) + p.eps);
        if (threadIdx.x == 0 && p.mean) {
            p.mean[u] = mean;
            p.rstd[u] = rstd;
        }
#pragma unroll
        for (int i = 0; i < kSmallEach; ++i) {
            int64_t where;
            int c;
            if (i * kBlock < a.count && a.at(p, i, where, c)) {
                const float z = fmaf((x[i] - mean) * rstd, channel_value<1>(p.weight, p.weight_f32, c, 1.f),
                                     channel_value<1>(p.bias, p.weight_f32, c, 0.f));
                static_cast<T*>(p.out)[where] = from_float<T>(p.silu ? silu(z) : z);
            }
        }
    }
}

template <typename T, typename TG>
__global__ __launch_bounds__(kBlock) void group_small_grad_kernel(GroupParams p)
{
    __shared__ float2 s_part[kBlock / 64], s_value[kBlock * kSmallEach], s_sum[kBlock];
    for (int64_t u = blockIdx.x; u < p.images * p.groups; u += gridDim.x) {
        const SmallPlace a(p, u);
        const int64_t image = u / p.groups;
        const float mean = p.mean_in[u], rstd = p.rstd_in[u];
        float xh[kSmallEach], g[kSmallEach];
        float2 sum = make_float2(0.f, 0.f);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSmallEach; ++i) {
            int64_t where;
            int c;
            xh[i] = g[i] = 0.f;
            if (i * kBlock < a.count && a.at(p, i, where, c)) {
                xh[i] = (to_float(static_cast<const T*>(p.X)[where]) - mean) * rstd;
                const float w = channel_value<1>(p.weight, p.weight_f32, c, 1.f);
                float dz = to_float(static_cast<const TG*>(p.dY)[where]);
                if (p.silu) dz *= silu_slope(fmaf(xh[i], w, channel_value<1>(p.bias, p.weight_f32, c, 0.f)));
                g[i] = dz * w;
                s_value[i * kBlock + threadIdx.x] = make_float2(dz * xh[i], dz);
                sum.x += g[i];
                sum.y = fmaf(g[i], xh[i], sum.y);
            }
        }
        sum = block_sum(sum, s_part);
        const float n = static_cast<float>(a.count), mg = sum.x / n, mx = sum.y / n;
#pragma unroll
        for (int i = 0; i < kSmallEach; ++i) {
            int64_t where;
            int c;
            if (i * kBlock < a.count && a.at(p, i, where, c))
                static_cast<TG*>(p.out)[where] = from_float<TG>(rstd * (g[i] - mg - xh[i] * mx));
        }
        // each channel's sums over the pixels
        over_slots(p.width, a.count / p.width, s_sum, [&](int k, int c) { return s_value[k * p.width + c]; },
                   [&](int c, float2 x) {
                       p.sums[(image * 2) * p.C + a.c0 + c] = x.x;
                       p.sums[(image * 2 + 1) * p.C + a.c0 + c] = x.y;
                   });
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
    p.div_width = make_div(static_cast<uint32_t>(p.width));
    const int V = c.dtype == SCRAM_BF16 ? kChunk<uint16_t> : kChunk<float>;
    int common = V;
    while (c.channels % common) common /= 2;
    p.chunks = c.channels / common;
    p.pixels_super = V / common;
    p.slots = p.chunks < kBlock ? kBlock / p.chunks : 1;
    p.columns = (p.chunks + kBlock - 1) / kBlock;
    p.supers = (c.pixels + p.pixels_super - 1) / p.pixels_super;
    // blocks of an image: two per CU over all images, whole batches to each (4 x 256 x 256 x 128 bf16, the three kernels: 48.0
    // us with 512 blocks, 50.6 with 1024, 61.5 with 2048; batches of 8 instead of 4 52.7)
    int64_t blocks = 512 / (p.images < 512 ? p.images * p.columns : 512);
    if (blocks < 1) blocks = 1;
    const int64_t batch = int64_t(kGroupBatch) * p.slots;
    p.per = ((p.supers + blocks - 1) / blocks + batch - 1) / batch * batch;
    p.blocks = static_cast<int>((p.supers + p.per - 1) / p.per);
    return p;
}

// Whether a block holds a group: up to 4096 values, where all is small, as a group's short rows are read by a block each and
// share their lines with others'.  bf16, forward / gradients, held against not: 2 images of 8 x 8 x 256 5.1 / 7.9 us against
// 12.5 / 15.3; 2 MB in rows of 8 bytes 12.1 / 20.6 against 13.8 / 17.7, of 64 bytes 7.3 / 10.5 against 15.1 / 15.9; 4 MB in rows
// of 8 bytes 17.1 / 25.0 against 14.4 / 18.7, of 32 bytes 10.9 / 18.5 against 15.1 / 16.5; 67 MB of 64 bytes 122 / 197 against
// 64 / 90.
bool group_small(const GroupCall& c)
{
    const int64_t count = c.pixels * (c.channels / c.groups), bytes = c.dtype == SCRAM_BF16 ? 2 : 4;
    return count <= kBlock * kSmallEach && c.images * c.pixels * c.channels * bytes <= ((c.channels / c.groups) * bytes >= 32 ? 4 : 2) << 20;
}

uint32_t group_grid(int64_t units) { return static_cast<uint32_t>(units < (1 << 20) ? units : 1 << 20); }

size_t group_parts_bytes(const GroupParams& p, int each)
{
    return round256(size_t(p.images) * p.blocks * p.C * p.pixels_super * each * sizeof(float));
}

}  // namespace

size_t group_norm_workspace_bytes(const GroupCall& c)
{
    if (group_small(c)) return 0;
    const GroupParams p = group_params(c);
    return group_parts_bytes(p, 3) + round256(8 * size_t(p.images) * p.groups);
}

hipError_t launch_group_norm(const GroupCall& c, void* Y, float* mean, float* rstd, void* workspace, hipStream_t stream)
{
    GroupParams p = group_params(c);
    p.out = Y;
    p.parts = static_cast<float*>(workspace);
    p.mean = mean;
    p.rstd = rstd;
    if (!mean && !group_small(c)) {
        p.mean = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + group_parts_bytes(p, 3));
        p.rstd = p.mean + p.images * p.groups;
    }
    const dim3 grid(group_grid(p.images * p.columns * p.blocks)), joins(group_grid(p.images * p.groups)), block(kBlock);
    auto run = [&](auto type) {
        using T = decltype(type);
        if (group_small(c)) {
            hipLaunchKernelGGL(group_small_kernel<T>, joins, block, 0, stream, p);
            return hipGetLastError();
        }
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
    if (group_small(c)) return round256(8 * size_t(p.images) * p.C);
    return group_parts_bytes(p, 2) + round256(8 * size_t(p.images) * p.C) + round256(8 * size_t(p.images) * p.groups);
}

hipError_t launch_group_norm_backward(const GroupCall& c, const float* mean, const float* rstd, void* dX, float* dweight,
                                      float* dbias, void* workspace, hipStream_t stream)
{
    GroupParams p = group_params(c);
    p.out = dX;
    p.dweight = dweight;
    p.dbias = dbias;
    p.weight_blocks = static_cast<uint32_t>((2 * p.C + 31) / 32);
    p.mean_in = mean;
    p.rstd_in = rstd;
    unsigned char* const at = static_cast<unsigned char*>(workspace);
    p.parts = reinterpret_cast<float*>(at);
    p.sums = reinterpret_cast<float*>(at + (group_small(c) ? 0 : group_parts_bytes(p, 2)));
    p.means = reinterpret_cast<float*>(at + group_parts_bytes(p, 2) + round256(8 * size_t(p.images) * p.C));
    const dim3 grid(group_grid(p.images * p.columns * p.blocks)), joins(group_grid(p.images * p.groups)), block(kBlock);
    auto run = [&](auto type, auto grad) {
        using T = decltype(type);
        using TG = decltype(grad);
        if (group_small(c)) {
            hipLaunchKernelGGL((group_small_grad_kernel<T, TG>), joins, block, 0, stream, p);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            hipLaunchKernelGGL(group_weights_kernel, dim3(p.weight_blocks), block, 0, stream, p);
            return hipGetLastError();
        }
        hipLaunchKernelGGL((group_sums_kernel<T, TG>), grid, block, 0, stream, p);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(group_means_kernel, joins, block, 0, stream, p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        hipLaunchKernelGGL((group_grad_kernel<T, TG>), dim3(grid.x + p.weight_blocks), block, 0, stream, p);
        return hipGetLastError();
    };
    return c.dtype == SCRAM_F32 ? run(float{}, float{}) : c.grad_dtype == SCRAM_F32 ? run(uint16_t{}, float{}) : run(uint16_t{}, uint16_t{});
}

}  // namespace scram
