// Tiles of the attention over every key (scram_dense.hip and
// scram_dense_backward.hip).
//
// Every product runs on the matrix cores as 32 x 32 tiles: bf16 rows with
// their 32 x 32 x 16 instruction, fp32 rows with the fp32 one (32 x 32 x 2), so
// that fp32 products lose nothing.  A chain of products (scores, then their
// softmax times the values) never leaves the registers: the first product is
// taken transposed, so that a lane holds one query's scores of 16 keys of the
// tile, and those registers, packed in their order, are the right operand of
// the second product.  The instruction's rows and the order in which it wants
// the second product's inner index differ, so the rows of the first product's
// left operand are dealt in an order (tile_row) that makes them agree.
//
// Everything here lives in an unnamed namespace, like scram_device.h.

#pragma once

#include "scram_rows.h"

namespace scram {
namespace {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kMost = 3.402823466e38f;

// Bias on the plane of offsets: offset (dy, dx) of a key from its query, each from 1 - the axis' length on, stands at place
// place(key) - place(query) + origin with place(y, x) = y (2 W - 1) + x.
struct DensePlane {
    int width, origin, rows;  // 2 W - 1, the place of offset 0, heads in the table
    int64_t size;             // places of a head
};

struct DenseParams {
    const void* Q;
    const void* K;
    const void* V;
    const void* bias;        // nullable [plane.rows, plane.size]
    const int32_t* lengths;  // nullable [key slices]
    const int32_t* origin;   // nullable [S]
    int share;               // slices of queries to a slice of keys
    int groups, rows;        // runs of query rows that read one slice of keys, rows of each
    int per_group;           // slices of queries in a group (1 or share)
    int nq, nk;
    int causal, first;
    Div div_nq, div_wk;
    DensePlane plane;
    float scale, scale2;     // the softmax's temperature, and in base 2
};

// Rows of D elements of T in LDS, kPad bytes apart.
template <typename T, int D>
struct DenseRow {
    static constexpr int kBytes = D * static_cast<int>(sizeof(T));
    static constexpr int kStride = kBytes + 16;             // 16 lanes' vectors of 16 bytes then lie in different banks
    static constexpr int kChunks = kBytes / 16;
    static constexpr int kSteps = kBytes / 32;              // steps of a product's inner index over the channels
    static constexpr int kInner = 32 / static_cast<int>(sizeof(T));  // that a step takes: 16 (bf16) or 8
    static constexpr int kRowSteps = 32 / kInner;           // steps of a product whose inner index runs over a tile's 32 rows
    static constexpr int kColumns = D < 32 ? 1 : D / 32;    // tiles of 32 channels (of 16: half of one)
    static constexpr int kSlack = 64 * static_cast<int>(sizeof(T));  // bytes that transposed reads may pass the last row by
};

// The wave's place in its block, as a number that the compiler knows to be the same for all lanes.
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6); }

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2_t));
}

// The row of its 32 that lane index m (of 32) of a left operand reads, so that register i of lane half h of the result holds
// row tile_slot<T>(i) + tile_half<T>() * h.
template <typename T>
__device__ __forceinline__ int tile_row(int m)
{
    return sizeof(T) == 2 ? (m & 0x13) | ((m & 4) << 1) | ((m & 8) >> 1) : m;
}
template <typename T>
constexpr __device__ int tile_slot(int i)
{
    return sizeof(T) == 2 ? 16 * (i >> 3) + (i & 7) : 8 * (i >> 2) + (i & 3);
}
template <typename T>
constexpr __device__ int tile_half()
{
    return sizeof(T) == 2 ? 8 : 4;
}

// c + a b for a step of the inner index: 16 (bf16) or 8 (fp32) of it, 16 bytes of each operand a lane.
template <typename T>
__device__ __forceinline__ f32x16_t mma(uint4 a, uint4 b, f32x16_t c)
{
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    } else {
        const f32x4_t x = __builtin_bit_cast(f32x4_t, a), y = __builtin_bit_cast(f32x4_t, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], c, 0, 0, 0);
        return c;
    }
}

// Step s of the registers x of a 32 x 32 result as the right operand of a product whose inner index runs over its rows.  bf16:
// rounded to the nearest, off by at most half a step (2^-8 of the value).
template <typename T>
__device__ __forceinline__ uint4 as_operand(const f32x16_t& x, int s)
{
    if constexpr (sizeof(T) == 2) {
        return make_uint4(pack2(x[8 * s], x[8 * s + 1]), pack2(x[8 * s + 2], x[8 * s + 3]), pack2(x[8 * s + 4], x[8 * s + 5]),
                          pack2(x[8 * s + 6], x[8 * s + 7]));
    } else {
        return make_uint4(__float_as_uint(x[4 * s]), __float_as_uint(x[4 * s + 1]), __float_as_uint(x[4 * s + 2]),
                          __float_as_uint(x[4 * s + 3]));
    }
}

// 16 bytes of a staged row: those of step s for lane half h.
template <typename T, int D>
__device__ __forceinline__ uint4 row_operand(const unsigned char* tile, int row, int h, int s)
{
    return *reinterpret_cast<const uint4*>(tile + row * DenseRow<T, D>::kStride + 32 * s + 16 * h);
}

// Left operand of a product whose inner index runs over staged rows (row0 on, step s of 32 of them) and whose rows are channels
// 32 o .. 32 o + 31.  bf16: the transposing load hands lane i of each 16 the element e of the 8 bytes that lane 4 e + i / 4
// addresses.
template <typename T, int D>
__device__ __forceinline__ uint4 column_operand(const unsigned char* tile, int row0, int s, int o)
{
    using R = DenseRow<T, D>;
    const int lane = threadIdx.x & 63, h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
        const int i = lane & 15;
        const unsigned char* const at =
            tile + (row0 + 16 * s + 8 * h + (i >> 2)) * R::kStride + 64 * o + 2 * (lane & 16) + 8 * (i & 3);
        using lds_v4 = __attribute__((address_space(3))) bf16x4_t*;
        const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_v4)(at));
        const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_v4)(at + 4 * R::kStride));
        return __builtin_bit_cast(uint4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = *reinterpret_cast<const uint32_t*>(tile + (row0 + 8 * s + 4 * h + j) * R::kStride + 128 * o + 4 * (lane & 31));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// N rows of a tile on their way from memory to LDS, in the registers of a block of kBlock threads; rows from `live` on are zeros.
template <typename T, int D, int N>
struct DenseLoad {
    using R = DenseRow<T, D>;
    static constexpr int kTotal = N * R::kChunks;
    static constexpr int kEach = (kTotal + kBlock - 1) / kBlock;
    uint4 x[kEach];

    __device__ __forceinline__ void load(const void* rows, int64_t row0, int live)
    {
        const unsigned char* const from = static_cast<const unsigned char*>(rows) + row0 * R::kBytes;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int c = i * kBlock + static_cast<int>(threadIdx.x);
            x[i] = make_uint4(0u, 0u, 0u, 0u);
            if (c / R::kChunks < live && c < kTotal) x[i] = *reinterpret_cast<const uint4*>(from + 16 * c);
        }
    }
    __device__ __forceinline__ void store(unsigned char* tile) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int c = i * kBlock + static_cast<int>(threadIdx.x);
            if (c < kTotal) *reinterpret_cast<uint4*>(tile + c / R::kChunks * R::kStride + 16 * (c % R::kChunks)) = x[i];
        }
    }
};

// The same for a block of THREADS threads; the rows from `live` (> 0) on are row live - 1 again, whose products count nowhere.
template <typename T, int D, int N, int THREADS>
struct DenseStage {
    using R = DenseRow<T, D>;
    static constexpr int kTotal = N * R::kChunks;
    static constexpr int kEach = (kTotal + THREADS - 1) / THREADS;
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    words x[kEach];

    __device__ __forceinline__ void load(const void* rows, int64_t row0, int live)
    {
        const unsigned char* const from = static_cast<const unsigned char*>(rows) + row0 * R::kBytes;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int c = i * THREADS + static_cast<int>(threadIdx.x);
            const uint32_t at = min(c / R::kChunks, live - 1) * R::kBytes + 16 * (c % R::kChunks);
            x[i] = *reinterpret_cast<const words*>(from + at);
        }
    }
    __device__ __forceinline__ void store(unsigned char* tile) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int c = i * THREADS + static_cast<int>(threadIdx.x);
            if (kTotal % THREADS == 0 || c < kTotal)
                *reinterpret_cast<words*>(tile + c / R::kChunks * R::kStride + 16 * (c % R::kChunks)) = x[i];
        }
    }
};

// A row of D elements as the right operand of products over its channels.
template <typename T, int D>
__device__ __forceinline__ void load_operand(const void* rows, int64_t row, int h, uint4 (&x)[DenseRow<T, D>::kSteps])
{
    const unsigned char* const from = static_cast<const unsigned char*>(rows) + row * DenseRow<T, D>::kBytes + 16 * h;
#pragma unroll
    for (int s = 0; s < DenseRow<T, D>::kSteps; ++s) x[s] = *reinterpret_cast<const uint4*>(from + 32 * s);
}

__device__ __forceinline__ float bias_base2(float b)
{
    // in base 2; finite where it was (a mask of the type's lowest value hides a key behind any other, but not all of them)
    return fabsf(b) <= kMost ? fminf(fmaxf(b * kLog2e, -kMost), kMost) : b;
}

// A block's window of the bias plane in LDS: the places of a run of queries against a run of keys.  Places rise with the
// raster index, so that they lie between those of the runs' ends.
template <typename T>
struct BiasWindow {
    int base;  // place(key) - place(query) - base is the index

    static __device__ __forceinline__ int place(const DenseParams& p, int at)
    {
        uint32_t y, x;
        divmod(static_cast<uint32_t>(at), p.div_wk, y, x);
        return static_cast<int>(y) * p.plane.width + static_cast<int>(x);
    }
    // queries q0 .. q1, keys k0 .. k1
    __device__ __forceinline__ void stage(const DenseParams& p, int head, int q0, int q1, int k0, int k1, float* window)
    {
        const T* const table = static_cast<const T*>(p.bias) + head * p.plane.size + p.plane.origin;
        base = place(p, k0) - place(p, q1);
        const int n = place(p, k1) - place(p, q0) - base + 1;
        for (int i = threadIdx.x; i < n; i += kBlock) window[i] = bias_base2(to_float(table[base + i]));
    }
};

// Place of a raster index on the bias' plane, as of an offset from index 0.
__device__ __forceinline__ int bias_place(const DenseParams& p, int at)
{
    uint32_t y, x;
    divmod(static_cast<uint32_t>(at), p.div_wk, y, x);
    return static_cast<int>(y) * p.plane.width + static_cast<int>(x);
}

__device__ __forceinline__ int bias_place_or(bool biased, const DenseParams& p, int at) { return biased ? bias_place(p, at) : 0; }

// A window of the bias' plane on its way to LDS, by a block's THREADS threads: queries q0 .. q1 against keys k0 .. k1.  Places
// rise with the raster index, so that they lie between those of the runs' ends: the window's start is place(k0) - place(q1),
// and a pair's index its place less that.
template <typename T, int THREADS>
struct BiasStage {
    float x[2];
    const T* from;
    int n;

    __device__ __forceinline__ void load(const DenseParams& p, int head, int q0, int q1, int k0, int k1)
    {
        const int base = bias_place(p, k0) - bias_place(p, q1);
        from = static_cast<const T*>(p.bias) + head * p.plane.size + p.plane.origin + base;
        n = bias_place(p, k1) - bias_place(p, q0) - base + 1;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = static_cast<int>(threadIdx.x) + j * THREADS;
            x[j] = i < n ? to_float(from[i]) : 0.f;
        }
    }
    __device__ __forceinline__ void store(float* window) const
    {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = static_cast<int>(threadIdx.x) + j * THREADS;
            if (i < n) window[i] = bias_base2(x[j]);
        }
        for (int i = static_cast<int>(threadIdx.x) + 2 * THREADS; i < n; i += THREADS) window[i] = bias_base2(to_float(from[i]));
    }
};

__device__ __forceinline__ float bias_at(const float* window, int bytes)
{
    return *reinterpret_cast<const float*>(reinterpret_cast<const unsigned char*>(window) + bytes);
}

// Most places between the ends of a run of q queries against one of k keys.
inline int64_t bias_window(int q, int k, int Hk, int Wk)
{
    if (Hk == 1) return q + k;
    // n positions over rows that are 2 Wk - 1 places apart
    auto span = [&](int64_t n) { return n + (Wk - 1) * ((n - 1) / Wk + 1); };
    return span(q) + span(k);
}

// Launch of kBlock threads with LDS of a size known at the launch.
template <int THREADS = kBlock, typename P>
hipError_t launch_dense_kernel(void (*kernel)(P), uint64_t blocks, size_t lds, hipStream_t st, hipEvent_t start, hipEvent_t stop,
                               const P& p)
{
    if (blocks == 0 || blocks > 0xFFFFFFFFull / THREADS) return hipErrorInvalidConfiguration;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 static_cast<int>(lds));
        if (e != hipSuccess) return e;
    }
    if (start || stop)
        hipExtLaunchKernelGGL(kernel, dim3(blocks), dim3(THREADS), lds, st, start, stop, 0, p);
    else
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(THREADS), lds, st, p);
    return hipGetLastError();
}

// The parameters that the forward and the gradients share.
inline DenseParams dense_params(const DenseCall& c)
{
    DenseParams p{};
    p.Q = c.Q;
    p.K = c.K;
    p.V = c.V;
    p.bias = c.bias;
    p.lengths = c.lengths;
    p.origin = c.origin;
    p.share = c.g.S / c.key_slices;
    p.nq = c.g.Hq * c.g.Wq;
    p.nk = c.g.Hk * c.g.Wk;
    // without a bias the query slices of a key slice are one run of rows: few queries of many heads share a tile
    p.per_group = c.bias ? 1 : p.share;
    p.groups = c.g.S / p.per_group;
    p.rows = p.nq * p.per_group;
    p.causal = c.causal ? 1 : 0;
    p.first = c.first;
    p.div_nq = make_div(static_cast<uint32_t>(p.nq));
    p.div_wk = make_div(static_cast<uint32_t>(c.g.Wk));
    const int64_t width = 2 * int64_t(c.g.Wk) - 1;
    p.plane = DensePlane{static_cast<int>(width), static_cast<int>((c.g.Hk - 1) * width + c.g.Wk - 1), c.bias_rows,
                         (2 * int64_t(c.g.Hk) - 1) * width};
    p.scale = c.scale;
    p.scale2 = c.scale * kLog2e;
    return p;
}

}  // namespace
}  // namespace scram
