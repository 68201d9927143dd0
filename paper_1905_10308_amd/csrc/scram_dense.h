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

// Rows of D elements of T.  In LDS they lie side by side, each row's 16-byte chunks in an order of its own (chunk c of row r at
// place c ^ order(r)), so that sixteen rows' chunks c, and four rows' chunks 4 k .. 4 k + 3, lie in different banks.
template <typename T, int D>
struct DenseRow {
    static constexpr int kBytes = D * static_cast<int>(sizeof(T));
    static constexpr int kChunks = kBytes / 16;
    static constexpr int kSteps = kBytes / 32;              // steps of a product's inner index over the channels
    static constexpr int kInner = 32 / static_cast<int>(sizeof(T));  // that a step takes: 16 (bf16) or 8
    static constexpr int kRowSteps = 32 / kInner;           // steps of a product whose inner index runs over a tile's 32 rows
    static constexpr int kColumns = D < 32 ? 1 : D / 32;    // tiles of 32 channels (of 16: half of one)

    static __device__ __forceinline__ int order(int r)
    {
        if constexpr (kChunks == 2) return (r >> 3) & 1;
        if constexpr (kChunks == 4) return (r >> 2) & 3;
        if constexpr (kChunks == 8) return ((r & 2) << 1) | ((r >> 2) & 3);
        return ((r & 3) << 2) | ((r >> 2) & 3);
    }
    static __device__ __forceinline__ int place(int r, int c) { return r * kBytes + 16 * (c ^ order(r)); }
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

// Step s of the registers x of a 32 x 32 result as the right operand of a product whose inner index runs over its rows.  bf16: as
// two parts that add up to them to 2^-16, each rounded to the nearest (half a step of 2^-8 of the value, then of what that left).
// With the first alone what that rounds off shows beside the results' own rounding: they are off by 2.1 .. 2.5e-3 of their size
// (most the gradients', whose ds nearly cancel), with both by the 1.6 .. 1.7e-3 that rounding them leaves in any arithmetic.  The
// second part costs a product and three operations a weight: 4 slices of 128 x 128, 64 channels, 418 us for 314, 16 of 32 x 32
// with a bias 17.0 for 15.4, the gradients of 16 of 64 x 64 with a bias 726 for 652.
template <typename T>
struct RightOperand {
    uint4 high, low;
};

__device__ __forceinline__ uint32_t rest2(float a, float b, uint32_t high)
{
    return pack2(a - __uint_as_float(high << 16), b - __uint_as_float(high & 0xFFFF0000u));
}

template <typename T>
__device__ __forceinline__ RightOperand<T> as_operand(const f32x16_t& x, int s)
{
    RightOperand<T> w;
    if constexpr (sizeof(T) == 2) {
        w.high = make_uint4(pack2(x[8 * s], x[8 * s + 1]), pack2(x[8 * s + 2], x[8 * s + 3]), pack2(x[8 * s + 4], x[8 * s + 5]),
                            pack2(x[8 * s + 6], x[8 * s + 7]));
        w.low = make_uint4(rest2(x[8 * s], x[8 * s + 1], w.high.x), rest2(x[8 * s + 2], x[8 * s + 3], w.high.y),
                           rest2(x[8 * s + 4], x[8 * s + 5], w.high.z), rest2(x[8 * s + 6], x[8 * s + 7], w.high.w));
    } else {
        w.high = make_uint4(__float_as_uint(x[4 * s]), __float_as_uint(x[4 * s + 1]), __float_as_uint(x[4 * s + 2]),
                            __float_as_uint(x[4 * s + 3]));
    }
    return w;
}

template <typename T>
__device__ __forceinline__ f32x16_t mma(uint4 a, const RightOperand<T>& w, f32x16_t c)
{
    c = mma<T>(a, w.high, c);
    if constexpr (sizeof(T) == 2) c = mma<T>(a, w.low, c);
    return c;
}

// 16 bytes of a staged row: those of step s for lane half h.
template <typename T, int D>
__device__ __forceinline__ uint4 row_operand(const unsigned char* tile, int row, int h, int s)
{
    return *reinterpret_cast<const uint4*>(tile + DenseRow<T, D>::place(row, 2 * s + h));
}

using lds_bytes = __attribute__((address_space(3))) const unsigned char*;

// A lane's places in 32 staged rows, kept for all the tiles that it reads: `at` is the bytes of a tile behind the first.
template <typename T, int D>
struct TileReader {
    using R = DenseRow<T, D>;
    using words = uint32_t __attribute__((ext_vector_type(4)));
    lds_bytes base;
    int row_x, column_x;  // places of a lane's first chunks in a tile; those of the others follow by exclusive or

    __device__ __forceinline__ void set(const unsigned char* tile)
    {
        const int lane = threadIdx.x & 63, m = lane & 31, h = lane >> 5, i = lane & 15;
        base = (lds_bytes)tile;
        row_x = R::place(tile_row<T>(m), h);
        column_x = R::place(8 * h + (i >> 2), (D < 32 ? 0 : (lane & 16) >> 3) + ((i & 2) >> 1)) + 8 * (i & 1);
    }
    // Keeps the compiler from holding every chunk's place in a register of its own throughout a loop, which spills.
    __device__ __forceinline__ void renew()
    {
        asm volatile("" : "+v"(row_x));
        if constexpr (sizeof(T) == 2) asm volatile("" : "+v"(column_x));
    }
    // Left operand of products over the channels, step s: rows in the order of tile_row.
    __device__ __forceinline__ uint4 row(int s, int at) const
    {
        using lds_words = __attribute__((address_space(3))) const words*;
        return __builtin_bit_cast(uint4, *(lds_words)(base + (row_x ^ 32 * s) + at));
    }
    // Left operand of a product whose inner index runs over the rows (step s of 32 of them) and whose rows are channels 32 o ..
    // 32 o + 31 (of 16 channels: each twice).  bf16: the transposing load hands lane i of each 16 the element e of the 8 bytes
    // that lane 4 e + i / 4 addresses.
    __device__ __forceinline__ uint4 column(int s, int o, int at) const
    {
        if constexpr (sizeof(T) == 2) {
            using lds_v4 = __attribute__((address_space(3))) bf16x4_t*;
            constexpr int kFourDown = R::kChunks > 2 ? 16 : 0;  // how the order differs four rows further down
            const lds_bytes from = base + (at + 16 * s * R::kBytes);
            const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_v4)(from + (column_x ^ 64 * o)));
            const bf16x4_t hi =
                __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_v4)(from + ((column_x ^ 64 * o ^ kFourDown) + 4 * R::kBytes)));
            return __builtin_bit_cast(uint4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            using lds_word = __attribute__((address_space(3))) const uint32_t*;
            const int lane = threadIdx.x & 63, h = lane >> 5;
            const int c = 8 * o + ((lane & (D < 32 ? 15 : 31)) >> 2), r = 8 * (s & 1) + 4 * h;
            const lds_bytes from = base + at + 8 * (s & ~1) * R::kBytes + 4 * (lane & 3);
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = *(lds_word)(from + R::place(r + j, c));
            return make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
};

// N rows of a tile on their way from memory to LDS, past the registers of a block of THREADS threads: a wave's load writes its
// lanes' 16 bytes one after another from the place in m0 on, so the order of a row's chunks is that in which lanes fetch them.
// The rows from `live` (> 0) on are row live - 1 again, whose products count nowhere.  Issued in assembly, since for the
// builtin the compiler would wait for the rows on their way before it reads any others; wait() waits for them, and for the
// other waves' a barrier.  (The compiler writes m0, as an operand; a scalar write of it and the load keep an instruction between.)
template <typename T, int D, int N, int THREADS>
struct DenseStage {
    using R = DenseRow<T, D>;
    static constexpr int kTotal = N * R::kBytes / 1024;  // loads of a wave
    static constexpr int kWaves = THREADS / 64, kEach = (kTotal + kWaves - 1) / kWaves;
    static_assert(N * R::kBytes % 1024 == 0, "whole loads");

    static __device__ __forceinline__ uint32_t offset(int load, int live)
    {
        const int i = load * 64 + static_cast<int>(threadIdx.x & 63), r = i / R::kChunks;
        return min(r, live - 1) * R::kBytes + 16 * ((i % R::kChunks) ^ R::order(r));
    }
    static __device__ __forceinline__ void load(const void* rows, int64_t row0, int live, unsigned char* tile)
    {
        const unsigned char* const from = static_cast<const unsigned char*>(rows) + row0 * R::kBytes;
        const uint32_t to = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_bytes)tile));
        const int wave = wave_index();
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int load = j * kWaves + wave;
            if (kTotal % kWaves == 0 || load < kTotal)
                asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                             :
                             : "{m0}"(to + 1024u * load), "v"(offset(load, live)), "s"(from)
                             : "memory");
        }
    }
    static __device__ __forceinline__ void wait() { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); }
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

// Place of a raster index on the bias' plane, as of an offset from index 0.
__device__ __forceinline__ int bias_place(const DenseParams& p, int at)
{
    uint32_t y, x;
    divmod(static_cast<uint32_t>(at), p.div_wk, y, x);
    return static_cast<int>(y) * p.plane.width + static_cast<int>(x);
}

// A window of the bias' plane on its way to LDS, by a block's threads or a share of them: queries q0 .. q1 against keys k0 .. k1.
// Places rise with the raster index, so that they lie between those of the runs' ends: the window's start is
// place(k0) - place(q1), and a pair's index its place less that.
template <typename T>
struct BiasStage {
    float x[2];
    const T* from;
    int n;

    __device__ __forceinline__ void load(const DenseParams& p, int head, int q0, int q1, int k0, int k1, int thread, int threads)
    {
        const int base = bias_place(p, k0) - bias_place(p, q1);
        from = static_cast<const T*>(p.bias) + head * p.plane.size + p.plane.origin + base;
        n = bias_place(p, k1) - bias_place(p, q0) - base + 1;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = thread + j * threads;
            x[j] = i < n ? to_float(from[i]) : 0.f;
        }
    }
    __device__ __forceinline__ void store(float* window, int thread, int threads) const
    {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = thread + j * threads;
            if (i < n) window[i] = bias_base2(x[j]);
        }
        for (int i = thread + 2 * threads; i < n; i += threads) window[i] = bias_base2(to_float(from[i]));
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

// ---------------------------------------------------------------------------
// Blocks that hold queries and pass over keys (the forward pass, and the query side of the gradients)
// ---------------------------------------------------------------------------

constexpr int kQueryThreads = 512;

struct DenseQueries : DenseParams {
    int64_t all_rows;
    int tiles, splits;  // of a group's rows; of the keys over blocks
    int window;         // floats of LDS for the bias, of each slice in a tile
    int window_shift;   // log2 of the shares of a block's threads that stage them
    int buffers;        // steps whose rows fit in LDS: with two, the next one's are stored while this one's are read
    int runs;           // whether grid rows are whole vectors of tile_half rows: those of keys, which begin at a multiple, lie in one
};

// Keys of a wave in a block's step: 64, which halves the barriers, 32 where two steps' rows would not fit in LDS.
constexpr int wave_keys(int row_bytes, int kw) { return kw * row_bytes <= 512 ? 64 : 32; }
template <typename T, int D, int KW>
constexpr int kWaveKeys = wave_keys(D * sizeof(T), KW);

// Bytes of a step's rows in LDS.
template <typename T, int D, int KW>
constexpr size_t kTileBytes = 2 * (KW * kWaveKeys<T, D, KW> * DenseRow<T, D>::kBytes);

// What a block of queries may take of LDS in arrays of its own (3104 bytes in the gradients' kernel: maxima, sums and means of its
// waves' rows, their last keys; 288 in the forward's: those last, and the vote on another pass).
constexpr size_t kQueryStatic = 6144 - 64;

// The rest: staged rows, with a bias the places of their keys and its windows (floats of a step; behind the last a vector's), and in
// the place of all these at the end what the waves of the same queries join.
constexpr size_t query_lds(int d, int elem_bytes, int kw, int buffers, int64_t bias_floats)
{
    const size_t row = size_t(d) * elem_bytes, rows = 2 * size_t(kw) * wave_keys(int(row), kw) * row;
    const size_t steps = buffers * (rows + bias_floats * sizeof(float)) + (bias_floats ? 64 : 0);
    const size_t join = 8 * 64 * sizeof(float) * (16 * (d < 32 ? 1 : d / 32) + 2);
    return steps > join ? steps : join;
}

// s scale2 + bias for a 32 x 32 tile: places are those of the rows of the tile (4 a place), mine the lane's, so that a row's
// value lies SIGN (its place - mine) bytes into the window.
template <typename T, int SIGN>
__device__ __forceinline__ void add_bias(f32x16_t& s, float scale2, const float* window, const int* places, int mine, int h, bool runs)
{
    constexpr int N = tile_half<T>();
    if (runs) {  // a vector's rows lie side by side on the grid
#pragma unroll
        for (int g = 0; g < 16; g += N) {
            const int at = SIGN * (places[tile_slot<T>(g) + N * h] - mine);
#pragma unroll
            for (int j = 0; j < N; ++j) s[g + j] = fmaf(s[g + j], scale2, bias_at(window, at + 4 * SIGN * j));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], scale2, bias_at(window, SIGN * (places[tile_slot<T>(i) + N * h] - mine)));
    }
}

// A block's rows of queries and its passes over the keys.  Its eight waves share the rows (32 each) and the keys: KW of them
// take different keys of the same rows.
template <typename T, int D, bool BIAS, int KW>
struct QueryBlock {
    using R = DenseRow<T, D>;
    static constexpr int kRows = 32 * 8 / KW, kEach = kWaveKeys<T, D, KW>, kKeys = KW * kEach;

    const DenseQueries& p;
    unsigned char* lds;
    int* s_places;
    int bias_floats;  // of a step: places of its keys, windows
    int lane, m, h, wave, qw, kw;
    int split, tile, group, slice_k, row;
    bool live;
    uint32_t head;
    int end, least, most_keys;  // first key behind those that the lane's query sees; of the wave's queries the fewest and most
    int last, t0, t1;           // the block's keys, its steps
    int64_t out_row;
    float scale2;
    int my_at, my_end, my_place;
    int q0, q1, my_window, my_thread, my_threads;
    using Stage = DenseStage<T, D, kKeys, kQueryThreads>;
    BiasStage<T> bl;
    TileReader<T, D> reader;  // of the wave's keys
    static constexpr int kValues = kKeys * R::kBytes;  // bytes from a step's keys to its values

    __device__ __forceinline__ int begin_of(int slice) const { return p.origin ? min(max(p.origin[slice], 0), p.nk - p.nq) : p.first; }

    __device__ __forceinline__ QueryBlock(const DenseQueries& params, unsigned char* memory) : p(params), lds(memory)
    {
        s_places = reinterpret_cast<int*>(lds + p.buffers * kTileBytes<T, D, KW>);
        bias_floats = kKeys + p.per_group * p.window;
        const uint32_t b = xcd_remap(blockIdx.x, gridDim.x);
        split = static_cast<int>(b % static_cast<uint32_t>(p.splits));
        tile = static_cast<int>(b / static_cast<uint32_t>(p.splits) % static_cast<uint32_t>(p.tiles));
        if (p.causal) tile = p.tiles - 1 - tile;  // those of many keys first
        group = static_cast<int>(b / static_cast<uint32_t>(p.splits) / static_cast<uint32_t>(p.tiles));
        lane = threadIdx.x & 63;
        m = lane & 31;
        h = lane >> 5;
        wave = wave_index();
        qw = wave % (8 / KW);
        kw = wave / (8 / KW);
        slice_k = p.per_group == 1 ? group / p.share : group;
        const int length = p.lengths ? min(max(p.lengths[slice_k], 0), p.nk) : p.nk;
        row = tile * kRows + qw * 32 + m;
        live = row < p.rows;
        out_row = static_cast<int64_t>(group) * p.rows + row;
        uint32_t q;
        divmod(static_cast<uint32_t>(min(row, p.rows - 1)), p.div_nq, head, q);
        const int begin = begin_of(group * p.per_group + static_cast<int>(head)), at = begin + static_cast<int>(q);
        end = live ? (p.causal ? min(length, at + 1) : length) : 0;
        least = live ? end : p.nk;
        most_keys = end;
        for (int k = 16; k >= 1; k >>= 1) {
            least = min(least, __shfl_xor(least, k));
            most_keys = max(most_keys, __shfl_xor(most_keys, k));
        }
        least = __builtin_amdgcn_readfirstlane(least);
        most_keys = __builtin_amdgcn_readfirstlane(most_keys);
        last = length;
        if (p.causal) {
            __shared__ int s_end[8];
            if (lane == 0) s_end[wave] = most_keys;
            __syncthreads();
            last = s_end[0];
            for (int w = 1; w < 8 / KW; ++w) last = max(last, s_end[w]);
        }
        const int all = (last + kKeys - 1) / kKeys;
        t0 = static_cast<int>(static_cast<int64_t>(all) * split / p.splits);
        t1 = static_cast<int>(static_cast<int64_t>(all) * (split + 1) / p.splits);
        scale2 = p.scale2;
        reader.set(lds + kw * kEach * R::kBytes);
        if constexpr (BIAS) {
            // a tile of several slices (whole ones then) has a window for each, which a share of the threads stages
            q0 = p.per_group == 1 ? tile * kRows : 0;
            q1 = min(q0 + kRows, p.nq) - 1;
            my_threads = kQueryThreads >> p.window_shift;
            my_window = static_cast<int>(threadIdx.x) / my_threads;
            my_thread = static_cast<int>(threadIdx.x) % my_threads;
            // the place of a step's first key less that of the slice's last query is its window's start
            my_at = bias_place(p, at);
            my_end = bias_place(p, begin + q1) + (p.per_group > 1 ? static_cast<int>(head) * p.window : 0);
        }
    }

    __device__ __forceinline__ int64_t from_row() const { return live ? out_row : static_cast<int64_t>(group) * p.rows; }

    // Scores largest where the rows' products are: a negative scale is taken into the queries.
    __device__ __forceinline__ void positive_scale(uint4 (&qf)[R::kSteps])
    {
        if (scale2 < 0.f) {
            scale2 = -scale2;
            constexpr uint32_t kSign = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
#pragma unroll
            for (int c = 0; c < R::kSteps; ++c) qf[c] = make_uint4(qf[c].x ^ kSign, qf[c].y ^ kSign, qf[c].z ^ kSign, qf[c].w ^ kSign);
        }
        // (a key that is not seen has a score of minus infinity, and a weight of 0 by it; the others' weights, whose products stay
        // under 2^128, differ by less than 2^-21)
        if (scale2 == 0.f) scale2 = 0x1p-149f;
    }

    // The rows of step t, on their way to their buffer.
    __device__ __forceinline__ void fetch(int t)
    {
        const int k0 = t * kKeys;
        const int64_t k_row = static_cast<int64_t>(slice_k) * p.nk + k0;
        unsigned char* const tiles = lds + buffer(t) * kTileBytes<T, D, KW>;
        Stage::load(p.K, k_row, last - k0, tiles);
        Stage::load(p.V, k_row, last - k0, tiles + kValues);
    }
    __device__ __forceinline__ int buffer(int t) const { return p.buffers > 1 ? (t - t0) & 1 : 0; }
    // The bias of step t: from memory, and to LDS.
    __device__ __forceinline__ void fetch_bias(int t)
    {
        if constexpr (BIAS) {
            if (p.per_group == 1) {  // (numbers that are the same for all lanes)
                const int begin = begin_of(group), k0 = t * kKeys;
                bl.load(p, group % p.plane.rows, begin + q0, begin + q1, k0, min(k0 + kKeys, p.nk) - 1, threadIdx.x, kQueryThreads);
            } else if (my_window < p.per_group) {
                const int slice = group * p.per_group + my_window, begin = begin_of(slice), k0 = t * kKeys;
                bl.load(p, slice % p.plane.rows, begin + q0, begin + q1, k0, min(k0 + kKeys, p.nk) - 1, my_thread, my_threads);
            }
        }
    }
    __device__ __forceinline__ void store_bias(int t)
    {
        if constexpr (BIAS) {
            int* const places = s_places + buffer(t) * bias_floats;
            if (my_window < p.per_group)
                bl.store(reinterpret_cast<float*>(places + kKeys) + my_window * p.window, my_thread, my_threads);
            const int k0 = t * kKeys, k1 = min(k0 + kKeys, p.nk) - 1;
            if (threadIdx.x < kKeys) places[threadIdx.x] = 4 * bias_place(p, min(k0 + static_cast<int>(threadIdx.x), k1));
        }
    }

    // One pass: step(at, places, from, k0) for every 32 keys of the wave's, keys k0 .. of the slice, staged `at` bytes behind what
    // `reader` begins at, a constant; `places` are those of the step's keys, of which these are from ..
    template <typename F>
    __device__ __forceinline__ void pass(F&& step)
    {
        const lds_bytes first_base = reader.base;
        if (t0 < t1) {
            fetch(t0);
            fetch_bias(t0);
            store_bias(t0);
        }
        Stage::wait();
        __syncthreads();
        for (int t = t0; t < t1; ++t) {
            const int k0 = t * kKeys + kw * kEach;
            const bool more = t + 1 < t1;
            if (more && p.buffers > 1) fetch(t + 1);
            if (more) fetch_bias(t + 1);
            if constexpr (BIAS) my_place = 4 * (my_at + bias_place(p, t * kKeys) - my_end);
            const int* const places = s_places + buffer(t) * bias_floats;
            reader.base = first_base + buffer(t) * static_cast<int>(kTileBytes<T, D, KW>);
            reader.renew();
            if (k0 < most_keys) step(std::integral_constant<int, 0>{}, places, kw * kEach, k0);
            if constexpr (kEach == 64) {
                __builtin_amdgcn_sched_barrier(0);  // (both at once would need more registers)
                reader.renew();
                if (k0 + 32 < most_keys) step(std::integral_constant<int, 32 * R::kBytes>{}, places, kw * kEach + 32, k0 + 32);
            }
            if (p.buffers == 1) {
                __syncthreads();
                if (more) fetch(t + 1);
            }
            if (more) store_bias(t + 1);
            Stage::wait();
            __syncthreads();
        }
        reader.base = first_base;
    }

    // Transposed products of 32 staged rows with a lane's row.
    __device__ __forceinline__ f32x16_t products(int at, const uint4 (&x)[R::kSteps]) const
    {
        f32x16_t s(0.f);
#pragma unroll
        for (int c = 0; c < R::kSteps; ++c) s = mma<T>(reader.row(c, at), x[c], s);
        return s;
    }
    // The scores of products s of the keys k0 .. (from .. of the step's) in base 2 (RAW: before the scale), minus infinity where
    // a key is not seen.
    template <bool RAW>
    __device__ __forceinline__ void scores(f32x16_t& s, const int* places, int from, int k0) const
    {
        if constexpr (BIAS)
            add_bias<T, 1>(s, scale2, reinterpret_cast<const float*>(places + kKeys), places + from, my_place, h, p.runs);
        else if constexpr (!RAW)
            s *= scale2;
        if (k0 + 32 > least) {
            asm volatile("");  // (not for every step, by selects)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = k0 + tile_slot<T>(i) + tile_half<T>() * h < end ? s[i] : -INFINITY;
        }
    }
};

// How a call's queries are dealt to blocks: the waves that share a block's keys, splits of the keys.  split: whether blocks may
// share a tile's keys.  Times below: bf16, 64 channels, forward, unless said otherwise.
struct QueryPlan {
    int key_waves;
    int64_t blocks;
};

constexpr int kMostSplits = 256;

inline QueryPlan query_plan(const DenseCall& c, int elem_bytes, bool split, DenseQueries& p)
{
    const int bytes = c.g.d * elem_bytes;
    auto room = [&](int kw, int slices, int buffers, int blocks = 1) {
        const int64_t keys = kw * wave_keys(bytes, kw), rows = 256 / kw;
        const int64_t windows = c.bias ? slices * bias_window(int(rows), int(keys), c.g.Hk, c.g.Wk) + keys : 0;
        return blocks * (query_lds(c.g.d, elem_bytes, kw, buffers, windows) + kQueryStatic) <= kLdsMost;
    };
    // A tile that holds the queries of all slices of a key slice, each with a window: the keys are read once (64 slices of two
    // queries on 4 of 64 x 64 keys 16.4 us, 17.4 with a tile a slice; 128 of one on 8 of 32 x 32 12.3 and 13.0).
    const bool together = c.bias && p.share > 1 && int64_t(p.share) * p.nq <= 32 && p.share <= 16 && bytes <= 256 && room(8, p.share, 1);
    if (!c.bias || together) {
        p.per_group = p.share;
        p.groups = c.g.S / p.share;
        p.rows = p.nq * p.share;
    }
    auto blocks = [&](int kw) { return int64_t(p.groups) * ((p.rows + 256 / kw - 1) / (256 / kw)); };
    // The more queries a block holds the fewer times keys are staged, but every CU needs a block.  Slices of 32 x 32, with
    // 8 / 4 / 2 waves to a step's keys: 8 of them 12.1 / 16.3 / 18.0 us, 16 17.3 / 15.4 / 21.5, 32 29.7 / 22.7 / 20.0.
    int kw = 8;
    if (p.rows > 32 && blocks(4) >= 256) kw = 4;
    if (p.rows > 64 && blocks(2) >= 256) kw = 2;
    if (bytes > 256 && kw == 8) kw = 4;  // (a step of eight waves' rows of 512 bytes does not fit)
    if (!room(kw, together ? p.share : 1, 1)) kw = 2;  // (which any window fits beside that a call may have: kBiasWindowMost)
    // The next step's rows are on their way while this one's are met: 2500 queries of 128 channels 120 us, with one buffer 131.
    // Two blocks a CU do as much for each other, and more where their registers let them (300 / 1024 slices of 48 queries
    // on 1008 keys 23.1 / 55 us, 32.4 / 69 with two buffers; 256 of them, a block a CU, 21.1 and 19.5).
    p.buffers = room(kw, together ? p.share : 1, 2) ? 2 : 1;
    if (!c.bias && bytes <= 128 && blocks(kw) > 256 && !room(kw, 1, 2, 2) && room(kw, 1, 1, 2)) p.buffers = 1;
    p.tiles = (p.rows + 256 / kw - 1) / (256 / kw);
    const int keys = kw * wave_keys(bytes, kw);
    if (c.bias) p.window = int(bias_window(256 / kw, keys, c.g.Hk, c.g.Wk));
    while ((1 << p.window_shift) < p.per_group && c.bias) ++p.window_shift;
    // one place then serves a vector's keys: 16 slices of 64 x 64 141 us, with a place a key 150
    p.runs = c.g.Wk % (elem_bytes == 2 ? 8 : 4) == 0;
    // fewer blocks than CUs leave CUs idle: 8 slices of 4 queries on 64 x 64 keys 14.5 us in the 16 parts of one step each with
    // their join, 12.7 in 8, 23.7 whole; 4 slices of 16 x 16 queries on as many 14.9 in 4 and 24.0.  Where the blocks fill the
    // CUs the join only costs (32 slices of 32 x 32: 22.4 us, 35.3 in two parts)
    const int64_t steps = (p.nk + keys - 1) / keys;
    int64_t n = split ? 256 / blocks(kw) : 1;
    if (n > steps) n = steps;
    if (n > kMostSplits) n = kMostSplits;
    p.splits = n < 1 ? 1 : int(n);
    p.all_rows = int64_t(p.groups) * p.rows;
    return QueryPlan{kw, blocks(kw) * p.splits};
}

// Bytes of LDS of a block of queries.
template <typename T, int D, bool BIAS, int KW>
size_t query_block_lds(const DenseQueries& p)
{
    constexpr int keys = KW * kWaveKeys<T, D, KW>;
    return query_lds(D, sizeof(T), KW, p.buffers, BIAS ? keys + int64_t(p.per_group) * p.window : 0);
}

// All bytes of a plan's block.
inline size_t query_plan_lds(const DenseQueries& p, const DenseCall& c, int elem_bytes, int kw)
{
    const int64_t keys = kw * wave_keys(c.g.d * elem_bytes, kw);
    return query_lds(c.g.d, elem_bytes, kw, p.buffers, c.bias ? keys + int64_t(p.per_group) * p.window : 0) + kQueryStatic;
}

// f(BIAS, KW) of a plan
template <typename T, int D, typename F>
hipError_t query_dispatch(bool biased, int key_waves, F&& f)
{
    auto with = [&](auto b) {
        if (key_waves == 2) return f(b, std::integral_constant<int, 2>{});
        if constexpr (D * sizeof(T) <= 256)
            if (key_waves == 8) return f(b, std::integral_constant<int, 8>{});
        return f(b, std::integral_constant<int, 4>{});
    };
    return biased ? with(std::true_type{}) : with(std::false_type{});
}

// Launch of kBlock threads with LDS of a size known at the launch.
template <int THREADS = kBlock, typename P>
hipError_t launch_dense_kernel(void (*kernel)(P), uint64_t blocks, size_t lds, hipStream_t st, hipEvent_t start, hipEvent_t stop,
                               const P& p)
{
    if (blocks == 0 || blocks > 0xFFFFFFFFull / THREADS) return hipErrorInvalidConfiguration;
    if (lds > 64 * 1024) {
        // (the most that any call takes: a number for all threads of the program, which another may set before the launch)
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 static_cast<int>(kLdsMost - kQueryStatic));
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
