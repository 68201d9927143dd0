// Attention over every key: out_i = sum_j softmax_j(scale q_i.k_j + bias) v_j.
//
// 4 d operations for each pair of a query and a key, on the matrix cores; the
// rows are read once per tile of queries, so every call but those of a few
// queries is bound by computing.  A block holds 128 queries, 32 a wave, and
// passes over the keys once in tiles of 64 that it stages in LDS; maximum, sum
// and output of the softmax stay in registers.  Scores are formed transposed
// (scram_dense.h), so a query's statistics are a lane's own.
//
// Calls of few queries split the keys over blocks (`splits`); a second kernel
// joins their parts.  With a bias a block's queries are of one slice, and the
// part of the bias' plane that a tile of keys can meet is staged beside it.

#include "scram_dense.h"

namespace scram {
namespace {

constexpr int kRowsBlock = 128;  // queries of a block
// keys of a tile: 64, 32 where a row has 512 bytes (the tile's next rows wait in registers)
template <typename T, int D>
constexpr int kKeysTile = D * sizeof(T) > 256 ? 32 : 64;

struct DenseForward : DenseParams {
    void* out;
    float* part;       // [splits][all rows][D], then [splits][all rows][2]: maximum, sum
    int64_t all_rows;
    int tiles, splits;
    int window;        // floats of LDS for the bias
};

template <typename T, int D>
constexpr size_t forward_lds()
{
    using R = DenseRow<T, D>;
    return 2 * (kKeysTile<T, D> * R::kStride) + R::kSlack;
}

template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(kBlock) void dense_kernel(DenseForward p)
{
    using R = DenseRow<T, D>;
    constexpr int kKeys = kKeysTile<T, D>, U = kKeys / 32;
    extern __shared__ __align__(16) unsigned char lds[];
    unsigned char* const k_tile = lds;
    unsigned char* const v_tile = lds + kKeys * R::kStride;
    int* const s_place = reinterpret_cast<int*>(lds + forward_lds<T, D>());
    float* const s_bias = reinterpret_cast<float*>(s_place + kKeys);

    const uint32_t b = xcd_remap(blockIdx.x, gridDim.x);
    const int split = static_cast<int>(b % static_cast<uint32_t>(p.splits));
    const int tile = static_cast<int>(b / static_cast<uint32_t>(p.splits) % static_cast<uint32_t>(p.tiles));
    const int group = static_cast<int>(b / static_cast<uint32_t>(p.splits) / static_cast<uint32_t>(p.tiles));
    const int lane = threadIdx.x & 63, wave = wave_index(), m = lane & 31, h = lane >> 5;
    const int slice_k = p.per_group == 1 ? group / p.share : group;
    const int length = p.lengths ? min(max(p.lengths[slice_k], 0), p.nk) : p.nk;

    // the lane's query, and the first key behind those that it sees
    const int row = tile * kRowsBlock + wave * 32 + m;
    const bool live = row < p.rows;
    uint32_t head, q;
    divmod(static_cast<uint32_t>(min(row, p.rows - 1)), p.div_nq, head, q);
    const int slice = group * p.per_group + static_cast<int>(head);
    const int begin = p.origin ? min(max(p.origin[slice], 0), p.nk - p.nq) : p.first;
    const int at = begin + static_cast<int>(q);
    const int end = live ? (p.causal ? min(length, at + 1) : length) : 0;
    // of the block's keys: up to the last that any of its queries sees
    int last = length;
    if (p.causal) {
        __shared__ int s_end[4];
        int e = end;
        for (int k = 32; k >= 1; k >>= 1) e = max(e, __shfl_xor(e, k));
        if (lane == 0) s_end[wave] = e;
        __syncthreads();
        last = max(max(s_end[0], s_end[1]), max(s_end[2], s_end[3]));
    }
    const int all = (last + kKeys - 1) / kKeys;
    const int t0 = static_cast<int>(static_cast<int64_t>(all) * split / p.splits);
    const int t1 = static_cast<int>(static_cast<int64_t>(all) * (split + 1) / p.splits);

    const int64_t out_row = static_cast<int64_t>(group) * p.rows + row;
    uint4 qf[R::kSteps];
    load_operand<T, D>(p.Q, live ? out_row : static_cast<int64_t>(group) * p.rows, h, qf);

    f32x16_t o[R::kColumns];
#pragma unroll
    for (int c = 0; c < R::kColumns; ++c) o[c] = f32x16_t(0.f);
    float top = -INFINITY, sum = 0.f;

    DenseLoad<T, D, kKeys> kl, vl;
    const int64_t k_row = static_cast<int64_t>(slice_k) * p.nk;
    if (t0 < t1) {
        kl.load(p.K, k_row + t0 * kKeys, last - t0 * kKeys);
        vl.load(p.V, k_row + t0 * kKeys, last - t0 * kKeys);
    }
    BiasWindow<T> win{};
    int my_place = 0;
    if constexpr (BIAS) my_place = BiasWindow<T>::place(p, at);
    for (int t = t0; t < t1; ++t) {
        const int k0 = t * kKeys;
        kl.store(k_tile);
        vl.store(v_tile);
        if constexpr (BIAS) {
            const int k1 = min(k0 + kKeys, p.nk) - 1;
            const int q0 = tile * kRowsBlock, q1 = min(q0 + kRowsBlock, p.rows) - 1;
            win.stage(p, slice % p.plane.rows, begin + q0, begin + q1, k0, k1, s_bias);
            if (threadIdx.x < kKeys) s_place[threadIdx.x] = BiasWindow<T>::place(p, min(k0 + static_cast<int>(threadIdx.x), k1));
        }
        __syncthreads();
        if (t + 1 < t1) {
            kl.load(p.K, k_row + k0 + kKeys, last - k0 - kKeys);
            vl.load(p.V, k_row + k0 + kKeys, last - k0 - kKeys);
        }
        f32x16_t s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[u] = f32x16_t(0.f);
#pragma unroll
            for (int c = 0; c < R::kSteps; ++c)
                s[u] = mma<T>(row_operand<T, D>(k_tile, 32 * u + tile_row<T>(m), h, c), qf[c], s[u]);
        }
        float most = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = 32 * u + tile_slot<T>(i) + tile_half<T>() * h;
                float x = s[u][i] * p.scale2;
                if constexpr (BIAS) x = fmaf(s[u][i], p.scale2, s_bias[s_place[key] - my_place - win.base]);
                s[u][i] = x;
            }
        if (!__all(end >= k0 + kKeys))
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[u][i] = k0 + 32 * u + tile_slot<T>(i) + tile_half<T>() * h < end ? s[u][i] : -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, s[u][i]);
        most = fmaxf(most, __shfl_xor(most, 32));
        const float next = fmaxf(top, most);
        const float shift = next == -INFINITY ? 0.f : next;  // no key yet: every weight is 0
        if (__any(next > top)) {
            const float keep = __builtin_amdgcn_exp2f(top - shift);
            sum *= keep;
#pragma unroll
            for (int c = 0; c < R::kColumns; ++c) o[c] *= keep;
        }
        top = next;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[u][i] = __builtin_amdgcn_exp2f(s[u][i] - shift);
                sum += s[u][i];
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < R::kRowSteps; ++r) {
                const uint4 w = as_operand<T>(s[u], r);
#pragma unroll
                for (int c = 0; c < R::kColumns; ++c) o[c] = mma<T>(column_operand<T, D>(v_tile, 32 * u, r, c), w, o[c]);
            }
        __syncthreads();
    }
    sum += __shfl_xor(sum, 32);
    if (!live) return;
    if (p.splits > 1) {
        const int64_t at_part = static_cast<int64_t>(split) * p.all_rows + out_row;
        float* const ml = p.part + static_cast<int64_t>(p.splits) * p.all_rows * D + 2 * at_part;
        if (h == 0) {
            ml[0] = top;
            ml[1] = sum;
        }
        if (sum == 0.f) return;  // a part without a key is not read
        float* const to = p.part + at_part * D;
#pragma unroll
        for (int c = 0; c < R::kColumns; ++c)
#pragma unroll
            for (int i = 0; i < (D < 32 ? 2 : 4); ++i)
                *reinterpret_cast<float4*>(to + 32 * c + 8 * i + 4 * h) =
                    make_float4(o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]);
        return;
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    T* const to = static_cast<T*>(p.out) + out_row * D;
#pragma unroll
    for (int c = 0; c < R::kColumns; ++c)
#pragma unroll
        for (int i = 0; i < (D < 32 ? 2 : 4); ++i) {
            vec<T, 4> x;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = from_float<T>(o[c][4 * i + j] * inv);
            store_vec<T, 4>(to + 32 * c + 8 * i + 4 * h, x);
        }
}

// Joins the parts of the splits: a thread takes four channels of a row.
template <typename T, int D>
__global__ __launch_bounds__(kBlock) void dense_join_kernel(DenseForward p)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x;
    const int64_t row = i / (D / 4);
    if (row >= p.all_rows) return;
    const int c = static_cast<int>(i % (D / 4)) * 4;
    const float* const ml = p.part + static_cast<int64_t>(p.splits) * p.all_rows * D + 2 * row;
    float top = -INFINITY;
    for (int s = 0; s < p.splits; ++s) top = fmaxf(top, ml[2 * s * p.all_rows]);
    float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < p.splits; ++s) {
        const float one = ml[2 * s * p.all_rows + 1];
        if (one == 0.f) continue;  // no key
        const float w = __builtin_amdgcn_exp2f(ml[2 * s * p.all_rows] - top);
        sum = fmaf(w, one, sum);
        const float4 x = *reinterpret_cast<const float4*>(p.part + (s * p.all_rows + row) * D + c);
        o[0] = fmaf(w, x.x, o[0]);
        o[1] = fmaf(w, x.y, o[1]);
        o[2] = fmaf(w, x.z, o[2]);
        o[3] = fmaf(w, x.w, o[3]);
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    vec<T, 4> y;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = from_float<T>(o[j] * inv);
    store_vec<T, 4>(static_cast<T*>(p.out) + row * D + c, y);
}

// Splits of the keys: blocks of fewer than two per CU leave CUs idle, and a part is worth a block from two tiles on.
int dense_splits(const DenseParams& p)
{
    const int64_t blocks = int64_t(p.groups) * ((p.rows + kRowsBlock - 1) / kRowsBlock);
    const int64_t tiles = (p.nk + 63) / 64;
    int64_t n = 512 / blocks;
    if (n > tiles / 2) n = tiles / 2;
    return n < 1 ? 1 : static_cast<int>(n);
}

}  // namespace

// Most places of the bias' plane between the ends of 128 queries against 128 keys.
int64_t dense_bias_window(int Hk, int Wk)
{
    if (Hk == 1) return 256;
    // n positions over rows that are 2 Wk - 1 places apart
    auto span = [&](int64_t n) { return n + (Wk - 1) * ((n - 1) / Wk + 1); };
    return 2 * span(128);
}

size_t dense_workspace_bytes(const DenseCall& c)
{
    const DenseParams p = dense_params(c);
    const int n = dense_splits(p);
    return n == 1 ? 0 : size_t(n) * p.groups * p.rows * (c.g.d + 2) * sizeof(float);
}

uint64_t dense_blocks(const DenseCall& c)
{
    const DenseParams p = dense_params(c);
    return uint64_t(p.groups) * ((p.rows + kRowsBlock - 1) / kRowsBlock) * dense_splits(p);
}

hipError_t launch_dense(int dtype, const DenseCall& c, void* out, void* workspace, hipStream_t stream, hipEvent_t start,
                        hipEvent_t stop)
{
    DenseForward p{};
    static_cast<DenseParams&>(p) = dense_params(c);
    p.out = out;
    p.part = static_cast<float*>(workspace);
    p.all_rows = int64_t(p.groups) * p.rows;
    p.tiles = (p.rows + kRowsBlock - 1) / kRowsBlock;
    p.splits = dense_splits(p);
    p.window = c.bias ? static_cast<int>(dense_bias_window(c.g.Hk, c.g.Wk)) : 0;
    const uint64_t blocks = uint64_t(p.groups) * p.tiles * p.splits;
    return dispatch_value(dtype, c.g.d, hipErrorInvalidValue, [&](auto type, auto width) {
        using T = std::conditional_t<std::is_same<decltype(type), float>::value, float, uint16_t>;
        constexpr int D = decltype(width)::value;
        const size_t lds = forward_lds<T, D>() + (c.bias ? (kKeysTile<T, D> + p.window) * sizeof(float) : 0);
        const hipEvent_t end = p.splits == 1 ? stop : nullptr;
        hipError_t e = c.bias ? launch_dense_kernel(dense_kernel<T, D, true>, blocks, lds, stream, start, end, p)
                              : launch_dense_kernel(dense_kernel<T, D, false>, blocks, lds, stream, start, end, p);
        if (e != hipSuccess || p.splits == 1) return e;
        return launch_dense_kernel(dense_join_kernel<T, D>, (p.all_rows * (D / 4) + kBlock - 1) / kBlock, 0, stream, nullptr, stop, p);
    });
}

}  // namespace scram
