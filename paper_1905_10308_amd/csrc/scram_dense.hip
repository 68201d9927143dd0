// Attention over every key: out_i = sum_j softmax_j(scale q_i.k_j + bias) v_j.
//
// 4 d operations for each pair of a query and a key, on the matrix cores; the
// rows are read once per tile of queries, so every call but those of a few
// queries is bound by computing: by the vector units' exponentials and sums
// beside the products, which eight waves of a block overlap.  A wave holds 32
// queries and passes over keys that the block stages in LDS; maximum, sum and
// output of the softmax stay in registers.  Scores are formed transposed
// (scram_dense.h), so a query's statistics are a lane's own.
//
// The waves of a block share its queries (32, 64 or 128) and its keys: KW of
// them take different keys of the same queries and join at the end.  Calls of
// few queries also split the keys over blocks; a second kernel joins those
// parts.  With a bias the part of its plane that the staged keys can meet is
// staged beside them.

#include "scram_dense.h"

namespace scram {
namespace {

constexpr int kThreads = 512;

struct DenseForward : DenseParams {
    void* out;
    float* part;       // [splits][all rows][D], then [splits][all rows][2]: maximum, sum
    int64_t all_rows;
    int tiles, splits;
    int window;        // floats of LDS for the bias, of each slice in a tile
};

// Keys of a wave in a block's step: 64, 32 where a row has 512 bytes or the block's queries are few.
template <typename T, int D, int KW>
constexpr int kWaveKeys = KW > 2 || D * sizeof(T) > 256 ? 32 : 64;

// Bytes of a step's rows in LDS, and whether two steps' fit: the next one's are then stored while this one's are read.
template <typename T, int D, int KW>
constexpr size_t kTileBytes = 2 * (KW * kWaveKeys<T, D, KW> * DenseRow<T, D>::kStride);
template <typename T, int D, int KW>
constexpr int kBuffers = kTileBytes<T, D, KW> <= 72 * 1024 ? 2 : 1;

template <typename T, int D, int KW>
constexpr size_t forward_lds()
{
    using R = DenseRow<T, D>;
    constexpr size_t tiles = kBuffers<T, D, KW> * kTileBytes<T, D, KW> + R::kSlack;
    constexpr size_t join = (8 - 8 / KW) * 64 * sizeof(float) * (16 * R::kColumns + 2);  // all waves but those that write
    return tiles > join ? tiles : join;
}

template <typename T, int D, bool BIAS, int KW>
__global__ __launch_bounds__(kThreads, D * sizeof(T) > 128 || (BIAS && D * sizeof(T) > 64) || KW == 8 ? 2 : 4) void dense_kernel(DenseForward p)
{
    using R = DenseRow<T, D>;
    constexpr int kRows = 32 * 8 / KW, kEach = kWaveKeys<T, D, KW>, kKeys = KW * kEach, kBuffered = kBuffers<T, D, KW>;
    // in bf16 without a bias the scale and the shift enter the exponential's argument in one step (a certain key's weight is
    // then off 1 by a rounding, which its rounding to bf16 takes back)
    constexpr bool kFold = sizeof(T) == 2 && !BIAS;
    extern __shared__ __align__(16) unsigned char lds[];
    const int bias_floats = kKeys + p.per_group * p.window;  // of a step: places of its keys, windows
    int* const s_places = reinterpret_cast<int*>(lds + forward_lds<T, D, KW>());

    const uint32_t b = xcd_remap(blockIdx.x, gridDim.x);
    const int split = static_cast<int>(b % static_cast<uint32_t>(p.splits));
    int tile = static_cast<int>(b / static_cast<uint32_t>(p.splits) % static_cast<uint32_t>(p.tiles));
    if (p.causal) tile = p.tiles - 1 - tile;  // those of many keys first
    const int group = static_cast<int>(b / static_cast<uint32_t>(p.splits) / static_cast<uint32_t>(p.tiles));
    const int lane = threadIdx.x & 63, wave = wave_index(), m = lane & 31, h = lane >> 5;
    const int qw = wave % (8 / KW), kw = wave / (8 / KW);
    const int slice_k = p.per_group == 1 ? group / p.share : group;
    const int length = p.lengths ? min(max(p.lengths[slice_k], 0), p.nk) : p.nk;

    // the lane's query, and the first key behind those that it sees
    const int row = tile * kRows + qw * 32 + m;
    const bool live = row < p.rows;
    uint32_t head, q;
    divmod(static_cast<uint32_t>(min(row, p.rows - 1)), p.div_nq, head, q);
    const int slice = group * p.per_group + static_cast<int>(head);
    const int begin = p.origin ? min(max(p.origin[slice], 0), p.nk - p.nq) : p.first;
    const int at = begin + static_cast<int>(q);
    const int end = live ? (p.causal ? min(length, at + 1) : length) : 0;
    // of the wave's queries the fewest and most keys; of the block's most
    int least = live ? end : p.nk, most_keys = end;
    for (int k = 16; k >= 1; k >>= 1) {
        least = min(least, __shfl_xor(least, k));
        most_keys = max(most_keys, __shfl_xor(most_keys, k));
    }
    least = __builtin_amdgcn_readfirstlane(least);
    most_keys = __builtin_amdgcn_readfirstlane(most_keys);
    int last = length;
    if (p.causal) {
        __shared__ int s_end[8];
        if (lane == 0) s_end[wave] = most_keys;
        __syncthreads();
        last = s_end[0];
        for (int w = 1; w < 8 / KW; ++w) last = max(last, s_end[w]);
    }
    const int all = (last + kKeys - 1) / kKeys;
    const int t0 = static_cast<int>(static_cast<int64_t>(all) * split / p.splits);
    const int t1 = static_cast<int>(static_cast<int64_t>(all) * (split + 1) / p.splits);

    const int64_t out_row = static_cast<int64_t>(group) * p.rows + row;
    uint4 qf[R::kSteps];
    load_operand<T, D>(p.Q, live ? out_row : static_cast<int64_t>(group) * p.rows, h, qf);
    float scale2 = p.scale2;
    if (kFold && scale2 < 0.f) {  // so that the largest score has the largest product
        scale2 = -scale2;
#pragma unroll
        for (int c = 0; c < R::kSteps; ++c) qf[c] = make_uint4(qf[c].x ^ 0x80008000u, qf[c].y ^ 0x80008000u, qf[c].z ^ 0x80008000u, qf[c].w ^ 0x80008000u);
    }
    if (kFold && scale2 == 0.f) scale2 = 1e-37f;  // (a key that is not seen has a score of minus infinity, and a weight of 0 by it)

    f32x16_t o[R::kColumns];
    // Weights are exp2(score - shift).  Any shift will do that is near a query's largest score; the largest of its first keys
    // is, but for queries that far larger ones await.  So nothing is scaled on the way: the largest score is kept beside, and
    // where it leaves the shift too far behind, the block passes over its keys again.
    float sum, shift = 0.f, most;
    bool first;
    // with a bias: 4 (place of the query, less its slice's window)
    int my_place = 0;

    // the 32 keys from k0 on, staged from row `from` on
    auto step = [&](const unsigned char* tiles, const int* places, int k0, int from, bool choose) {
        f32x16_t s(0.f);
#pragma unroll
        for (int c = 0; c < R::kSteps; ++c) s = mma<T>(row_operand<T, D>(tiles, from + tile_row<T>(m), h, c), qf[c], s);
        if constexpr (BIAS) {
            const float* const window = reinterpret_cast<const float*>(places + kKeys);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[i] = fmaf(s[i], scale2, bias_at(window, places[from + tile_slot<T>(i) + tile_half<T>() * h] - my_place));
        } else if constexpr (!kFold) {
            s *= scale2;
        }
        if (k0 + 32 > least) {
            asm volatile("");  // (not for every step, by selects)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = k0 + tile_slot<T>(i) + tile_half<T>() * h < end ? s[i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, s[i]);
        if (choose && first) {
            first = false;
            const float x = fmaxf(most, __shfl_xor(most, 32));
            shift = x == -INFINITY ? 0.f : kFold ? x * scale2 : x;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] = __builtin_amdgcn_exp2f(kFold ? fmaf(s[i], scale2, -shift) : s[i] - shift);
            sum += s[i];
        }
#pragma unroll
        for (int r = 0; r < R::kRowSteps; ++r) {
            const uint4 w = as_operand<T>(s, r);
#pragma unroll
            for (int c = 0; c < R::kColumns; ++c)
                o[c] = mma<T>(column_operand<T, D>(tiles + kKeys * R::kStride, from, r, c), w, o[c]);
        }
    };

    DenseStage<T, D, kKeys, kThreads> kl, vl;
    BiasStage<T, kThreads> bl;
    const int64_t k_row = static_cast<int64_t>(slice_k) * p.nk;
    const int q0 = p.per_group == 1 ? tile * kRows : 0, q1 = min(q0 + kRows, p.nq) - 1;  // of a slice in the tile
    auto first_of = [&](int s) { return p.origin ? min(max(p.origin[s], 0), p.nk - p.nq) : p.first; };
    auto fetch = [&](int t) {
        const int k0 = t * kKeys;
        kl.load(p.K, k_row + k0, last - k0);
        vl.load(p.V, k_row + k0, last - k0);
        if constexpr (BIAS)
            if (p.per_group == 1)
                bl.load(p, group % p.plane.rows, begin + q0, begin + q1, k0, min(k0 + kKeys, p.nk) - 1);
    };
    auto store = [&](int t) {
        const int at = kBuffered > 1 ? t & 1 : 0;
        unsigned char* const tiles = lds + at * kTileBytes<T, D, KW>;
        kl.store(tiles);
        vl.store(tiles + kKeys * R::kStride);
        if constexpr (BIAS) {
            int* const places = s_places + at * bias_floats;
            float* const window = reinterpret_cast<float*>(places + kKeys);
            const int k0 = t * kKeys, k1 = min(k0 + kKeys, p.nk) - 1;
            if (p.per_group == 1) {
                bl.store(window);
            } else {  // the tile holds whole slices, each with a window of its own
                for (int w = 0; w < p.per_group; ++w) {
                    const int s = group * p.per_group + w;
                    bl.load(p, s % p.plane.rows, first_of(s) + q0, first_of(s) + q1, k0, k1);
                    bl.store(window + w * p.window);
                }
            }
            if (threadIdx.x < kKeys) places[threadIdx.x] = 4 * bias_place(p, min(k0 + static_cast<int>(threadIdx.x), k1));
        }
    };
    const int my_end = bias_place_or(BIAS, p, begin + q1), my_at = bias_place_or(BIAS, p, at);
    for (int pass = 0;; ++pass) {
#pragma unroll
        for (int c = 0; c < R::kColumns; ++c) o[c] = f32x16_t(0.f);
        sum = 0.f;
        most = -INFINITY;
        first = pass == 0;
        if (t0 < t1) {
            fetch(t0);
            store(t0);
        }
        __syncthreads();
        for (int t = t0; t < t1; ++t) {
            const int k0 = t * kKeys + kw * kEach, at_buffer = kBuffered > 1 ? t & 1 : 0;
            const unsigned char* const tiles = lds + at_buffer * kTileBytes<T, D, KW>;
            const int* const places = s_places + at_buffer * bias_floats;
            if (t + 1 < t1) fetch(t + 1);
            // of the step's window: the place of its first key less that of the slice's last query is its start
            if constexpr (BIAS)
                my_place = 4 * (my_at + bias_place(p, t * kKeys) - my_end - static_cast<int>(head) * p.window * (p.per_group > 1));
            const int steps = min(kEach, most_keys - k0);
#pragma unroll 1
            for (int u = 0; u < steps; u += 32) step(tiles, places, k0 + u, kw * kEach + u, pass == 0);
            if (kBuffered == 1) __syncthreads();
            if (t + 1 < t1) store(t + 1);
            __syncthreads();
        }
        if (pass == 1) break;
        most = fmaxf(most, __shfl_xor(most, 32));
        if (kFold && most != -INFINITY) most *= scale2;
        float worst = fabsf(sum);
#pragma unroll
        for (int c = 0; c < R::kColumns; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) worst = fmaxf(worst, (D >= 32 || i < 8) ? fabsf(o[c][i]) : 0.f);
        const bool again = live && most != -INFINITY && (fabsf(most - shift) > 64.f || !(worst < kMost));
        if (!__syncthreads_or(again)) break;
        shift = most == -INFINITY ? 0.f : most;
    }
    sum += __shfl_xor(sum, 32);
    float top = sum == 0.f ? -INFINITY : shift;
    // the waves of the same queries
    float* const joined = reinterpret_cast<float*>(lds);
    constexpr int kPart = 64 * (16 * R::kColumns + 2);
    if (kw > 0) {
        float* const to = joined + (wave - 8 / KW) * kPart + lane;
        to[0] = top;
        to[64] = sum;
#pragma unroll
        for (int c = 0; c < R::kColumns; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) to[64 * (2 + 16 * c + i)] = o[c][i];
    }
    __syncthreads();
    if (kw > 0 || !live) return;
    for (int k = 1; k < KW; ++k) {
        const float* const from = joined + (k * (8 / KW) + qw - 8 / KW) * kPart + lane;
        const float one = from[64];
        if (one == 0.f) continue;  // no key
        const float next = fmaxf(top, from[0]);
        const float a = sum == 0.f ? 0.f : __builtin_amdgcn_exp2f(top - next), e = __builtin_amdgcn_exp2f(from[0] - next);
        top = next;
        sum = sum * a + one * e;
#pragma unroll
        for (int c = 0; c < R::kColumns; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[c][i] = o[c][i] * a + from[64 * (2 + 16 * c + i)] * e;
    }
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
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
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

constexpr int kMostSplits = 256;

// Joins the parts of the splits: a wave takes a row, its lanes first the splits' statistics, then channels.
template <typename T, int D>
__global__ __launch_bounds__(kBlock) void dense_join_kernel(DenseForward p)
{
    constexpr int kShare = D < 64 ? 64 / D : 1, kEach = D < 64 ? 1 : D / 64;  // lanes of a channel, channels of a lane
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + wave_index();
    if (row >= p.all_rows) return;
    const int lane = threadIdx.x & 63;
    const float* const ml = p.part + static_cast<int64_t>(p.splits) * p.all_rows * D + 2 * row;
    float w[kMostSplits / 64], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int k = 0; k < kMostSplits / 64; ++k) {
        const int s = 64 * k + lane;
        w[k] = s < p.splits && ml[2 * s * p.all_rows + 1] != 0.f ? ml[2 * s * p.all_rows] : -INFINITY;
        top = fmaxf(top, w[k]);
    }
    for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
#pragma unroll
    for (int k = 0; k < kMostSplits / 64; ++k) {
        const int s = 64 * k + lane;
        const float one = s < p.splits ? ml[2 * s * p.all_rows + 1] : 0.f;
        w[k] = one == 0.f ? 0.f : __builtin_amdgcn_exp2f(w[k] - top);
        sum += one == 0.f ? 0.f : w[k] * one;
    }
    for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
    float o[kEach];
#pragma unroll
    for (int c = 0; c < kEach; ++c) o[c] = 0.f;
#pragma unroll
    for (int k = 0; k < kMostSplits / 64; ++k) {
        const int n = min(64, p.splits - 64 * k);
        for (int s0 = 0; s0 < n; s0 += 8 * kShare) {
            float f[8], x[8][kEach];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int mine = s0 + j * kShare + (kShare > 1 ? lane / D : 0);
                f[j] = mine < 64 ? __shfl(w[k], mine) : 0.f;
                const float* const from = p.part + ((64 * k + mine) * p.all_rows + row) * D + lane % D;
#pragma unroll
                for (int c = 0; c < kEach; ++c) x[j][c] = mine < n && f[j] != 0.f ? from[64 * c] : 0.f;  // (0: nothing was written)
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int c = 0; c < kEach; ++c) o[c] = fmaf(f[j], x[j][c], o[c]);
        }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int c = 0; c < kEach; ++c) {
        for (int m = D; m < 64; m <<= 1) o[c] += __shfl_xor(o[c], m);
        if (lane < D) static_cast<T*>(p.out)[row * D + lane + 64 * c] = from_float<T>(o[c] * inv);
    }
}

struct ForwardPlan {
    DenseForward p;
    int key_waves;
    int64_t blocks;
};

// How a call's waves share queries and keys, and the splits of the keys over blocks.
ForwardPlan forward_plan(const DenseCall& c, int elem_bytes)
{
    ForwardPlan plan{};
    DenseForward& p = plan.p;
    static_cast<DenseParams&>(p) = dense_params(c);
    const int bytes = c.g.d * elem_bytes;
    auto room = [&](int kw, int slices) {
        const int64_t keys = kw * (kw > 2 || bytes > 256 ? 32 : 64), rows = 256 / kw;
        const int64_t windows = c.bias ? slices * bias_window(int(rows), int(keys), c.g.Hk, c.g.Wk) : 0;
        const int64_t tiles = 2 * keys * (bytes + 16);
        return (tiles <= 72 * 1024 ? 2 : 1) * (tiles + 4 * (windows + keys)) + 1024 <= 158 * 1024;
    };
    // a tile that holds the queries of all slices of a key slice, each with a window
    const bool together = c.bias && p.share > 1 && int64_t(p.share) * p.nq <= 32 && p.share <= 16 && room(8, p.share);
    if (!c.bias || together) {
        p.per_group = p.share;
        p.groups = c.g.S / p.share;
        p.rows = p.nq * p.share;
    }
    auto blocks = [&](int kw) { return int64_t(p.groups) * ((p.rows + 256 / kw - 1) / (256 / kw)); };
    int kw = 8;
    if (p.rows > 32 && blocks(4) >= 256) kw = 4;
    if (p.rows > 64 && blocks(2) >= 256) kw = 2;
    if (!room(kw, together ? p.share : 1)) kw = bytes > 256 && room(4, 1) ? 4 : 2;
    plan.key_waves = kw;
    p.tiles = (p.rows + 256 / kw - 1) / (256 / kw);
    const int keys = kw * (kw > 2 || bytes > 256 ? 32 : 64);
    if (c.bias) p.window = int(bias_window(256 / kw, keys, c.g.Hk, c.g.Wk));
    // a part is worth a block from one step on where the queries are few, and fewer than two blocks per CU leave CUs idle
    const int64_t steps = (p.nk + keys - 1) / keys;
    int64_t n = 512 / blocks(kw);
    if (n > steps) n = steps;
    if (n > kMostSplits) n = kMostSplits;
    p.splits = n < 1 ? 1 : int(n);
    p.all_rows = int64_t(p.groups) * p.rows;
    plan.blocks = blocks(kw) * p.splits;
    return plan;
}

int elem_bytes_of(int dtype) { return dtype == SCRAM_BF16 ? 2 : 4; }

}  // namespace

// Most places of the bias' plane between the ends of 128 queries against 128 keys.
int64_t dense_bias_window(int Hk, int Wk) { return bias_window(128, 128, Hk, Wk); }

size_t dense_workspace_bytes(int dtype, const DenseCall& c)
{
    const ForwardPlan plan = forward_plan(c, elem_bytes_of(dtype));
    return plan.p.splits == 1 ? 0 : size_t(plan.p.splits) * plan.p.all_rows * (c.g.d + 2) * sizeof(float);
}

uint64_t dense_blocks(int dtype, const DenseCall& c) { return 2 * uint64_t(forward_plan(c, elem_bytes_of(dtype)).blocks); }

hipError_t launch_dense(int dtype, const DenseCall& c, void* out, void* workspace, hipStream_t stream, hipEvent_t start,
                        hipEvent_t stop)
{
    ForwardPlan plan = forward_plan(c, elem_bytes_of(dtype));
    DenseForward& p = plan.p;
    p.out = out;
    p.part = static_cast<float*>(workspace);
    return dispatch_value(dtype, c.g.d, hipErrorInvalidValue, [&](auto type, auto width) {
        using T = std::conditional_t<std::is_same<decltype(type), float>::value, float, uint16_t>;
        constexpr int D = decltype(width)::value;
        const hipEvent_t end = p.splits == 1 ? stop : nullptr;
        auto run = [&](auto biased, auto key_waves) {
            constexpr int KW = decltype(key_waves)::value;
            constexpr bool kBiased = decltype(biased)::value;
            constexpr int keys = KW * kWaveKeys<T, D, KW>;
            const size_t lds =
                forward_lds<T, D, KW>() + (kBiased ? kBuffers<T, D, KW> * (keys + size_t(p.per_group) * p.window) * sizeof(float) : 0);
            return launch_dense_kernel<kThreads>(dense_kernel<T, D, kBiased, KW>, plan.blocks, lds, stream, start, end, p);
        };
        auto with = [&](auto biased) {
            if (plan.key_waves == 2) return run(biased, std::integral_constant<int, 2>{});
            if constexpr (D * sizeof(T) <= 256)
                if (plan.key_waves == 8) return run(biased, std::integral_constant<int, 8>{});
            return run(biased, std::integral_constant<int, 4>{});
        };
        const hipError_t e = c.bias ? with(std::true_type{}) : with(std::false_type{});
        if (e != hipSuccess || p.splits == 1) return e;
        return launch_dense_kernel(dense_join_kernel<T, D>, (p.all_rows + 3) / 4, 0, stream, nullptr, stop, p);
    });
}

}  // namespace scram
