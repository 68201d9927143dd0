// Gradients of the attention over every key.
//
//   p_ij = softmax_j(scale q_i.k_j + bias), dp_ij = dO_i.v_j, D_i = sum_j p_ij dp_ij, ds_ij = p_ij (dp_ij - D_i)
//   dQ_i = scale sum_j ds_ij k_j, dK_j = scale sum_i ds_ij q_i, dV_j = sum_i p_ij dO_i, dB_o = sum of ds_ij at offset o
//
// Bound by computing: five products of a pair's rows are what cannot be done
// without, 10 d operations a pair.  Three kernels, each with one writer for
// every result and sums of a fixed order:
// - queries: a block holds 128 and passes over the keys twice.  The first pass
//   gives the softmax's statistics and D (of fp32 weights: where one weight is
//   nearly 1, dp - D is what is left of two nearly equal numbers, which a D
//   from the rounded output would bury), the second dQ;
// - keys: a block holds 128 and passes over the queries: dK and dV;
// - offsets, with a bias: scores and ds once more, added up in registers over
//   all pairs of tiles at one offset, whose diagonals are then one offset each.
// The products with p and ds take them from the registers that formed them
// (scram_dense.h); in bf16 both go in two parts, which add up to them to 2^-16,
// as the matrix cores take 8 bits a number, and sums stay in 32 bits.
//
// Measured, bf16, 16 slices of 64 x 64, 64 channels, a bias: queries 276 us,
// keys 261, offsets 204 (the vector units are busy for 0.60, 0.48 and 0.45 of
// that, the matrix cores for 0.31, 0.31 and 0.14); 16 slices of a row of 2500
// on 4 of keys, 128 channels, causal: queries 166 us, keys 202, their parts 8.

#include "scram_dense.h"

namespace scram {
namespace {

constexpr int kKeysBlock = 128;  // keys of a block of the key side

struct DenseBackward : DenseQueries {
    const void* dO;
    void* dQ;
    void* dK;
    void* dV;
    void* dbias;       // nullable
    float4* stats;     // [all query rows] row_stats()
    float* part;       // key side: [splits][all keys][2][D]
    float* diagonals;  // [bias rows][2 Hk - 1][2 x_tiles - 1][64]
    int64_t all_keys;
    int key_tiles;     // of a slice's keys
    int key_splits;    // runs of query tiles, at most
    int key_each;      // causal, one place of all slices' queries: query tiles of a run
    int key_window;    // floats of LDS for the key side's bias
    int x_tiles, Hk, Wk, key_slices, S;
    int cuts;          // of a column's grid rows among waves
};

// A row's softmax for the other kernels: weights are exp2(x - x0) f for scores x in base 2, x0 the logarithm of their sum and
// f 1.  Scores so large that adding the logarithm would lose it (a bias of the type's lowest values) keep them apart: x0 is
// the maximum, f one over the sum.  The third value is D.
__device__ __forceinline__ float4 row_stats(float top, float sum, float dsum)
{
    if (sum == 0.f) return make_float4(INFINITY, 1.f, 0.f, 0.f);  // no key: exp2(x - infinity) = 0
    const bool apart = fabsf(top) > 4096.f;
    return make_float4(apart ? top : top + __builtin_amdgcn_logf(sum), apart ? 1.f / sum : 1.f, dsum / sum, 0.f);
}

// The query side: two passes over the keys.  Four waves a SIMD as in the forward pass: 745 us, 779 with two (all kernels, 16
// slices of 64 x 64 with a bias); with one block a CU two (8 of 48 x 48: 244 us, 253 with four).  fp32 rows of 128 channels spill
// 232 to 328 bytes a lane with two.
template <typename T, int D, bool BIAS, int KW>
__global__ __launch_bounds__(kQueryThreads, D * sizeof(T) > 128 || (BIAS && KW > 2) ? 2 : 4) void dense_query_kernel(DenseBackward p)
{
    using R = DenseRow<T, D>;
    constexpr bool kFold = sizeof(T) == 2 && !BIAS;  // as in the forward pass; the first pass keeps a certain key's weight at 1
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ float s_join[3][8][32];
    QueryBlock<T, D, BIAS, KW> q(p, lds);
    const int lane = q.lane, m = q.m, h = q.h, wave = q.wave, qw = q.qw, kw = q.kw;
    const int64_t out_row = q.out_row;
    uint4 qf[R::kSteps], gf[R::kSteps];
    load_operand<T, D>(p.Q, q.from_row(), h, qf);
    load_operand<T, D>(p.dO, q.from_row(), h, gf);
    if constexpr (kFold) q.positive_scale(qf);

    // a lane's maximum, sum, and sum of dp: of its half of the keys
    float top = -INFINITY, sum = 0.f, dsum = 0.f;
    q.pass([&](auto at, const int* places, int from, int k0) {
        constexpr int kAt = decltype(at)::value;
        f32x16_t s = q.products(kAt, qf);
        q.template scores<false>(s, places, from, k0);
        if constexpr (BIAS) __builtin_amdgcn_sched_barrier(0);
        const f32x16_t g = q.products(kAt + q.kValues, gf);
        float most = top;
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, s[i]);
        const float shift = most == -INFINITY ? 0.f : most, keep = __builtin_amdgcn_exp2f(top - shift);
        sum *= keep;
        dsum *= keep;
        top = most;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float e = __builtin_amdgcn_exp2f(s[i] - shift);
            sum += e;
            dsum = fmaf(e, g[i], dsum);
        }
    });
    auto join = [&](float t, float a, float b) {
        const float most = fmaxf(top, t), shift = most == -INFINITY ? 0.f : most;
        const float x = __builtin_amdgcn_exp2f(top - shift), y = __builtin_amdgcn_exp2f(t - shift);
        sum = sum * x + a * y;
        dsum = dsum * x + b * y;
        top = most;
    };
    join(__shfl_xor(top, 32), __shfl_xor(sum, 32), __shfl_xor(dsum, 32));
    if (h == 0) {
        s_join[0][wave][m] = top;
        s_join[1][wave][m] = sum;
        s_join[2][wave][m] = dsum;
    }
    __syncthreads();
    top = -INFINITY;
    sum = dsum = 0.f;
#pragma unroll
    for (int k = 0; k < KW; ++k) join(s_join[0][k * (8 / KW) + qw][m], s_join[1][k * (8 / KW) + qw][m], s_join[2][k * (8 / KW) + qw][m]);
    const float4 stats = row_stats(top, sum, dsum);
    if (q.live && h == 0 && kw == 0) p.stats[out_row] = stats;
    // here the sum divides once, at the end
    const float shift = top == -INFINITY ? 0.f : top, mean = stats.z, scale2 = q.scale2;
    const float factor = sum == 0.f ? 0.f : p.scale / sum;

    f32x16_t o[R::kColumns];
#pragma unroll
    for (int c = 0; c < R::kColumns; ++c) o[c] = f32x16_t(0.f);
    q.pass([&](auto at, const int* places, int from, int k0) {
        constexpr int kAt = decltype(at)::value;
        f32x16_t s = q.products(kAt, qf);
        q.template scores<kFold>(s, places, from, k0);
        if constexpr (BIAS) __builtin_amdgcn_sched_barrier(0);
        const f32x16_t g = q.products(kAt + q.kValues, gf);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            s[i] = __builtin_amdgcn_exp2f(kFold ? fmaf(s[i], scale2, -shift) : s[i] - shift) * (g[i] - mean);
#pragma unroll
        for (int r = 0; r < R::kRowSteps; ++r) {
            const RightOperand<T> w = as_operand<T>(s, r);
#pragma unroll
            for (int c = 0; c < R::kColumns; ++c) o[c] = mma<T>(q.reader.column(r, c, kAt), w, o[c]);
        }
    });
    // the waves of the same queries: each joins a share of the channels
    constexpr int kPart = 64 * 16 * R::kColumns;
    float* const joined = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int c = 0; c < R::kColumns; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) joined[wave * kPart + 64 * (16 * c + i) + lane] = o[c][i];
    __syncthreads();
    if (!q.live) return;
    constexpr int kQuads = D < 32 ? 2 : 4 * R::kColumns;
    for (int g = kw; g < kQuads; g += KW) {
        vec<T, 4> y;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float x = 0.f;
#pragma unroll
            for (int k = 0; k < KW; ++k) x += joined[(k * (8 / KW) + qw) * kPart + 64 * (4 * g + j) + lane];
            y[j] = from_float<T>(x * factor);
        }
        store_vec<T, 4>(static_cast<T*>(p.dQ) + out_row * D + 8 * g + 4 * h, y);
    }
}

// Rows of queries that a block of the key side stages at a time; two such steps are in LDS.
constexpr int staged_rows(int row_bytes) { return row_bytes > 256 ? 32 : 64; }
template <typename T, int D>
constexpr int kStaged = staged_rows(D * sizeof(T));
template <typename T, int D>
constexpr size_t kKeyTile = 2 * (kStaged<T, D> * DenseRow<T, D>::kBytes);

constexpr size_t kKeyStatic = 64 * sizeof(float);  // the vote on a step's factors

inline size_t key_lds(int d, int elem_bytes, const DenseBackward& p, bool biased)
{
    const size_t row = size_t(d) * elem_bytes, staged = staged_rows(int(row));
    return 2 * (2 * staged * row) + 2 * sizeof(float) * (3 * staged + (biased ? staged + p.key_window : 0)) + 64;
}

// The query tiles of a slice that see some key of the block at key k_first: `count` from `low` on; the runs that those of all
// slices are dealt in.  (Where slices have places of their own, the tiles of none are told apart beforehand.)
struct KeyRuns {
    int low, count, all, runs;
};
__host__ __device__ inline KeyRuns key_runs(const DenseBackward& p, int rows, int k_first)
{
    const int tiles = (p.nq + rows - 1) / rows;
    if (!p.causal || p.origin) return KeyRuns{0, tiles, tiles * p.share, p.key_splits};
    const int behind = k_first - p.first;  // queries before these see none of the keys
    const int low = behind >= p.nq ? tiles : behind > 0 ? behind / rows : 0, all = (tiles - low) * p.share;
    const int runs = (all + p.key_each - 1) / p.key_each;
    return KeyRuns{low, tiles - low, all, runs < 1 ? 1 : runs};
}

// A number of each of a tile's 32 rows, as registers of a result hold them.
template <typename T>
__device__ __forceinline__ f32x16_t row_numbers(const float* of, int h)
{
    f32x16_t x;
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
        const float4 v = *reinterpret_cast<const float4*>(of + tile_slot<T>(i) + tile_half<T>() * h);
        x[i] = v.x;
        x[i + 1] = v.y;
        x[i + 2] = v.z;
        x[i + 3] = v.w;
    }
    return x;
}

// The key side: a block's 128 keys against a run of the query tiles of the slices that read them.  Two waves a SIMD, as many as
// 512 blocks are: squeezed into registers for three 16 slices of 64 x 64 with a bias took 773 us where all kernels take 745.
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(kBlock) void dense_key_kernel(DenseBackward p)
{
    using R = DenseRow<T, D>;
    constexpr int kRows = kStaged<T, D>, U = kRows / 32;
    extern __shared__ __align__(16) unsigned char lds[];
    // of each of two steps: logarithms, factors and means of the queries' softmax, their places, the bias' window
    float* const s_stats = reinterpret_cast<float*>(lds + 2 * kKeyTile<T, D>);
    const int stats_floats = 3 * kRows + (BIAS ? kRows + p.key_window : 0);

    const uint32_t b = xcd_remap(blockIdx.x, gridDim.x);
    const int split = static_cast<int>(b % static_cast<uint32_t>(p.key_splits));
    const int tile = static_cast<int>(b / static_cast<uint32_t>(p.key_splits) % static_cast<uint32_t>(p.key_tiles));
    const int slice_k = static_cast<int>(b / static_cast<uint32_t>(p.key_splits) / static_cast<uint32_t>(p.key_tiles));
    const int lane = threadIdx.x & 63, wave = wave_index(), m = lane & 31, h = lane >> 5;
    // the keys that count and that some query sees: no others are read
    int length = p.lengths ? min(max(p.lengths[slice_k], 0), p.nk) : p.nk;
    auto begin_of = [&](int slice) { return p.origin ? min(max(p.origin[slice], 0), p.nk - p.nq) : p.first; };
    if (p.causal) {
        int reach = 0;
        for (int s = 0; s < (p.origin ? p.share : 1); ++s) reach = max(reach, begin_of(slice_k * p.share + s) + p.nq);
        length = min(length, reach);
    }
    const int k_first = tile * kKeysBlock, k_wave = k_first + wave * 32, key = k_wave + m;
    const bool seen = key < length;
    const int64_t k_row = static_cast<int64_t>(slice_k) * p.nk;

    uint4 kf[R::kSteps], vf[R::kSteps];
#pragma unroll
    for (int c = 0; c < R::kSteps; ++c) kf[c] = vf[c] = make_uint4(0u, 0u, 0u, 0u);
    if (seen) {
        load_operand<T, D>(p.K, k_row + key, h, kf);
        load_operand<T, D>(p.V, k_row + key, h, vf);
    }
    f32x16_t dk[R::kColumns], dv[R::kColumns];
#pragma unroll
    for (int c = 0; c < R::kColumns; ++c) dk[c] = dv[c] = f32x16_t(0.f);
    const int k_last = min(k_first + kKeysBlock, p.nk) - 1;
    int key_place = 0, first_place = 0;
    if constexpr (BIAS) {
        key_place = bias_place(p, min(key, p.nk - 1));
        first_place = bias_place(p, k_first);
    }

    const KeyRuns of = key_runs(p, kRows, k_first);
    if (split >= of.runs) return;
    const int t0 = static_cast<int>(static_cast<int64_t>(of.all) * split / of.runs);
    const int t1 = k_first < length ? static_cast<int>(static_cast<int64_t>(of.all) * (split + 1) / of.runs) : t0;
    auto slice_of = [&](int t) { return slice_k * p.share + t / of.count; };
    auto query_of = [&](int t) { return (of.low + t % of.count) * kRows; };
    // the next tile of which a query sees a key of the block, from t on
    auto seek = [&](int t) {
        if (p.causal && p.origin)
            while (t < t1 && begin_of(slice_of(t)) + min(query_of(t) + kRows, p.nq) <= k_first) ++t;
        return t;
    };
    using Stage = DenseStage<T, D, kRows, kBlock>;
    BiasStage<T> bl;
    float4 st = make_float4(INFINITY, 1.f, 0.f, 0.f);
    // of the fetched tile: its first query and that one's place; places on the bias' plane
    int next_q = 0, next_at = 0, next_end = 0, next_place = 0;
    auto fetch = [&](int t, int at) {
        const int slice = slice_of(t), q0 = query_of(t), begin = begin_of(slice);
        const int64_t row = static_cast<int64_t>(slice) * p.nq + q0;
        Stage::load(p.Q, row, p.nq - q0, lds + at * kKeyTile<T, D>);
        Stage::load(p.dO, row, p.nq - q0, lds + at * kKeyTile<T, D> + kRows * R::kBytes);
        const int q = static_cast<int>(threadIdx.x);
        st = make_float4(INFINITY, 1.f, 0.f, 0.f);
        if (q < kRows && q0 + q < p.nq) st = p.stats[row + q];
        next_q = q0;
        next_at = begin + q0;
        if constexpr (BIAS) {
            const int q1 = begin + min(q0 + kRows, p.nq) - 1;
            bl.load(p, slice % p.plane.rows, begin + q0, q1, k_first, k_last, q, kBlock);
            next_end = bias_place(p, q1);
            if (q < kRows) next_place = 4 * bias_place(p, min(begin + q0 + q, q1));
        }
    };
    bool apart = false;
    auto store = [&](int at) {
        float* const stats = s_stats + at * stats_floats;
        const int q = static_cast<int>(threadIdx.x);
        if (q < kRows) {
            stats[q] = st.x;
            stats[kRows + q] = st.y;
            stats[2 * kRows + q] = st.z;
            if constexpr (BIAS) reinterpret_cast<int*>(stats)[3 * kRows + q] = next_place;
        }
        if constexpr (BIAS) bl.store(stats + 4 * kRows, q, kBlock);
        return st.y != 1.f;
    };
    TileReader<T, D> reader;
    reader.set(lds);
    constexpr int kG = kRows * R::kBytes;
    const lds_bytes first_base = reader.base;
    int t = seek(t0), at = 0;
    if (t < t1) {
        fetch(t, 0);
        apart = store(0);
    }
    Stage::wait();
    apart = __syncthreads_or(apart);
    while (t < t1) {
        reader.base = first_base + at * static_cast<int>(kKeyTile<T, D>);
        const int at0 = next_at;  // place of the tile's first query
        // 4 (place of the key, less the window's start)
        const int my_place = 4 * (key_place - (first_place - next_end));
        const float* const stats = s_stats + at * stats_floats;
        const int q_now = next_q;
        t = seek(t + 1);
        if (t < t1) fetch(t, at ^ 1);
        // a query after which some key of the wave's comes, or a key that is not seen
        const bool masked = (p.causal && at0 < k_wave + 31) || k_wave + 32 > length;
        // a vector's rows are queries here, which lie side by side where it does not cross a grid row: grid rows of whole vectors
        // and a tile that begins at one (16 slices of a run of 4080 on 64 x 64, all kernels: from place 8 on 746 us, from 5 on 757;
        // rows behind the last query may meet what lies before the window, a number, with an infinite logarithm: a weight of 0)
        const bool runs = p.runs && (p.Hk == 1 || at0 % tile_half<T>() == 0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            reader.renew();
            // nothing to add: queries before the wave's keys, or behind the slice's last
            if ((p.causal && at0 + 32 * u + 31 < k_wave) || q_now + 32 * u >= p.nq) continue;
            f32x16_t s(0.f), g(0.f);
#pragma unroll
            for (int c = 0; c < R::kSteps; ++c) {
                s = mma<T>(reader.row(c, 32 * u * R::kBytes), kf[c], s);
                g = mma<T>(reader.row(c, kG + 32 * u * R::kBytes), vf[c], g);
            }
            f32x16_t w;
            if constexpr (BIAS) {
                add_bias<T, -1>(s, p.scale2, stats + 4 * kRows, reinterpret_cast<const int*>(stats) + 3 * kRows + 32 * u, my_place, h,
                                runs);
                w = s - row_numbers<T>(stats + 32 * u, h);
            } else {
                const f32x16_t x0 = row_numbers<T>(stats + 32 * u, h);
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = fmaf(s[i], p.scale2, -x0[i]);
            }
            if (masked) {
                asm volatile("");  // (not for every tile, by selects)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    w[i] = seen && (!p.causal || key <= at0 + 32 * u + tile_half<T>() * h + tile_slot<T>(i)) ? w[i] : -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = __builtin_amdgcn_exp2f(w[i]);
            if (apart) {
                asm volatile("");
                w *= row_numbers<T>(stats + kRows + 32 * u, h);
            }
            s = w * (g - row_numbers<T>(stats + 2 * kRows + 32 * u, h));
#pragma unroll
            for (int r = 0; r < R::kRowSteps; ++r) {
                const RightOperand<T> a = as_operand<T>(w, r), d = as_operand<T>(s, r);
#pragma unroll
                for (int c = 0; c < R::kColumns; ++c) {
                    dv[c] = mma<T>(reader.column(r, c, kG + 32 * u * R::kBytes), a, dv[c]);
                    dk[c] = mma<T>(reader.column(r, c, 32 * u * R::kBytes), d, dk[c]);
                }
            }
        }
        at ^= 1;
        apart = t < t1 ? store(at) : false;
        Stage::wait();
        apart = __syncthreads_or(apart);
    }
    if (key >= p.nk) return;
    if (p.key_splits > 1) {
        float* const to = p.part + (static_cast<int64_t>(split) * p.all_keys + k_row + key) * (2 * D);
#pragma unroll
        for (int c = 0; c < R::kColumns; ++c)
#pragma unroll
            for (int i = 0; i < (D < 32 ? 2 : 4); ++i) {
                float* const x = to + 32 * c + 8 * i + 4 * h;
                *reinterpret_cast<float4*>(x) = make_float4(dk[c][4 * i], dk[c][4 * i + 1], dk[c][4 * i + 2], dk[c][4 * i + 3]);
                *reinterpret_cast<float4*>(x + D) = make_float4(dv[c][4 * i], dv[c][4 * i + 1], dv[c][4 * i + 2], dv[c][4 * i + 3]);
            }
        return;
    }
    T* const to_k = static_cast<T*>(p.dK) + (k_row + key) * D;
    T* const to_v = static_cast<T*>(p.dV) + (k_row + key) * D;
#pragma unroll
    for (int c = 0; c < R::kColumns; ++c)
#pragma unroll
        for (int i = 0; i < (D < 32 ? 2 : 4); ++i) {
            vec<T, 4> x, y;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = from_float<T>(dk[c][4 * i + j] * p.scale);
                y[j] = from_float<T>(dv[c][4 * i + j]);
            }
            store_vec<T, 4>(to_k + 32 * c + 8 * i + 4 * h, x);
            store_vec<T, 4>(to_v + 32 * c + 8 * i + 4 * h, y);
        }
}

// Adds up the parts of the key side's splits: a thread takes four values of dK's or dV's row.
template <typename T, int D>
__global__ __launch_bounds__(kBlock) void dense_key_join_kernel(DenseBackward p)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x, row = i / (D / 2);
    if (row >= p.all_keys) return;
    const int c = static_cast<int>(i % (D / 2)) * 4;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    const int runs = key_runs(p, kStaged<T, D>, static_cast<int>(row % p.nk) / kKeysBlock * kKeysBlock).runs;
    for (int s = 0; s < runs; ++s) {
        const float4 y = *reinterpret_cast<const float4*>(p.part + (static_cast<int64_t>(s) * p.all_keys + row) * (2 * D) + c);
        x[0] += y.x;
        x[1] += y.y;
        x[2] += y.z;
        x[3] += y.w;
    }
    vec<T, 4> y;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = from_float<T>(c < D ? x[j] * p.scale : x[j]);
    store_vec<T, 4>((c < D ? static_cast<T*>(p.dK) + c : static_cast<T*>(p.dV) + c - D) + row * D, y);
}

// 32 rows on their way through a wave's own part of LDS: read from memory as they lie there, a row by neighbouring lanes, and
// from LDS as operands, a row by a lane (operands straight from memory touch 32 lines an instruction: 289 us where this took
// 207, 16 slices of 64 x 64, 64 channels).
template <typename T, int D>
struct WaveTile {
    using R = DenseRow<T, D>;
    static constexpr int kEach = R::kChunks / 2;
    static constexpr int kBytes = 32 * R::kBytes;
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    words x[kEach];

    // rows first .. last - 1 (one at least) of the tile that begins at `row0`; those before and after them are its ends again
    __device__ __forceinline__ void load(const void* rows, int64_t row0, int first, int last)
    {
        const unsigned char* const from = static_cast<const unsigned char*>(rows) + row0 * R::kBytes;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int c = i * 64 + static_cast<int>(threadIdx.x & 63);
            x[i] = *reinterpret_cast<const words*>(from + min(max(c / R::kChunks, first), last - 1) * R::kBytes + 16 * (c % R::kChunks));
        }
    }
    // the operands of row `row` for this lane
    __device__ __forceinline__ void turn(unsigned char* tile, int row, uint4 (&y)[R::kSteps]) const
    {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int c = i * 64 + static_cast<int>(threadIdx.x & 63);
            *reinterpret_cast<words*>(tile + R::place(c / R::kChunks, c % R::kChunks)) = x[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int s = 0; s < R::kSteps; ++s) y[s] = row_operand<T, D>(tile, row, (threadIdx.x & 63) >> 5, s);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
};

// The offset side: an offset dy of rows, and tiles of 32 columns `apart`, of one head.  A wave goes down the grid rows of a column
// of tiles (of every fourth column and slice); a tile's scores are formed transposed, so that a query's statistics are its
// lane's, and what a pair of tiles leaves is added up in registers by the place in the tile.  Two rows of offsets a block, with a
// tile of keys kept for the next step, read half as much, but leave half the blocks, of half the waves a CU: 16 slices of
// 64 x 64 210 us, this 230; 64 of 32 x 32 127 and 90; 4 of 93 x 125 574 and 491.
template <typename T, int D>
__global__ __launch_bounds__(kBlock, D * sizeof(T) > 256 ? 1 : 2) void dense_offset_kernel(DenseBackward p)
{
    using R = DenseRow<T, D>;
    __shared__ float s_sum[32][33];
    __shared__ __align__(16) float s_bias[4][64][4];  // by register and lane
    __shared__ __align__(16) unsigned char s_turn[4][WaveTile<T, D>::kBytes];
    const uint32_t b = xcd_remap(blockIdx.x, gridDim.x);
    const int apart_all = 2 * p.x_tiles - 1, height = 2 * p.Hk - 1;
    const int apart = static_cast<int>(b % static_cast<uint32_t>(apart_all)) - p.x_tiles + 1;
    const int dy = static_cast<int>(b / static_cast<uint32_t>(apart_all) % static_cast<uint32_t>(height)) - p.Hk + 1;
    const int head = static_cast<int>(b / static_cast<uint32_t>(apart_all) / static_cast<uint32_t>(height));
    const int lane = threadIdx.x & 63, wave = wave_index(), m = lane & 31, h = lane >> 5;
    const int W = p.Wk, columns = p.x_tiles - abs(apart), column0 = apart < 0 ? -apart : 0;
    const int64_t row = static_cast<int64_t>(head) * height + dy + p.Hk - 1;  // of all heads' rows of offsets
    for (int i = threadIdx.x; i < 1024; i += kBlock) {
        const int e = i & 3, l = (i >> 2) & 63, r = i >> 8;
        const int dx = 32 * apart + tile_slot<T>(4 * r + e) + tile_half<T>() * (l >> 5) - (l & 31);
        const T* const table = static_cast<const T*>(p.bias) + row * p.plane.width;
        s_bias[r][l][e] = abs(dx) < W ? bias_base2(to_float(table[W - 1 + dx])) : 0.f;
    }
    __syncthreads();
    f32x16_t sum(0.f);
    // no key comes after its query
    const bool none = p.causal && (dy > 0 || (dy == 0 && apart > 0));
    const int64_t strips = none ? 0 : static_cast<int64_t>(p.S / p.plane.rows) * columns * p.cuts;
    for (int64_t strip = wave; strip < strips; strip += 4) {
        const int cut = static_cast<int>(strip % p.cuts), column = static_cast<int>(strip / p.cuts % columns) + column0;
        const int slice = static_cast<int>(strip / p.cuts / columns) * p.plane.rows + head, slice_k = slice / p.share;
        const int begin = p.origin ? min(max(p.origin[slice], 0), p.nk - p.nq) : p.first;
        const int length = p.lengths ? min(max(p.lengths[slice_k], 0), p.nk) : p.nk;
        const int64_t q_row = static_cast<int64_t>(slice) * p.nq, k_row = static_cast<int64_t>(slice_k) * p.nk;
        const int qx0 = 32 * column, qx = qx0 + m, kx0 = 32 * (column + apart);
        const bool x_whole = qx0 + 32 <= W && kx0 + 32 <= W;
        const int low = max(begin / W, -dy), high = min((begin + p.nq - 1) / W, p.Hk - 1 - dy);
        const int from = low + (high - low + 1) * cut / p.cuts, to = low + (high - low + 1) * (cut + 1) / p.cuts;
        if (low > high) continue;
        for (int qy = from; qy < to; ++qy) {
            const int ky = qy + dy, key0 = ky * W + kx0, k_last = min(min(32, W - kx0), length - key0);
            const int q = qy * W + qx - begin;
            const int q0 = qy * W + qx0 - begin, q_first = max(0, -q0), q_last = min(min(32, W - qx0), p.nq - q0);
            if (k_last <= 0 || q_first >= q_last) continue;  // no key that counts, none of the run's queries
            const bool q_ok = qx < W && q >= 0 && q < p.nq;
            uint4 kf[R::kSteps], vf[R::kSteps], qf[R::kSteps], gf[R::kSteps];
            float4 st = make_float4(INFINITY, 1.f, 0.f, 0.f);
            {
                // all on their way before the first is waited for
                WaveTile<T, D> kl, vl, ql, gl;
                kl.load(p.K, k_row + key0, 0, k_last);
                vl.load(p.V, k_row + key0, 0, k_last);
                ql.load(p.Q, q_row + q0, q_first, q_last);
                gl.load(p.dO, q_row + q0, q_first, q_last);
                if (q_ok) st = p.stats[q_row + q];
                kl.turn(s_turn[wave], tile_row<T>(m), kf);
                vl.turn(s_turn[wave], tile_row<T>(m), vf);
                ql.turn(s_turn[wave], m, qf);
                gl.turn(s_turn[wave], m, gf);
            }
            f32x16_t s(0.f), g(0.f);
#pragma unroll
            for (int c = 0; c < R::kSteps; ++c) {
                s = mma<T>(kf[c], qf[c], s);
                g = mma<T>(vf[c], gf[c], g);
            }
            const bool whole = x_whole && k_last == 32 && !(p.causal && dy == 0 && apart == 0) && __all(q_ok);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float4 bias = *reinterpret_cast<const float4*>(s_bias[r][lane]);
                s[4 * r] = fmaf(s[4 * r], p.scale2, bias.x);
                s[4 * r + 1] = fmaf(s[4 * r + 1], p.scale2, bias.y);
                s[4 * r + 2] = fmaf(s[4 * r + 2], p.scale2, bias.z);
                s[4 * r + 3] = fmaf(s[4 * r + 3], p.scale2, bias.w);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) g[i] -= st.z;
            if (!whole)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int x1 = kx0 + tile_slot<T>(i) + tile_half<T>() * h, key = ky * W + x1;
                    const bool on = q_ok && x1 < W && key < length && (!p.causal || key <= q + begin);
                    s[i] = on ? s[i] : -INFINITY;
                    g[i] = on ? g[i] : 0.f;
                }
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i] - st.x);
            if (__any(st.y != 1.f)) {
                asm volatile("");
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] *= st.y;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[i] = fmaf(s[i], g[i], sum[i]);
        }
    }
    // the waves' sums one after another, then the diagonals
    for (int k = 0; k < 4; ++k) {
        if (wave == k)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float& at = s_sum[m][tile_slot<T>(i) + tile_half<T>() * h];
                at = k ? at + sum[i] : sum[i];
            }
        __syncthreads();
    }
    if (threadIdx.x < 63) {
        const int t = static_cast<int>(threadIdx.x) - 31;  // the key's column less the query's
        float x = 0.f;
        for (int r = max(0, -t); r < min(32, 32 - t); ++r) x += s_sum[r][r + t];
        p.diagonals[(row * apart_all + apart + p.x_tiles - 1) * 64 + threadIdx.x] = x;
    }
}

// dbias of an offset: the diagonals of the (at most two) pairs of tiles that hold it.
template <typename T>
__global__ __launch_bounds__(kBlock) void dense_offset_join_kernel(DenseBackward p)
{
    const int apart_all = 2 * p.x_tiles - 1;
    const int64_t all = p.plane.rows * p.plane.size;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x; i < all; i += static_cast<int64_t>(gridDim.x) * kBlock) {
        const int64_t row = i / p.plane.width;  // of all heads' rows
        const int dx = static_cast<int>(i % p.plane.width) - p.Wk + 1;
        const int apart = dx >= 0 ? dx / 32 : -((31 - dx) / 32), t = dx - 32 * apart;  // 0 <= t < 32
        const float* const from = p.diagonals + (row * apart_all + apart + p.x_tiles - 1) * 64;
        float x = apart > -p.x_tiles ? from[31 + t] : 0.f;
        if (t > 0 && apart + 1 < p.x_tiles) x += from[64 + t - 1];  // 31 + (t - 32)
        static_cast<T*>(p.dbias)[i] = from_float<T>(x);
    }
}

size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

struct BackwardPlan {
    DenseBackward p;
    QueryPlan queries;
    int64_t key_blocks, offset_blocks;
    size_t stats, part, diagonals;  // bytes
};

BackwardPlan backward_plan(const DenseCall& c, int elem_bytes)
{
    BackwardPlan plan{};
    DenseBackward& p = plan.p;
    static_cast<DenseParams&>(p) = dense_params(c);
    plan.queries = query_plan(c, elem_bytes, false, p);
    p.S = c.g.S;
    p.Hk = c.g.Hk;
    p.Wk = c.g.Wk;
    p.key_slices = c.key_slices;
    p.all_keys = int64_t(c.key_slices) * p.nk;
    p.key_tiles = (p.nk + kKeysBlock - 1) / kKeysBlock;
    if (c.bias) p.key_window = int(bias_window(64, kKeysBlock, c.g.Hk, c.g.Wk) + 3) & ~3;
    const int64_t tiles = int64_t(c.key_slices) * p.key_tiles;
    // splits of the queries: fewer than two blocks per CU leave CUs idle, and a part is worth a block from four tiles on (16 slices
    // of 2500 on 4 of keys, 128 channels, all kernels: 840 us whole, 541 / 544 / 448 / 482 in 2 / 4 / 6 / 8 parts, of which this
    // takes 6)
    const int rows = staged_rows(c.g.d * elem_bytes);
    if (c.causal && !c.origin && tiles <= 512) {
        // a key's runs by how many queries see it: the first keys' are many, and all blocks are as long, one a CU (all kernels:
        // 4 rows of 6000, 32 channels 212 us in equal numbers of runs, so 179, with blocks half as long 172; 16 of 2500 on
        // 4 of keys, 128 channels 381, 368 and 394)
        p.key_each = 1;
        int64_t all = 0;
        for (int t = 0; t < p.key_tiles; ++t) all += c.key_slices * int64_t(key_runs(p, rows, t * kKeysBlock).all);
        p.key_each = static_cast<int>((all + 255) / 256);
        if (p.key_each < 4) p.key_each = 4;
        p.key_splits = key_runs(p, rows, 0).runs;
    } else {
        const int64_t all = int64_t(p.share) * ((p.nq + rows - 1) / rows);
        int64_t n = 512 / tiles;
        if (n > all / 4) n = all / 4;
        p.key_splits = n < 1 ? 1 : int(n);
        p.key_each = 1 << 30;
    }
    plan.key_blocks = tiles * p.key_splits;
    plan.stats = round256(size_t(c.g.S) * p.nq * sizeof(float4));
    plan.part = p.key_splits > 1 ? round256(size_t(p.key_splits) * p.all_keys * 2 * c.g.d * sizeof(float)) : 0;
    if (c.bias) {
        p.x_tiles = (c.g.Wk + 31) / 32;
        // four runs of grid rows for the waves of a block at least (all kernels: 8 slices of 64 x 64, 8 heads 423 us, 466 uncut;
        // 16 of 7 x 7 27.6 and 33.2; cut in vain, 32 of 64 x 64 1524 and 1493, 16 of one row of 100 35.1 and 30.5)
        const int64_t columns = int64_t(c.g.S / c.bias_rows) * (p.x_tiles > 1 ? p.x_tiles - 1 : 1);
        p.cuts = columns >= 4 || c.g.Hk == 1 ? 1 : 4;
        plan.offset_blocks = int64_t(c.bias_rows) * (2 * int64_t(c.g.Hk) - 1) * (2 * p.x_tiles - 1);
        plan.diagonals = round256(size_t(plan.offset_blocks) * 64 * sizeof(float));
    }
    return plan;
}

int elem_bytes_of(int dtype) { return dtype == SCRAM_BF16 ? 2 : 4; }

}  // namespace

// Of a call with or without the causal mask, wherever its queries stand: the first keys' runs are most where they stand first.
size_t dense_backward_workspace_bytes(int dtype, const DenseCall& c)
{
    DenseCall any = c;
    any.origin = nullptr;
    any.first = 0;
    any.causal = false;
    const BackwardPlan plan = backward_plan(any, elem_bytes_of(dtype));
    any.causal = true;
    const size_t part = backward_plan(any, elem_bytes_of(dtype)).part;
    return plan.stats + (part > plan.part ? part : plan.part) + plan.diagonals;
}

DenseNeeds dense_backward_needs(int dtype, const DenseCall& c)
{
    const int eb = elem_bytes_of(dtype);
    const BackwardPlan plan = backward_plan(c, eb);
    uint64_t blocks = 2 * uint64_t(plan.queries.blocks);
    if (uint64_t(plan.key_blocks) > blocks) blocks = plan.key_blocks;
    if (uint64_t(plan.offset_blocks) > blocks) blocks = plan.offset_blocks;
    const size_t query = query_plan_lds(plan.p, c, eb, plan.queries.key_waves);
    const size_t key = key_lds(c.g.d, eb, plan.p, c.bias) + kKeyStatic;
    return DenseNeeds{blocks, query > key ? query : key};
}

hipError_t launch_dense_backward(int dtype, const DenseCall& c, const void* dO, void* dQ, void* dK, void* dV, void* dbias,
                                 void* workspace, hipStream_t stream, hipEvent_t start, hipEvent_t stop)
{
    BackwardPlan plan = backward_plan(c, elem_bytes_of(dtype));
    DenseBackward& p = plan.p;
    p.dO = dO;
    p.dQ = dQ;
    p.dK = dK;
    p.dV = dV;
    p.dbias = dbias;
    unsigned char* const ws = static_cast<unsigned char*>(workspace);
    p.stats = reinterpret_cast<float4*>(ws);
    p.part = reinterpret_cast<float*>(ws + plan.stats);
    p.diagonals = reinterpret_cast<float*>(ws + plan.stats + plan.part);
    return dispatch_value(dtype, c.g.d, hipErrorInvalidValue, [&](auto type, auto width) {
        using T = std::conditional_t<std::is_same<decltype(type), float>::value, float, uint16_t>;
        constexpr int D = decltype(width)::value;
        hipError_t e = query_dispatch<T, D>(c.bias, plan.queries.key_waves, [&](auto biased, auto key_waves) {
            constexpr int KW = decltype(key_waves)::value;
            constexpr bool kBiased = decltype(biased)::value;
            return launch_dense_kernel<kQueryThreads>(dense_query_kernel<T, D, kBiased, KW>, plan.queries.blocks,
                                                      query_block_lds<T, D, kBiased, KW>(p), stream, start, nullptr, p);
        });
        if (e != hipSuccess) return e;
        const hipEvent_t end = p.key_splits == 1 && !dbias ? stop : nullptr;
        const size_t lds = key_lds(D, sizeof(T), p, c.bias);
        e = c.bias ? launch_dense_kernel(dense_key_kernel<T, D, true>, plan.key_blocks, lds, stream, nullptr, end, p)
                   : launch_dense_kernel(dense_key_kernel<T, D, false>, plan.key_blocks, lds, stream, nullptr, end, p);
        if (e != hipSuccess) return e;
        if (p.key_splits > 1) {
            e = launch_dense_kernel(dense_key_join_kernel<T, D>, (p.all_keys * (D / 2) + kBlock - 1) / kBlock, 0, stream, nullptr,
                                    dbias ? nullptr : stop, p);
            if (e != hipSuccess) return e;
        }
        if (!dbias) return hipSuccess;
        e = launch_dense_kernel(dense_offset_kernel<T, D>, plan.offset_blocks, 0, stream, nullptr, nullptr, p);
        if (e != hipSuccess) return e;
        const int64_t blocks = (p.plane.rows * p.plane.size + kBlock - 1) / kBlock;
        return launch_dense_kernel(dense_offset_join_kernel<T>, blocks < 8192 ? blocks : 8192, 0, stream, nullptr, stop, p);
    });
}

}  // namespace scram
