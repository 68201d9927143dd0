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
// Measured, bf16, 64 channels: 4 slices of 16384 queries and keys 428 us, 640 TFLOP/s (960 with the second part of the weights'
// product, without which it took 314 us), where a large matrix product reaches 1130 on the same card; its vector units are busy
// for 0.74 of the time and the matrix cores for 0.47 at 1.74 GHz, the clock that this load leaves.  16 slices of 4096 with a bias
// 141 us, 490 TFLOP/s.
//
// The waves of a block share its queries (32, 64 or 128) and its keys: KW of
// them take different keys of the same queries and join at the end.  Calls of
// few queries also split the keys over blocks; a second kernel joins those
// parts.  With a bias the part of its plane that the staged keys can meet is
// staged beside them.

#include "scram_dense.h"

namespace scram {
namespace {

struct DenseForward : DenseQueries {
    void* out;
    float* part;  // [splits][all rows][D], then [splits][all rows][2]: maximum, sum
};

// Waves to a SIMD: four where the registers suffice, also at the price of some spilled ones outside the steps (with a bias and two
// waves to a step's keys, 16 slices of 64 x 64: 147 us, with two waves a SIMD 161).  Calls of fewer queries have no more than
// one block a CU, which spilling only slows down (16 of 32 x 32: 16.8 us, 19.1 spilled).  fp32 rows of 128 channels with a bias
// spill with two waves too (96 bytes a lane).
template <typename T, int D, bool BIAS, int KW>
__global__ __launch_bounds__(kQueryThreads, D * sizeof(T) > 128 || (BIAS && KW > 2) ? 2 : 4) void dense_kernel(
    DenseForward p)
{
    using R = DenseRow<T, D>;
    // in bf16 without a bias the scale and the shift enter the exponential's argument in one step (a certain key's weight is
    // then off 1 by the shift's rounding, as their sum is, which divides it)
    constexpr bool kFold = sizeof(T) == 2 && !BIAS;
    extern __shared__ __align__(16) unsigned char lds[];
    QueryBlock<T, D, BIAS, KW> q(p, lds);
    const int lane = q.lane, h = q.h, wave = q.wave, qw = q.qw, kw = q.kw, split = q.split;
    const bool live = q.live;
    const int64_t out_row = q.out_row;
    uint4 qf[R::kSteps];
    load_operand<T, D>(p.Q, q.from_row(), h, qf);
    if constexpr (kFold) q.positive_scale(qf);
    const float scale2 = q.scale2;

    f32x16_t o[R::kColumns];
    // Weights are exp2(score - shift).  Any shift will do that is near a query's largest score; the largest of its first keys
    // is, but for queries that far larger ones await.  So nothing is scaled on the way: the largest score is kept beside, and
    // where it leaves the shift too far behind, the block passes over its keys again.
    float sum, shift = 0.f, most;
    for (int pass = 0;; ++pass) {
#pragma unroll
        for (int c = 0; c < R::kColumns; ++c) o[c] = f32x16_t(0.f);
        sum = 0.f;
        most = -INFINITY;
        bool first = pass == 0;
        q.pass([&](auto at, const int* places, int from, int k0) {
            constexpr int kAt = decltype(at)::value;
            f32x16_t s = q.products(kAt, qf);
            q.template scores<kFold>(s, places, from, k0);
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, s[i]);
            if (first) {
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
                const RightOperand<T> w = as_operand<T>(s, r);
#pragma unroll
                for (int c = 0; c < R::kColumns; ++c)
                    o[c] = mma<T>(q.reader.column(r, c, kAt + q.kValues), w, o[c]);
            }
        });
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
    // the waves of the same queries: each joins a share of the channels
    constexpr int kPart = 64 * (16 * R::kColumns + 2);
    float* const joined = reinterpret_cast<float*>(lds);
    {
        float* const to = joined + wave * kPart + lane;
        to[0] = sum == 0.f ? -INFINITY : shift;
        to[64] = sum;
#pragma unroll
        for (int c = 0; c < R::kColumns; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) to[64 * (2 + 16 * c + i)] = o[c][i];
    }
    __syncthreads();
    if (!live) return;
    const float* const from = joined + qw * kPart + lane;
    float top = -INFINITY, factor[KW];
    for (int k = 0; k < KW; ++k) top = fmaxf(top, from[k * (8 / KW) * kPart]);
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < KW; ++k) {
        const float one = from[k * (8 / KW) * kPart + 64];
        factor[k] = one == 0.f ? 0.f : __builtin_amdgcn_exp2f(from[k * (8 / KW) * kPart] - top);  // 0: no key
        sum = fmaf(one, factor[k], sum);
    }
    float* ml = nullptr;
    if (p.splits > 1) {
        const int64_t at_part = static_cast<int64_t>(split) * p.all_rows + out_row;
        ml = p.part + static_cast<int64_t>(p.splits) * p.all_rows * D + 2 * at_part;
        if (h == 0 && kw == 0) {
            ml[0] = top;
            ml[1] = sum;
        }
        if (sum == 0.f) return;  // a part without a key is not read
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    constexpr int kQuads = D < 32 ? 2 : 4 * R::kColumns;
    for (int g = kw; g < kQuads; g += KW) {
        float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KW; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float y = from[k * (8 / KW) * kPart + 64 * (2 + 4 * g + j)];
                x[j] = factor[k] == 0.f ? x[j] : fmaf(factor[k], y, x[j]);
            }
        const int channel = 8 * g + 4 * h;
        if (p.splits > 1) {
            *reinterpret_cast<float4*>(p.part + (static_cast<int64_t>(split) * p.all_rows + out_row) * D + channel) =
                make_float4(x[0], x[1], x[2], x[3]);
        } else {
            vec<T, 4> y;
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = from_float<T>(x[j] * inv);
            store_vec<T, 4>(static_cast<T*>(p.out) + out_row * D + channel, y);
        }
    }
}

// Joins the parts of the splits: a thread takes four channels of a row, eight parts at a time.
template <typename T, int D>
__global__ __launch_bounds__(kBlock) void dense_join_kernel(DenseForward p)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x, row = i / (D / 4);
    if (row >= p.all_rows) return;
    const int c = static_cast<int>(i % (D / 4)) * 4;
    const float2* const ml = reinterpret_cast<const float2*>(p.part + static_cast<int64_t>(p.splits) * p.all_rows * D) + row;
    float top = -INFINITY;
    for (int s0 = 0; s0 < p.splits; s0 += 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, s0 + j < p.splits ? ml[(s0 + j) * p.all_rows].x : -INFINITY);
    }
    float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < p.splits; s0 += 8) {
        float2 st[8];
        float4 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            st[j] = s0 + j < p.splits ? ml[(s0 + j) * p.all_rows] : make_float2(0.f, 0.f);
            // (nothing was written for a part without a key)
            x[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (st[j].y != 0.f) x[j] = *reinterpret_cast<const float4*>(p.part + ((s0 + j) * p.all_rows + row) * D + c);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float w = st[j].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(st[j].x - top);
            sum = fmaf(w, st[j].y, sum);
            o[0] = fmaf(w, x[j].x, o[0]);
            o[1] = fmaf(w, x[j].y, o[1]);
            o[2] = fmaf(w, x[j].z, o[2]);
            o[3] = fmaf(w, x[j].w, o[3]);
        }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    vec<T, 4> y;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = from_float<T>(o[j] * inv);
    store_vec<T, 4>(static_cast<T*>(p.out) + row * D + c, y);
}

struct ForwardPlan {
    DenseForward p;
    QueryPlan queries;
};

ForwardPlan forward_plan(const DenseCall& c, int elem_bytes)
{
    ForwardPlan plan{};
    static_cast<DenseParams&>(plan.p) = dense_params(c);
    plan.queries = query_plan(c, elem_bytes, true, plan.p);
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

DenseNeeds dense_needs(int dtype, const DenseCall& c)
{
    const int eb = elem_bytes_of(dtype);
    const ForwardPlan plan = forward_plan(c, eb);
    return DenseNeeds{2 * uint64_t(plan.queries.blocks), query_plan_lds(plan.p, c, eb, plan.queries.key_waves)};
}

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
        const hipError_t e = query_dispatch<T, D>(c.bias, plan.queries.key_waves, [&](auto biased, auto key_waves) {
            constexpr int KW = decltype(key_waves)::value;
            constexpr bool kBiased = decltype(biased)::value;
            return launch_dense_kernel<kQueryThreads>(dense_kernel<T, D, kBiased, KW>, plan.queries.blocks,
                                                      query_block_lds<T, D, kBiased, KW>(p), stream, start, end, p);
        });
        if (e != hipSuccess || p.splits == 1) return e;
        return launch_dense_kernel(dense_join_kernel<T, D>, (p.all_rows * (D / 4) + kBlock - 1) / kBlock, 0, stream, nullptr, stop, p);
    });
}

}  // namespace scram
