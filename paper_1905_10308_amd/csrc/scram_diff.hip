// Differential attention over the match windows: forward.

#include "scram_diff.h"

namespace scram {
namespace {

// A lane group per query (WAVE: the lane groups of a wave share one query and
// add up at the end, for calls of a few queries).  One walk over the key set
// keeps two online softmaxes (base-2 domain) and their sums of values.  A key
// that is left out is not accumulated at all: whatever its rows hold stays out.
// MK = 0: one window, no mask; else up to MK windows and/or the causal mask.
template <typename T, int D, int G, int MK, bool WAVE>
__global__ __launch_bounds__(WAVE ? 64 : kBlock) void diff_attend_kernel(DiffParams p)
{
    constexpr bool MULTI = MK > 0;
    using RW = Row<T, D, G>;
    static_assert(RW::kCh == 2, "two chunks per lane: one of each half");
    constexpr int E = 2 * RW::kEpc;
    constexpr int kNb = 4;
    constexpr int kTeam = WAVE ? 64 / G : 1;
    const int lane = threadIdx.x & (G - 1);
    const int member = WAVE ? threadIdx.x / G : 0;
    uint32_t g;
    if constexpr (WAVE) {
        g = blockIdx.x;
    } else {
        if (!tile_item<RW::kQpb>(p.tq, xcd_remap(blockIdx.x, gridDim.x), threadIdx.x / G, g)) return;
    }
    uint32_t s, rem;
    divmod(g, p.div_plane, s, rem);
    const size_t slice = static_cast<size_t>(s) * p.nkeys * D;
    const T* Ks = static_cast<const T*>(p.K) + slice;
    const T* Vs = static_cast<const T*>(p.V) + slice;
    uint4 q[2];
    load_row<T, D, G>(static_cast<const T*>(p.Q), g, lane, q);
    WindowSet<(MK > 0 ? MK : 1)> ws;
    if constexpr (MULTI) {
        ws = make_window_set<MK>(p, g, rem);
        ws.local = causal_limit(p, s, rem);
    }

    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    float acc[2][E];
#pragma unroll
    for (int i = 0; i < E; ++i) acc[0][i] = acc[1][i] = 0.f;
    for (int e = 0; e < (MULTI ? p.kappa : 1); ++e) {
        uint32_t u, v;
        if constexpr (MULTI)
            ws.centre(e, u, v);
        else
            divmod(static_cast<uint32_t>(clamp_index(p.J[g], p.nkeys)), p.div_wk, u, v);
        walk_window<T, D, G, kNb, MK>(p, Ks, Vs, ws, e, u, v, member, kTeam, lane, [&](const auto& ok, const auto& kr, const auto& vr) {
            float sc[2][kNb];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float mb = m[h];
#pragma unroll
                for (int j = 0; j < kNb; ++j) {
                    sc[h][j] = half_score<T, G>(q[h], kr[j][h]) * p.scale_log2e;
                    mb = ok[j] ? fmaxf(mb, sc[h][j]) : mb;
                }
                if (mb > m[h] + kRescaleSlack) {
                    const float alpha = __builtin_amdgcn_exp2f(m[h] - mb);  // 0 on the first batch
                    l[h] *= alpha;
#pragma unroll
                    for (int i = 0; i < E; ++i) acc[h][i] *= alpha;
                    m[h] = mb;
                }
            }
#pragma unroll
            for (int j = 0; j < kNb; ++j) {
                if (!ok[j]) continue;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // (no score above -inf yet: weights 0, and a NaN score makes the row NaN)
                    const float pj = __builtin_amdgcn_exp2f(sc[h][j] - (m[h] == -INFINITY ? 0.f : m[h]));
                    l[h] += pj;
                    accumulate_row<T, 2>(acc[h], pj, vr[j]);
                }
            }
        });
    }
    if constexpr (WAVE) {
#pragma unroll
        for (int mask = G; mask < 64; mask <<= 1) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float mo = __shfl_xor(m[h], mask), top = fmaxf(m[h], mo);
                const float a = m[h] == top ? 1.f : __builtin_amdgcn_exp2f(m[h] - top);
                const float b = mo == top ? 1.f : __builtin_amdgcn_exp2f(mo - top);
                m[h] = top;
                l[h] = l[h] * a + __shfl_xor(l[h], mask) * b;
#pragma unroll
                for (int i = 0; i < E; ++i) acc[h][i] = acc[h][i] * a + __shfl_xor(acc[h][i], mask) * b;
            }
        }
        if (member != 0) return;
    }
    // an empty set gives a zero row
    const float i1 = l[0] != 0.f ? 1.f / l[0] : 0.f, i2 = l[1] != 0.f ? p.lam[s] / l[1] : 0.f;
    float o[E];
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = acc[0][i] * i1 - acc[1][i] * i2;
    store_row<T, D, G>(p.out, g, lane, o, 1.f);
}

template <typename T, int D, int MK>
hipError_t run_diff(const DiffParams& p0, hipStream_t st, hipEvent_t e0, hipEvent_t e1)
{
    constexpr int G = kDiffLanes<T, D>;
    DiffParams p = p0;
    if (p.n <= 4096) {
        if (e0 || e1)
            hipExtLaunchKernelGGL((diff_attend_kernel<T, D, G, MK, true>), dim3(p.n), dim3(64), 0, st, e0, e1, 0, p);
        else
            hipLaunchKernelGGL((diff_attend_kernel<T, D, G, MK, true>), dim3(p.n), dim3(64), 0, st, p);
        return hipGetLastError();
    }
    p.tq = make_tiling(p.Hq, p.Wq, Row<T, D, G>::kQpb, kLaneSkew);
    return launch(diff_attend_kernel<T, D, G, MK, false>, tiling_blocks(p.tq, p.n / p.tq.plane), st, e0, e1, p);
}

}  // namespace

hipError_t launch_diff_attend(int dtype, const DiffCall& c, void* out, hipStream_t stream, hipEvent_t start, hipEvent_t stop)
{
    DiffParams p{};
    fill_diff_params(p, c);
    p.out = out;
    return dispatch(dtype, c.g.d, [&](auto ty, auto d) {
        using T = decltype(ty);
        constexpr int D = decltype(d)::value;
        if (p.kappa == 1 && !p.causal) return run_diff<T, D, 0>(p, stream, start, stop);
        return p.kappa <= 2 ? run_diff<T, D, 2>(p, stream, start, stop) : run_diff<T, D, kMaxKappa>(p, stream, start, stop);
    });
}

uint64_t diff_attend_max_blocks(int dtype, const Grid& g)
{
    return dispatch_value(dtype, g.d, uint64_t(0), [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        return tiling_blocks(make_tiling(g.Hq, g.Wq, Row<T, D, kDiffLanes<T, D>>::kQpb, kLaneSkew), g.S);
    });
}

}  // namespace scram
