// Differential attention over the match windows: what the forward
// (scram_diff.hip) and the gradients (scram_diff_backward.hip) share.
//
// A row of D channels holds two maps' channels, the first half and the last.
// With W_i the key set of query i (the union of its windows, as in the attend),
// p1 and p2 the softmaxes of scale q1.k1 and scale q2.k2 over W_i and lam a
// weight per slice,
//   o_i = sum_j (p1_ij - lam p2_ij) v_j.
// The lanes of a query hold 32 bytes of a row each, as two 16-byte chunks, and
// chunk 0 of every lane lies in the first half, chunk 1 in the last.
//
// Everything here lives in an unnamed namespace, like scram_device.h.

#pragma once

#include "scram_grad.h"

namespace scram {
namespace {

struct DiffParams : BwdParams {
    void* out;
    const float* lam;      // [S]
    const int32_t* origin; // [S] raster index of each slice's first query among the keys (null: first)
    int first;
    int tile_blocks;       // most blocks of 16 keys a wave walks on the matrix cores
    float4* stats;         // [n] log2 normaliser and D of both maps (gradients); kOneKey
    double* lam_part;      // [slices, parts] sums over some queries each of D of the second map
    uint32_t slices, parts;
    float* dlam;           // [S]
};

template <typename T, int D>
constexpr int kDiffLanes = D * static_cast<int>(sizeof(T)) / 32;

// Raster index of the last key that query `rem` of slice s may see.
__device__ __forceinline__ uint32_t causal_limit(const DiffParams& p, uint32_t s, uint32_t rem)
{
    const int32_t at = p.origin != nullptr ? clamp_index(p.origin[s], p.nkeys) : p.first;
    return static_cast<uint32_t>(at) + rem;
}

// Whether query g's set is one key: centre(e, u, v) gives the centre of its window e, `limit` its last key.  With windows of
// more than one key and a grid of more than one only the causal mask leaves so few.
template <typename Centre>
__device__ __forceinline__ bool one_key_set(const DiffParams& p, uint32_t limit, int kappa, Centre&& centre)
{
    if (p.b > 0 && !p.causal && p.nkeys > 1) return false;
    if (!p.causal) limit = p.nkeys - 1;
    uint32_t only = 0xFFFFFFFFu;
    for (int e = 0; e < kappa; ++e) {
        int u, v;
        centre(e, u, v);
        // the window's first two keys in raster order
        const int r0 = max(u - p.b, 0), c0 = max(v - p.b, 0);
        const uint32_t first = static_cast<uint32_t>(r0) * p.Wk + c0;
        const uint32_t second = c0 < min(v + p.b, p.Wk - 1) ? first + 1 : r0 < min(u + p.b, p.Hk - 1) ? first + p.Wk : 0xFFFFFFFFu;
        if (first > limit) continue;
        if (second <= limit || (only != 0xFFFFFFFFu && only != first)) return false;
        only = first;
    }
    return only != 0xFFFFFFFFu;
}

// A set of one key: both softmaxes are 1 and the gradients of the scores 0, exactly, in whatever order the key side adds up
// the score and dP.  Such a query's statistics hold this number (a NaN that no sum gives) in the place of D of the second map.
constexpr uint32_t kOneKey = 0x7FFFFFFFu;

__device__ __forceinline__ bool is_one_key(const float4& stats) { return __float_as_uint(stats.w) == kOneKey; }

// A query's statistics; one: its set is one key, whose numbers are finite (what is not goes the common way and shows).
__device__ __forceinline__ float4 query_stats(const float (&lse)[2], const float (&D)[2], bool one)
{
    // (a NaN of the input's own is not to be taken for that number)
    const float last = __float_as_uint(D[1]) == kOneKey ? __uint_as_float(0x7FC00000u) : D[1];
    return make_float4(lse[0], D[0], lse[1], one ? __uint_as_float(kOneKey) : last);
}

__device__ __forceinline__ bool finite_stats(const float (&lse)[2], const float (&D)[2])
{
    return fabsf(lse[0]) < INFINITY && fabsf(lse[1]) < INFINITY && fabsf(D[0]) < INFINITY && fabsf(D[1]) < INFINITY;
}

// One half's part of a dot product, over the lane group.
template <typename T, int G>
__device__ __forceinline__ float half_score(uint4 a, uint4 b)
{
    const uint4 x[1] = {a}, y[1] = {b};
    return group_sum<G>(lane_dot<T, 1>(x, y));
}

// Walks one window (centre (u, v), clipped to the grid) in row order, kNb keys
// at a time with their key and value rows loaded together: member `member` of
// `team` lane groups takes slots member, member + team, ...
// fn(ok[], kr[][2], vr[][2]); slots that are left out read the centre's row.
template <typename T, int D, int G, int kNb, int MK, typename F>
__device__ __forceinline__ void walk_window(const DiffParams& p, const T* Ks, const T* Vs, const WindowSet<(MK > 0 ? MK : 1)>& ws,
                                            int e, uint32_t u, uint32_t v, int member, int team, int lane, F&& fn)
{
    const int r0 = max(static_cast<int>(u) - p.b, 0), r1 = min(static_cast<int>(u) + p.b, p.Hk - 1);
    const int c0 = max(static_cast<int>(v) - p.b, 0), c1 = min(static_cast<int>(v) + p.b, p.Wk - 1);
    const int cw = c1 - c0 + 1, nwin = (r1 - r0 + 1) * cw;
    const uint32_t centre = u * p.Wk + v;
    int r = r0, c = c0, qs = 0, rs = 1;
    if (team > 1) {
        r = r0 + member / cw, c = c0 + member % cw;
        qs = team / cw, rs = team % cw;
    }
    for (int k0 = member; k0 < nwin; k0 += kNb * team) {
        uint4 kr[kNb][2], vr[kNb][2];
        bool ok[kNb];
#pragma unroll
        for (int j = 0; j < kNb; ++j) {
            ok[j] = k0 + j * team < nwin;
            if constexpr (MK > 0) ok[j] = ok[j] && !ws.skip(e, r, c);
            const uint32_t row = ok[j] ? static_cast<uint32_t>(r * p.Wk + c) : centre;
            load_row<T, D, G>(Ks, row, lane, kr[j]);
            load_row<T, D, G>(Vs, row, lane, vr[j]);
            c += rs;
            r += qs;
            if (c > c1) {
                c -= cw;
                ++r;
            }
        }
        fn(ok, kr, vr);
    }
}

inline void fill_diff_params(DiffParams& p, const DiffCall& c)
{
    const Grid& g = c.g;
    p.Q = c.Q;
    p.K = c.K;
    p.V = c.V;
    p.J = c.J;
    p.lam = c.lam;
    p.origin = c.causal ? c.origin : nullptr;
    p.first = c.causal ? c.first : 0;
    p.n = static_cast<uint32_t>(g.S) * g.Hq * g.Wq;
    p.Hq = g.Hq;
    p.Wq = g.Wq;
    p.Hk = g.Hk;
    p.Wk = g.Wk;
    p.nkeys = static_cast<uint32_t>(g.Hk) * g.Wk;
    p.keys_total = static_cast<uint32_t>(g.S) * p.nkeys;
    p.div_plane = make_div(static_cast<uint32_t>(g.Hq) * g.Wq);
    p.div_wk = make_div(g.Wk);
    p.div_n = make_div(p.n);
    p.div_keys = make_div(p.nkeys);
    p.b = c.window / 2;
    p.scale = c.scale;
    p.scale_log2e = c.scale * 1.4426950408889634f;
    p.kappa = c.kappa;
    p.causal = c.causal ? 1 : 0;
}

}  // namespace
}  // namespace scram
