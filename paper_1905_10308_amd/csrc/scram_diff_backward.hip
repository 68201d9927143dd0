// Gradients of the differential attention over the match windows (maps held
// fixed).  With dp_ij = dO_i.v_j and D1_i = sum_j p1_ij dp_ij, D2_i likewise:
//   dQ1_i =       scale sum_j p1_ij (dp_ij - D1_i) k1_j
//   dQ2_i = - lam scale sum_j p2_ij (dp_ij - D2_i) k2_j
//   dK1_j =       scale sum_i p1_ij (dp_ij - D1_i) q1_i,  dK2_j likewise with - lam
//   dV_j  = sum_i (p1_ij - lam p2_ij) dO_i
//   dlam  = - sum_i D2_i over the slice's queries
// The query side walks each query's key set once, as the attend's gradients
// do; the key side gathers over the queries whose windows hold the key,
// through the inverse of the maps (scram_inverse.h).  No float atomics: every
// gradient row has one writer.

#include "scram_diff_tile.h"
#include "scram_strip.h"

#include <algorithm>

namespace scram {
namespace {

// Sum of x over the block's threads (kBlock), in a fixed order, on thread 0.
__device__ double block_sum(double x)
{
    __shared__ double s_wave[kBlock / 64];
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) x += __shfl_xor(x, m);
    if ((threadIdx.x & 63) == 0) s_wave[threadIdx.x >> 6] = x;
    __syncthreads();
    double t = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kBlock / 64; ++w) t += s_wave[w];
    return t;
}

// The inverse map's count of query g of slice s: one entry per match, and its slot among that match key's.
__device__ __forceinline__ void count_matches(const DiffParams& p, uint32_t g, uint32_t s)
{
    for (int e = 0; e < p.kappa; ++e) {
        const size_t x = static_cast<size_t>(e) * p.n + g;
        p.slots[x] = atomicAdd(p.counts + static_cast<size_t>(s) * p.nkeys + clamp_index(p.J[x], p.nkeys), 1);
    }
}

// Query g on a lane group: its dQ row and statistics; returns D of the second map (on lane 0, 0 on the others).  As in the
// attend's gradients the keys enter as k_j - k_ref, k_ref the key at the first match: the weights of a set sum to one, so
// dQ = scale (A - D B) / l for any fixed k_ref, and A - D B does not cancel where neighbouring keys are alike.
template <typename T, int D, int G, int MK>
__device__ __forceinline__ float diff_query_gradient(const DiffParams& p, uint32_t g, int lane)
{
    constexpr bool MULTI = MK > 0;
    using RW = Row<T, D, G>;
    static_assert(RW::kCh == 2, "two chunks per lane: one of each half");
    constexpr int H = RW::kEpc;  // channels per lane of each half
    constexpr int kNb = 3;
    uint32_t s, rem;
    divmod(g, p.div_plane, s, rem);
    const size_t slice = static_cast<size_t>(s) * p.nkeys * D;
    const T* Ks = static_cast<const T*>(p.K) + slice;
    const T* Vs = static_cast<const T*>(p.V) + slice;
    uint4 q[2], go[2];
    load_row<T, D, G>(static_cast<const T*>(p.Q), g, lane, q);
    load_row<T, D, G>(static_cast<const T*>(p.dO), g, lane, go);
    WindowSet<(MK > 0 ? MK : 1)> ws;
    if constexpr (MULTI) {
        ws = make_window_set<MK>(p, g, rem);
        ws.local = causal_limit(p, s, rem);
    }
    float kref[2 * H];
    {
        uint4 kr0[2] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
        const uint32_t at = static_cast<uint32_t>(clamp_index(p.J[g], p.nkeys));
        // (a match after the query is not in its set: its row stays out, and k_ref is 0)
        if (!MULTI || !p.causal || at <= ws.local) load_row<T, D, G>(Ks, at, lane, kr0);
        unpack_row<T, 2>(kr0, kref);
    }
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, dn[2] = {0.f, 0.f};
    float A[2][H], B[2][H];
#pragma unroll
    for (int i = 0; i < H; ++i) A[0][i] = A[1][i] = B[0][i] = B[1][i] = 0.f;
    for (int e = 0; e < (MULTI ? p.kappa : 1); ++e) {
        uint32_t u, v;
        if constexpr (MULTI)
            ws.centre(e, u, v);
        else
            divmod(static_cast<uint32_t>(clamp_index(p.J[g], p.nkeys)), p.div_wk, u, v);
        walk_window<T, D, G, kNb, MK>(p, Ks, Vs, ws, e, u, v, 0, 1, lane, [&](const auto& ok, const auto& kr, const auto& vr) {
            float sc[2][kNb], dp[kNb];
#pragma unroll
            for (int j = 0; j < kNb; ++j) dp[j] = row_score<T, D, G>(go, vr[j]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float mb = m[h];
#pragma unroll
                for (int j = 0; j < kNb; ++j) {
                    sc[h][j] = half_score<T, G>(q[h], kr[j][h]) * p.scale_log2e;
                    mb = ok[j] ? fmaxf(mb, sc[h][j]) : mb;
                }
                if (mb > m[h] + kRescaleSlack) {
                    const float alpha = __builtin_amdgcn_exp2f(m[h] - mb);
                    l[h] *= alpha;
                    dn[h] *= alpha;
#pragma unroll
                    for (int i = 0; i < H; ++i) A[h][i] *= alpha, B[h][i] *= alpha;
                    m[h] = mb;
                }
            }
#pragma unroll
            for (int j = 0; j < kNb; ++j) {
                if (!ok[j]) continue;
                float kf[2 * H];
                unpack_row<T, 2>(kr[j], kf);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float pj = __builtin_amdgcn_exp2f(sc[h][j] - (m[h] == -INFINITY ? 0.f : m[h]));
                    const float pd = pj * dp[j];
                    l[h] += pj;
                    dn[h] += pd;
#pragma unroll
                    for (int i = 0; i < H; ++i) {
                        const float kd = kf[h * H + i] - kref[h * H + i];
                        A[h][i] = fmaf(pd, kd, A[h][i]);
                        B[h][i] = fmaf(pj, kd, B[h][i]);
                    }
                }
            }
        });
    }
    float Dh[2], lse[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float inv = l[h] != 0.f ? 1.f / l[h] : 0.f;
        Dh[h] = dn[h] * inv;
        lse[h] = l[h] != 0.f ? m[h] + log2f(l[h]) : INFINITY;  // +inf: every weight is 0
        const float f = (h == 0 ? p.scale : -p.lam[s] * p.scale) * inv;
        float4* o = reinterpret_cast<float4*>(p.dQ + static_cast<size_t>(g) * D + (h * G + lane) * H);
#pragma unroll
        for (int i = 0; i < H / 4; ++i)
            o[i] = make_float4((A[h][4 * i] - Dh[h] * B[h][4 * i]) * f, (A[h][4 * i + 1] - Dh[h] * B[h][4 * i + 1]) * f,
                               (A[h][4 * i + 2] - Dh[h] * B[h][4 * i + 2]) * f, (A[h][4 * i + 3] - Dh[h] * B[h][4 * i + 3]) * f);
    }
    if (lane != 0) return 0.f;
    bool one = p.b == 0 || p.nkeys == 1;  // one window, no mask
    if constexpr (MULTI)
        one = one_key_set(p, ws.local, p.kappa, [&](int e, int& u, int& v) {
            uint32_t uu, vv;
            ws.centre(e, uu, vv);
            u = static_cast<int>(uu), v = static_cast<int>(vv);
        });
    p.stats[g] = query_stats(lse, Dh, one && finite_stats(lse, Dh));
    return Dh[1];
}

// A lane group per query.
template <typename T, int D, int G, int MK>
__global__ __launch_bounds__(kBlock) void diff_query_kernel(DiffParams p)
{
    const int lane = threadIdx.x & (G - 1);
    const uint32_t blk = xcd_remap(blockIdx.x, gridDim.x);
    uint32_t g;
    float D2 = 0.f;
    if (tile_item<Row<T, D, G>::kQpb>(p.tq, blk, threadIdx.x / G, g)) {
        if (lane == 0) {
            uint32_t s, rem;
            divmod(g, p.div_plane, s, rem);
            count_matches(p, g, s);
        }
        D2 = diff_query_gradient<T, D, G, MK>(p, g, lane);
    }
    const double part = block_sum(D2);
    if (threadIdx.x == 0) p.lam_part[blk] = part;
}

// Waves per SIMD that the tile kernel's registers are sized for.
constexpr int diff_grad_waves(int D) { return D == 128 ? 1 : D == 64 ? 2 : 3; }

// On the matrix cores (scram_diff_tile.h), bf16, a wave of 16 queries.  Per block of 16 keys
//   S1^T, S2^T = K_blk Q^T,  dP^T = V_blk dO^T         keys x queries
//   P1, P2 = 2^(S scale log2 e - reference) on the query's keys, 0 elsewhere;  PD = P dP
//   B^T += K_blk^T P^T,  A^T += K_blk^T PD^T           channels x queries: the first half's with P1, the last with P2
//   l += 1^T P^T,  dn += 1^T PD^T                      all-ones blocks, of each map
// with the weights as three bf16 parts that add up to them (the gradients are fp32).  With D = dn / l and k_ref the key at the
// first match (0 where the causal mask takes it away), dQ = scale ((A - dn k_ref) - D (B - l k_ref)) / l.  In exact arithmetic
// those are the lane group's sums; here whole keys are added up and k_ref comes off at the end, so a common offset of the keys
// is rounded with them: keys 8 (64) times their spread away from 0 cost 1.3e-6 (9e-6) of dQ, a plain 32-bit computation 1e-6
// (8e-6), a lane group 2.8e-7 whatever the offset.
// A query whose sums are not finite, or whose set is empty, is computed over again on a lane group, and so are a wave's
// queries whose matches lie too far apart to share rows.
// 16 x 128 x 128, 64 channels, two 5 x 5 windows: 190-203 us, at 2 waves per SIMD the vector units (splitting the weights) issuing
// in 67 % of the cycles, the loads' return path busy in 73 %, the matrix cores in 31 %.
template <int D, int W, bool CAUSAL, int MK>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(diff_grad_waves(D)))) void
diff_query_tile_kernel(DiffParams p)
{
    using TR = TileRow<D>;
    constexpr int kOt = D / 16, kRowB = 2 * D + kRowPad;
    constexpr int G = kDiffLanes<uint16_t, D>;
    __shared__ __align__(16) unsigned char tk[16 * kRowB], tv[16 * kRowB];
    const int lane = threadIdx.x, m = lane & 15, g4 = lane >> 4;
    const uint32_t one = xcd_remap(blockIdx.x, gridDim.x), blk = one / 4;
    const int wave = static_cast<int>(one % 4);
    const DiffTile<MK> t = diff_tile<W, MK>(p, blk, wave, lane, p.tile_blocks);
    if (t.valid && g4 == 0) count_matches(p, t.g, t.s);
    uint32_t todo = t.tc.nclu == 0 ? 0u : 0xFFFFu;  // queries left to the lane groups
    float D2 = 0.f;
    if (t.tc.nclu > 0) {
        const size_t slice = static_cast<size_t>(__builtin_amdgcn_readfirstlane(t.s)) * p.nkeys * static_cast<size_t>(2 * D);
        const unsigned char* const Kb = static_cast<const unsigned char*>(p.K) + slice;
        const unsigned char* const Vb = static_cast<const unsigned char*>(p.V) + slice;
        HalfQueries<D> q;
        q.load(static_cast<const unsigned char*>(p.Q) + static_cast<size_t>(t.gq) * (2 * D), g4);
        typename TR::Frag go[TR::kDs];
#pragma unroll
        for (int ds = 0; ds < TR::kDs; ++ds)
            go[ds] = TR::frag(static_cast<const unsigned char*>(p.dO) + static_cast<size_t>(t.gq) * (2 * D), ds, g4);
        MapReference ref[2];
        const bool held = !CAUSAL || t.centre <= t.limit;  // the first match is a key of the query's set
        {
            float s0[2];
            q.own_scores(Kb + t.centre * (2u * D), g4, s0);
            ref[0].start(s0[0], held, p.scale_log2e);
            ref[1].start(s0[1], held, p.scale_log2e);
        }
        const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
        const bf16x4_t ones = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f), static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
        f32x4_t A[kOt], B[kOt], l[2], dn[2];
#pragma unroll
        for (int o = 0; o < kOt; ++o) A[o] = B[o] = zero;
        l[0] = l[1] = dn[0] = dn[1] = zero;
        diff_walk<D, W, CAUSAL, MK>(p, t, Kb, Vb, tk, tv, lane, [&](f32x4_t bias) {
            f32x4_t sc[2], dp = zero;
            q.scores([&](int ds) { return TR::frag(tk + m * kRowB, ds, g4); }, bias, sc);
#pragma unroll
            for (int ds = 0; ds < TR::kDs; ++ds) dp = TR::product(TR::frag(tv + m * kRowB, ds, g4), go[ds], dp);
            float x[2][4];
            block_weights(ref, sc, p.scale_log2e, x, [&](int h, float f) {
                l[h] *= f;
                dn[h] *= f;
#pragma unroll
                for (int o = 0; o < kOt; ++o)
                    if (o / (kOt / 2) == h) A[o] *= f, B[o] *= f;
            });
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Parts3 w = parts3(x[h]);
                l[h] = product3(ones, w, l[h]);
                float y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = x[h][i] * dp[i];
                const Parts3 wd = parts3(y);
                dn[h] = product3(ones, wd, dn[h]);
#pragma unroll
                for (int o = h * (kOt / 2); o < (h + 1) * (kOt / 2); ++o) {
                    const bf16x4_t kt = column4<D>(tk, m, g4, o);
                    B[o] = product3(kt, w, B[o]);
                    A[o] = product3(kt, wd, A[o]);
                }
            }
        });
        float inv[2], Dh[2], lse[2], size = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            inv[h] = 1.f / l[h][0];  // an empty set's is infinite
            Dh[h] = dn[h][0] * inv[h];
            lse[h] = ref[h].ref + log2f(l[h][0]);
            size += inv[h] + fabsf(Dh[h]);
            inv[h] *= h == 0 ? p.scale : -p.lam[t.s] * p.scale;
        }
        bool one = false;
        if constexpr (CAUSAL) {
            one = one_key_set(p, t.limit, MK, [&](int e, int& u, int& v) {
                // (unrolled: indexes known at compile time keep the centres in registers; those past kappa repeat the first)
                u = t.u[0], v = t.v[0];
#pragma unroll
                for (int f = 1; f < MK; ++f)
                    if (f == e) u = t.u[f], v = t.v[f];
            }) && finite_stats(lse, Dh);
            if (one) inv[0] = inv[1] = 0.f;
        }
        // lane holds channels 16 o + 4 g4 + i of query m
        const unsigned char* const krow = Kb + t.centre * (2u * D);
#pragma unroll
        for (int o = 0; o < kOt; ++o) {
            const int h = o / (kOt / 2);
            uint2 kw = *reinterpret_cast<const uint2*>(krow + 32 * o + 8 * g4);
            if (CAUSAL && !held) kw = make_uint2(0u, 0u);  // (whatever that row holds stays out: k_ref is 0)
            const float kref[4] = {__uint_as_float(kw.x << 16), __uint_as_float(kw.x & 0xFFFF0000u), __uint_as_float(kw.y << 16),
                                   __uint_as_float(kw.y & 0xFFFF0000u)};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                A[o][i] = ((A[o][i] - dn[h][0] * kref[i]) - Dh[h] * (B[o][i] - l[h][0] * kref[i])) * inv[h];
                size += fabsf(A[o][i]);
            }
        }
        const uint64_t bad = __ballot(!(fabsf(size) < INFINITY));
        todo = static_cast<uint32_t>(bad | bad >> 16 | bad >> 32 | bad >> 48) & 0xFFFFu;
        if (t.valid && !((todo >> m) & 1u)) {
            if (g4 == 0) {
                p.stats[t.g] = query_stats(lse, Dh, one);
                D2 = Dh[1];
            }
#pragma unroll
            for (int o = 0; o < kOt; ++o)
                *reinterpret_cast<f32x4_t*>(p.dQ + static_cast<size_t>(t.g) * D + 16 * o + 4 * g4) = A[o];
        }
    }
    double part = D2;
    for (int i = lane / G; i < 16; i += 64 / G) {
        uint32_t g;
        if (((todo >> i) & 1u) && tile_item<kBlock / 4>(p.tq, blk, tile_wave_item(p.tq, wave, i), g))
            part += diff_query_gradient<uint16_t, D, G, (CAUSAL || MK > 1 ? MK : 0)>(p, g, lane & (G - 1));
    }
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) part += __shfl_xor(part, k);
    if (lane == 0) p.lam_part[one] = part;
}

// dlam of the slices: minus the sums of their parts, a block per slice at a time.
__device__ __forceinline__ void slice_sums(const DiffParams& p)
{
    for (uint32_t s = blockIdx.x; s < p.slices; s += gridDim.x) {
        double x = 0.0;
        for (uint32_t i = threadIdx.x; i < p.parts; i += kBlock) x += p.lam_part[static_cast<size_t>(s) * p.parts + i];
        x = block_sum(x);
        if (threadIdx.x == 0) p.dlam[s] = static_cast<float>(-x);
        __syncthreads();  // before the next sum's writes
    }
}

// Contributions of kNb entries (slots x[t], valid where ok[t]) to dK_j, dV_j
// (unscaled dK) for key j at (ju, jv): each query once -- through its first
// window holding j -- and, with the causal mask, only if j is not after it.
template <typename T, int D, int G, bool MULTI, int kNb>
__device__ __forceinline__ void diff_key_batch(const DiffParams& p, const int (&x)[kNb], const bool (&valid)[kNb], float lam,
                                               const KeyPos& k, int lane, const uint4 (&kj)[2], const uint4 (&vj)[2], float* dk,
                                               float* dv)
{
    constexpr int H = Row<T, D, G>::kEpc;
    uint4 qr[kNb][2], gr[kNb][2];
    float4 st[kNb];
    uint32_t e[kNb], g[kNb];
#pragma unroll
    for (int t = 0; t < kNb; ++t) divmod(static_cast<uint32_t>(p.entries[x[t]]), p.div_n, e[t], g[t]);
#pragma unroll
    for (int t = 0; t < kNb; ++t) {
        st[t] = p.stats[g[t]];
        load_row<T, D, G>(static_cast<const T*>(p.Q), g[t], lane, qr[t]);
        load_row<T, D, G>(static_cast<const T*>(p.dO), g[t], lane, gr[t]);
    }
#pragma unroll
    for (int t = 0; t < kNb; ++t) {
        bool ok = valid[t];
        if constexpr (MULTI) {
            for (int f = 0; f < static_cast<int>(e[t]) && ok; ++f) {
                uint32_t fu, fv;
                divmod(static_cast<uint32_t>(clamp_index(p.J[static_cast<size_t>(f) * p.n + g[t]], p.nkeys)), p.div_wk, fu, fv);
                ok = abs(static_cast<int>(fu) - static_cast<int>(k.ju)) > p.b || abs(static_cast<int>(fv) - static_cast<int>(k.jv)) > p.b;
            }
            if (ok && p.causal) {
                uint32_t gs, rem;
                divmod(g[t], p.div_plane, gs, rem);
                ok = k.j <= causal_limit(p, gs, rem);
            }
        }
        if (!ok) continue;
        const float dp = row_score<T, D, G>(gr[t], vj);
        const bool one = is_one_key(st[t]);
        const float p1 = __builtin_amdgcn_exp2f(half_score<T, G>(qr[t][0], kj[0]) * p.scale_log2e - st[t].x);
        const float p2 = lam * __builtin_amdgcn_exp2f(half_score<T, G>(qr[t][1], kj[1]) * p.scale_log2e - st[t].z);
        const float ds[2] = {one ? 0.f : p1 * (dp - st[t].y), one ? 0.f : -p2 * (dp - st[t].w)};
        const float w = p1 - p2;
        float qf[2 * H], gf[2 * H];
        unpack_row<T, 2>(qr[t], qf);
        unpack_row<T, 2>(gr[t], gf);
#pragma unroll
        for (int i = 0; i < 2 * H; ++i) {
            dk[i] = fmaf(ds[i / H], qf[i], dk[i]);
            dv[i] = fmaf(w, gf[i], dv[i]);
        }
    }
}

// The entries of key k's neighbourhood (`total` of them) taken by member `member` of a team of
// `team` lane groups.  RUNS: added up in runs of the square root of their
// number, and the runs then onto the sums: entries whose terms are alike round
// the same way, and one after another onto a sum of thousands lost 2e-5 of it
// (65536 queries of one key; 5e-4 at 2^20).
template <typename T, int D, int G, bool MULTI, bool RUNS>
__device__ __forceinline__ void diff_key_sums(const DiffParams& p, const KeyPos& k, int total, int member, int team, int lane,
                                              const uint4 (&kj)[2], const uint4 (&vj)[2], float* dk, float* dv)
{
    constexpr int kNb = 2, N = 2 * Row<T, D, G>::kEpc;
    const int32_t* off = p.offsets + static_cast<size_t>(k.s) * p.nkeys;
    const float lam = p.lam[k.s];
    float rk[RUNS ? N : 1], rv[RUNS ? N : 1];
    const int run = RUNS ? max(16, static_cast<int>(sqrtf(static_cast<float>(total / (kNb * team))))) : 0;
    int left = run;
    auto flush = [&](bool first) {
#pragma unroll
        for (int i = 0; i < (RUNS ? N : 0); ++i) {
            if (!first) dk[i] += rk[i], dv[i] += rv[i];
            rk[i] = rv[i] = 0.f;
        }
        left = run;
    };
    auto batch = [&](const int (&x)[kNb], const bool (&valid)[kNb]) {
        diff_key_batch<T, D, G, MULTI, kNb>(p, x, valid, lam, k, lane, kj, vj, RUNS ? rk : dk, RUNS ? rv : dv);
        if (RUNS && --left == 0) flush(false);
    };
    flush(true);
    if (k.r1 - k.r0 + 1 <= kMaxRows) {
        const Neighbourhood nb = load_neighbourhood(off, p.Wk, k.r0, k.r1, k.c0, k.c1);
        for (int v0 = member; v0 < nb.total; v0 += kNb * team) {
            int x[kNb];
            bool valid[kNb];
#pragma unroll
            for (int t = 0; t < kNb; ++t) {
                valid[t] = v0 + t * team < nb.total;
                x[t] = flat_slot(nb, min(v0 + t * team, nb.total - 1));
            }
            batch(x, valid);
        }
    } else {
        for (int r = k.r0; r <= k.r1; ++r) {
            const int lo = off[r * p.Wk + k.c0], hi = off[r * p.Wk + k.c1 + 1];
            for (int x0 = lo + member; x0 < hi; x0 += kNb * team) {
                int x[kNb];
                bool valid[kNb];
#pragma unroll
                for (int t = 0; t < kNb; ++t) {
                    valid[t] = x0 + t * team < hi;
                    x[t] = min(x0 + t * team, hi - 1);
                }
                batch(x, valid);
            }
        }
    }
    if constexpr (RUNS) flush(false);
}

// Entries of key k's neighbourhood.
__device__ __forceinline__ int key_entries(const DiffParams& p, const KeyPos& k)
{
    const int32_t* off = p.offsets + static_cast<size_t>(k.s) * p.nkeys;
    int total = 0;
    for (int r = k.r0; r <= k.r1; ++r) total += off[r * p.Wk + k.c1 + 1] - off[r * p.Wk + k.c0];
    return total;
}

// dK_j (times scale) and dV_j from the lane's channels.
template <typename T, int D, int G>
__device__ __forceinline__ void diff_store_key(const DiffParams& p, uint32_t kg, int lane, const float* dk, const float* dv)
{
    constexpr int H = Row<T, D, G>::kEpc;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float4* ok = reinterpret_cast<float4*>(p.dK + static_cast<size_t>(kg) * D + (h * G + lane) * H);
        float4* ov = reinterpret_cast<float4*>(p.dV + static_cast<size_t>(kg) * D + (h * G + lane) * H);
#pragma unroll
        for (int i = 0; i < H / 4; ++i) {
            const float *a = dk + h * H + 4 * i, *b = dv + h * H + 4 * i;
            ok[i] = make_float4(a[0] * p.scale, a[1] * p.scale, a[2] * p.scale, a[3] * p.scale);
            ov[i] = make_float4(b[0], b[1], b[2], b[3]);
        }
    }
}

// A key with more entries than this goes to the list of the kernel below.
constexpr int kDiffHeavy = 64;

// A lane group per key.
template <typename T, int D, int G, bool MULTI>
__global__ __launch_bounds__(kBlock) void diff_key_kernel(DiffParams p)
{
    using RW = Row<T, D, G>;
    const int lane = threadIdx.x & (G - 1);
    uint32_t kg;
    if (!tile_item<RW::kQpb>(p.tk, xcd_remap(blockIdx.x, gridDim.x), threadIdx.x / G, kg)) return;
    const KeyPos k = key_pos(p, kg);
    const int total = key_entries(p, k);
    if (total > kDiffHeavy) {
        if (lane == 0) p.heavy[atomicAdd(p.n_heavy, 1)] = static_cast<int32_t>(kg);
        return;
    }
    uint4 kj[2], vj[2];
    load_row<T, D, G>(static_cast<const T*>(p.K), kg, lane, kj);
    load_row<T, D, G>(static_cast<const T*>(p.V), kg, lane, vj);
    float dk[2 * RW::kEpc], dv[2 * RW::kEpc];
#pragma unroll
    for (int i = 0; i < 2 * RW::kEpc; ++i) dk[i] = dv[i] = 0.f;
    diff_key_sums<T, D, G, MULTI, false>(p, k, total, 0, 1, lane, kj, vj, dk, dv);
    diff_store_key<T, D, G>(p, kg, lane, dk, dv);
}

// The keys of the list, a wave each: its lane groups take the entries in turn
// and their sums are added up.  And, as the last launch of a call, dlam.
template <typename T, int D, int G, bool MULTI>
__global__ __launch_bounds__(kBlock) void diff_heavy_kernel(DiffParams p)
{
    slice_sums(p);
    constexpr int N = 2 * Row<T, D, G>::kEpc;
    const int lane = threadIdx.x & (G - 1), member = (threadIdx.x & 63) / G;
    const int count = *p.n_heavy;
    for (int h = blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6); h < count; h += gridDim.x * (kBlock / 64)) {
        const uint32_t kg = static_cast<uint32_t>(p.heavy[h]);
        const KeyPos k = key_pos(p, kg);
        uint4 kj[2], vj[2];
        load_row<T, D, G>(static_cast<const T*>(p.K), kg, lane, kj);
        load_row<T, D, G>(static_cast<const T*>(p.V), kg, lane, vj);
        float dk[N], dv[N];
#pragma unroll
        for (int i = 0; i < N; ++i) dk[i] = dv[i] = 0.f;
        diff_key_sums<T, D, G, MULTI, true>(p, k, key_entries(p, k), member, 64 / G, lane, kj, vj, dk, dv);
#pragma unroll
        for (int mask = G; mask < 64; mask <<= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                dk[i] += __shfl_xor(dk[i], mask);
                dv[i] += __shfl_xor(dv[i], mask);
            }
        if (member == 0) diff_store_key<T, D, G>(p, kg, lane, dk, dv);
    }
}

// ---------------------------------------------------------------------------
// Key side on the matrix cores, fp32 storage: the strips of scram_strip.h and the fp32 products (16x16x4), a chunk of 16
// entries at a time (lane (m, g4)):
//   S1^T, S2^T = Q_E K_w^T of each half, dP^T = dO_E V_w^T    lane group g4 contracts the channels g4 D / 8 .. of each half;
//       lane: entries 4 g4 + i, key m
//   dV_w += (P1 - lam P2) dO_E, dK_w += dS Q_E                step i contracts the entries 4 g4 + i.  Column m of channel tile
//       o stands for a channel of half o / (tiles / 2): with 16 channels the one tile holds both, m < 8 and the others, and
//       takes dS1 and dS2 in turn
// A chunk's rows load while the previous chunk is in the matrix cores, the entry codes a chunk before that.  A strip of more
// entries than p.heavy_entries, or whose sums are not finite, leaves its keys to the list.
// 4 x 93 x 125, 32 channels, two 3 x 3 windows: 30-35 us, waiting on results in 43 % of the waves' cycles with 1.7 waves on a
// SIMD.
// ---------------------------------------------------------------------------
template <int D>
struct DiffStripLds {
    static constexpr int kRowF = D + 4;  // row stride, floats (padded)
    __attribute__((aligned(16))) float q[kStripFE * kRowF], g[kStripFE * kRowF];
    float4 meta[kStripFE];      // lse2 and D of both maps
    uint32_t in[kStripFE];      // bit k: the entry counts for key k of the strip, bit 16 + k: also its score's gradients
    int32_t lo[kStripMaxRows], pre[kStripMaxRows + 1];
};

// Products over N channels of a lane's row and key, sums of two in the matrix cores, added pairwise.
template <int N>
__device__ __forceinline__ f32x4_t diff_dots(const float* a, const float* b)
{
    if constexpr (N == 2) {
        f32x4_t t = {0.f, 0.f, 0.f, 0.f};
        t = __builtin_amdgcn_mfma_f32_16x16x4f32(a[0], b[0], t, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x4f32(a[1], b[1], t, 0, 0, 0);
    } else {
        return diff_dots<N / 2>(a, b) + diff_dots<N / 2>(a + N / 2, b + N / 2);
    }
}

template <int D, int MODE, int TEAM>
__global__ __launch_bounds__(64 * TEAM) __attribute__((amdgpu_waves_per_eu(D >= 64 ? 2 : 3))) void diff_key_strip_f32_kernel(DiffParams p)
{
    constexpr bool MULTI = MODE == kStripMulti;
    constexpr int kCh = D / 8;      // channels of a half per lane group
    constexpr int kOt = D / 16;     // channel tiles
    constexpr int kOc = kOt > 1 ? kOt / 2 : 1;  // tiles of a half: consecutive channels of a lane
    constexpr int kLR = D / 4, kRpi = 64 / kLR, kRep = kStripFE / kRpi;  // lanes per staged row, rows per load, loads
    using Lds = DiffStripLds<D>;
    constexpr int kRowF = Lds::kRowF;
    __shared__ Lds all[TEAM];
    const int lane = threadIdx.x & 63, wave = TEAM > 1 ? threadIdx.x >> 6 : 0, m = lane & 15, g4 = lane >> 4;
    Lds& lds = all[wave];
    constexpr int kStep = kStripFE * TEAM;
    // 128 channels: no rows in flight, so that two waves fit a SIMD (8 x 128 x 128, two 5 x 5 windows: strips 343 us, one wave
    // with them 411, keys on lane groups 697)
    constexpr bool kAhead = D < 128;
    const KeyStripF t(p.tk, xcd_remap(blockIdx.x, gridDim.x));
    if (t.sr0 >= p.Hk || t.sc0 >= p.Wk) return;  // the strip lies past the grid's edge
    int nrows;
    const int E = strip_entries(p, t, lds, lane, nrows);
    int kx, ky;  // this lane's key: key m of the strip
    t.key(m, kx, ky);
    const bool key_ok = kx < p.Hk && ky < p.Wk;
    const size_t kslice = static_cast<size_t>(t.s) * p.nkeys;
    const size_t krow = kslice + (key_ok ? static_cast<size_t>(kx) * p.Wk + ky : static_cast<size_t>(t.sr0) * p.Wk + t.sc0);
    auto leave_keys = [&]() {
        if (key_ok && g4 == 0 && wave == 0) p.heavy[atomicAdd(p.n_heavy, 1)] = static_cast<int32_t>(krow);
    };
    if (E > p.heavy_entries) {
        leave_keys();
        return;
    }
    float kf[2][kCh], vf[2][kCh];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        load_floats<kCh>(kf[h], static_cast<const float*>(p.K) + krow * D + h * (D / 2) + g4 * kCh);
        load_floats<kCh>(vf[h], static_cast<const float*>(p.V) + krow * D + h * (D / 2) + g4 * kCh);
    }
    const float lam = p.lam[t.s];
    const uint32_t live = static_cast<uint32_t>(__ballot(key_ok)) & 0xFFFFu;  // keys of the strip inside the grid
    const f32x4_t zero = f32x4_t{0.f, 0.f, 0.f, 0.f};
    f32x4_t dk[kOt], dv[kOt];
#pragma unroll
    for (int o = 0; o < kOt; ++o) dk[o] = dv[o] = zero;

    auto slot_code = [&](int c0) {  // lane group 0's lane m finds entry slot m of a chunk (the others repeat it)
        const int v = c0 + m;
        if (v >= E) return -1;
        int lo = 0, hi = nrows - 1;  // halo row holding flat position v: the last with pre <= v
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (lds.pre[mid] <= v) lo = mid; else hi = mid - 1;
        }
        return static_cast<int>(p.entries[lds.lo[lo] + (v - lds.pre[lo])]);
    };
    const int er = lane / kLR, ep = lane % kLR;
    f32x4_t rq[kRep], rg[kRep];  // this lane's pieces of the next chunk's rows
    int32_t match = -1, earlier = 0;  // the entry's match, and the query's first one
    float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
    uint32_t qe = 0u, qg = 0u;
    int code = -1;
    auto fetch = [&]() {  // the rows and statistics of the chunk whose codes are in `code`
        if (code >= 0) divmod(static_cast<uint32_t>(code), p.div_n, qe, qg);
        match = -1;
        if (code >= 0 && g4 == 0) {
            match = p.J[code];
            st = p.stats[qg];
            if constexpr (MULTI) earlier = p.J[qg];
        }
        const int my_q = code >= 0 ? static_cast<int>(qg) : -1;
#pragma unroll
        for (int j = 0; j < kRep; ++j) {
            // (past the entries a zero row keeps the operands finite)
            const int qj = __shfl(my_q, er + kRpi * j, 64);
            const size_t at = static_cast<size_t>(max(qj, 0)) * D + 4 * ep;
            rq[j] = rg[j] = zero;
            if (qj >= 0) {
                rq[j] = *reinterpret_cast<const f32x4_t*>(static_cast<const float*>(p.Q) + at);
                rg[j] = *reinterpret_cast<const f32x4_t*>(static_cast<const float*>(p.dO) + at);
            }
        }
    };
    code = slot_code(kStripFE * wave);
    if constexpr (kAhead) fetch();
    int next = slot_code(kStripFE * wave + kStep);
    for (int c0 = kStripFE * wave; c0 < E; c0 += kStep) {
        if constexpr (!kAhead) fetch();
#pragma unroll
        for (int j = 0; j < kRep; ++j) {
            *reinterpret_cast<f32x4_t*>(lds.q + (er + kRpi * j) * kRowF + 4 * ep) = rq[j];
            *reinterpret_cast<f32x4_t*>(lds.g + (er + kRpi * j) * kRowF + 4 * ep) = rg[j];
        }
        if (g4 == 0) {
            float4 meta = make_float4(0.f, 0.f, 0.f, 0.f);
            uint32_t in = 0u;  // the strip's keys that the entry counts for
            if (code >= 0) {
                uint32_t mu, mv;
                divmod(static_cast<uint32_t>(clamp_index(match, p.nkeys)), p.div_wk, mu, mv);
                const int ru = static_cast<int>(mu) - t.sr0, cv = static_cast<int>(mv) - t.sc0;
                in = t.bits(ru - p.b, ru + p.b, cv - p.b, cv + p.b) & live;
                if (MODE != kStripPlain && p.causal) {
                    uint32_t sl, rem, lr, lc;
                    divmod(qg, p.div_plane, sl, rem);
                    divmod(causal_limit(p, sl, rem), p.div_wk, lr, lc);
                    const int last = static_cast<int>(lr) - t.sr0;
                    in &= t.bits(0, last - 1, 0, 15) | t.bits(last, last, 0, static_cast<int>(lc) - t.sc0);
                }
                if constexpr (MULTI) {
                    // less those that the query's windows 0 .. e - 1 hold
                    for (int f = 0; f < static_cast<int>(qe); ++f) {
                        uint32_t fu, fv;
                        const int32_t at = f == 0 ? earlier : p.J[static_cast<size_t>(f) * p.n + qg];
                        divmod(static_cast<uint32_t>(clamp_index(at, p.nkeys)), p.div_wk, fu, fv);
                        const int hu = static_cast<int>(fu) - t.sr0, hv = static_cast<int>(fv) - t.sc0;
                        in &= ~t.bits(hu - p.b, hu + p.b, hv - p.b, hv + p.b);
                    }
                }
                meta = st;
                // (a set of one key: its weights count, its score's gradients do not)
                if (MODE == kStripPlain || !is_one_key(st)) in |= in << 16;
            }
            lds.in[m] = in;
            lds.meta[m] = meta;
        }
        code = next;
        if constexpr (kAhead)
            if (c0 + kStep < E) fetch();
        next = slot_code(c0 + 2 * kStep);
        wave_lds_sync();

        const float *const qa = lds.q + m * kRowF + g4 * kCh, *const ga = lds.g + m * kRowF + g4 * kCh;
        float a[kCh];
        f32x4_t sc[2], dp = zero;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            load_floats<kCh>(a, qa + h * (D / 2));
            sc[h] = diff_dots<kCh>(a, kf[h]);
            load_floats<kCh>(a, ga + h * (D / 2));
            dp += diff_dots<kCh>(a, vf[h]);
        }
        float w[4], ds[2][4];  // of (key m, entry 4 g4 + i)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int te = 4 * g4 + i;
            const float4 mt = lds.meta[te];
            const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[0][i], p.scale_log2e, -mt.x));
            const float p2 = lam * __builtin_amdgcn_exp2f(fmaf(sc[1][i], p.scale_log2e, -mt.z));
            // (selected by bits: a key that is left out may hold anything)
            const int sets = static_cast<int>(lds.in[te]);
            auto kept = [](float x, int in) { return __uint_as_float(__float_as_uint(x) & static_cast<uint32_t>(in)); };
            const int in = __builtin_amdgcn_sbfe(sets, m, 1), in_ds = MODE == kStripPlain ? in : __builtin_amdgcn_sbfe(sets, m + 16, 1);
            w[i] = kept(p1 - p2, in);
            ds[0][i] = kept(p1 * (dp[i] - mt.y), in_ds);
            ds[1][i] = kept(p2 * (mt.w - dp[i]), in_ds);
        }
        // the chunk's sums first, then onto the strip's (sums of sums round less than one long sum)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x4_t ck[kOc], cv[kOc];
#pragma unroll
            for (int o = 0; o < kOc; ++o) ck[o] = cv[o] = zero;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float bq[kOc], bg[kOc];
                if constexpr (kOt > 1) {
                    load_floats<kOc>(bq, lds.q + (4 * g4 + i) * kRowF + h * (D / 2) + m * kOc);
                    load_floats<kOc>(bg, lds.g + (4 * g4 + i) * kRowF + h * (D / 2) + m * kOc);
                } else {  // the tile's columns of this half
                    const bool mine = (m < 8) == (h == 0);
                    bq[0] = mine ? lds.q[(4 * g4 + i) * kRowF + m] : 0.f;
                    bg[0] = mine ? lds.g[(4 * g4 + i) * kRowF + m] : 0.f;
                }
#pragma unroll
                for (int o = 0; o < kOc; ++o) {
                    cv[o] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[i], bg[o], cv[o], 0, 0, 0);
                    ck[o] = __builtin_amdgcn_mfma_f32_16x16x4f32(ds[h][i], bq[o], ck[o], 0, 0, 0);
                }
            }
#pragma unroll
            for (int o = 0; o < kOc; ++o) {
                dk[kOt > 1 ? h * kOc + o : 0] += ck[o];
                dv[kOt > 1 ? h * kOc + o : 0] += cv[o];
            }
        }
        wave_lds_sync();  // this chunk's LDS reads come before the next chunk's writes
    }
    if constexpr (TEAM > 1) {  // the other waves' sums, from their staging areas
        static_assert(sizeof(f32x4_t) * 128 * kOt <= sizeof(float) * 2 * kStripFE * kRowF, "16 keys' gradient rows fit 16 entries' rows");
        f32x4_t* const mine = reinterpret_cast<f32x4_t*>(&lds) + lane;
        if (wave > 0) {
#pragma unroll
            for (int o = 0; o < kOt; ++o) mine[128 * o] = dk[o], mine[128 * o + 64] = dv[o];
        }
        __syncthreads();
        if (wave > 0) return;
        for (int w = 1; w < TEAM; ++w) {
            const f32x4_t* const other = reinterpret_cast<const f32x4_t*>(&all[w]) + lane;
#pragma unroll
            for (int o = 0; o < kOt; ++o) dk[o] += other[128 * o], dv[o] += other[128 * o + 64];
        }
    }
    float sum = 0.f;
#pragma unroll
    for (int o = 0; o < kOt; ++o)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += fabsf(dk[o][r]) + fabsf(dv[o][r]);
    if (__any(!(sum < INFINITY))) {
        leave_keys();
        return;
    }
    // lane holds keys 4 g4 + r of the strip, channels h D / 2 + m kOc + o of tile h kOc + o
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        int ox, oy;
        t.key(4 * g4 + r, ox, oy);
        if (ox >= p.Hk || oy >= p.Wk) continue;
        const size_t row = (kslice + static_cast<size_t>(ox) * p.Wk + oy) * D;
#pragma unroll
        for (int h = 0; h < (kOt > 1 ? 2 : 1); ++h) {
            float ok[kOc], ov[kOc];
#pragma unroll
            for (int o = 0; o < kOc; ++o) ok[o] = dk[h * kOc + o][r] * p.scale, ov[o] = dv[h * kOc + o][r];
            store_floats<kOc>(p.dK + row + h * (D / 2) + m * kOc, ok);
            store_floats<kOc>(p.dV + row + h * (D / 2) + m * kOc, ov);
        }
    }
}

// Up to as many strips a team of four waves takes each, up to four times as many a team of two: a wave per strip would not
// fill the machine, and the strips of many entries would run on alone.  (fp32, 64 channels, some 3,000 strips: 3 x 3 117 us a call
// with one wave, 107 with two, 115 with four, 5 x 5 177, 161, 166; bf16, 288 strips: 68, 59, 56; 8192 strips: 252, 268 with four.)
constexpr uint64_t kTeamStrips = 1024;

size_t r256(size_t b) { return (b + 255) & ~static_cast<size_t>(255); }

// Parts of dlam: a block of lane groups (of one lane at least per query), or a wave of 16 queries, each.
uint64_t query_blocks_most(const Grid& g)
{
    uint64_t most = 4 * tiling_blocks(make_tiling(g.Hq, g.Wq, kBlock / 4), g.S);
    for (uint32_t items = kBlock; items >= kBlock / 16; items /= 2)
        most = std::max(most, tiling_blocks(make_tiling(g.Hq, g.Wq, items, kLaneSkew), g.S));
    return most;
}

template <int D, int W>
hipError_t run_diff_query_tile(const DiffParams& p, uint64_t waves, hipStream_t st)
{
    auto with = [&](auto mk) {
        constexpr int MK = decltype(mk)::value;
        return p.causal ? launch_wave(diff_query_tile_kernel<D, W, true, MK>, waves, st, nullptr, nullptr, p)
                        : launch_wave(diff_query_tile_kernel<D, W, false, MK>, waves, st, nullptr, nullptr, p);
    };
    return p.kappa == 1   ? with(std::integral_constant<int, 1>{})
           : p.kappa == 2 ? with(std::integral_constant<int, 2>{})
                          : with(std::integral_constant<int, 4>{});
}

// The query side on the matrix cores, if it takes this call (false: not launched).
template <typename T, int D>
bool run_diff_query_tiles(const DiffParams& p0, hipStream_t st, hipError_t& err)
{
    if constexpr (std::is_same<T, uint16_t>::value && D >= 32) {
        DiffParams p = p0;
        const uint64_t tiles = diff_tiles<D>(p);
        // (a grid of one key: every set is one key, which the tiles expect of the causal mask alone)
        if (tiles == 0 || p.nkeys == 1) return false;
        err = p.b == 1   ? run_diff_query_tile<D, 3>(p, 4 * tiles, st)
              : p.b == 2 ? run_diff_query_tile<D, 5>(p, 4 * tiles, st)
              : p.b == 3 ? run_diff_query_tile<D, 7>(p, 4 * tiles, st)
                         : run_diff_query_tile<D, 9>(p, 4 * tiles, st);
        return true;
    }
    return false;
}

template <typename T, int D, bool MULTI>
hipError_t run_diff_backward(const DiffParams& p0, int32_t* counts, int32_t* offsets, int32_t* sums, int32_t* entries,
                             hipStream_t st, hipEvent_t start, hipEvent_t stop)
{
    constexpr int G = kDiffLanes<T, D>;
    constexpr uint32_t kQpb = Row<T, D, G>::kQpb;
    DiffParams p = p0;
    p.tq = make_tiling(p.Hq, p.Wq, kQpb, kLaneSkew);
    p.tk = make_tiling(p.Hk, p.Wk, kQpb, kLaneSkew);
    const uint32_t S = p.n / p.tq.plane;
    const uint64_t qblocks = tiling_blocks(p.tq, S), kblocks = tiling_blocks(p.tk, S);
    const size_t N = p.keys_total;
    hipError_t e;
    if ((e = launch(zero_i32_kernel, stride_blocks(N), st, start, nullptr, counts, N, p.n_heavy)) != hipSuccess) return e;
    p.slices = S;
    p.parts = p.tq.div_slice.d;
    if (run_diff_query_tiles<T, D>(p, st, e)) {
        p.parts = 4 * make_tiling(p.Hq, p.Wq, kBlock / 4).div_slice.d;
    } else if constexpr (!MULTI)
        e = launch(diff_query_kernel<T, D, G, 0>, qblocks, st, nullptr, nullptr, p);
    else
        e = p.kappa <= 2   ? launch(diff_query_kernel<T, D, G, 2>, qblocks, st, nullptr, nullptr, p)
            : p.kappa <= 4 ? launch(diff_query_kernel<T, D, G, 4>, qblocks, st, nullptr, nullptr, p)
                           : launch(diff_query_kernel<T, D, G, kMaxKappa>, qblocks, st, nullptr, nullptr, p);
    if (e != hipSuccess) return e;
    if ((e = run_inverse(p, counts, offsets, sums, entries, st, nullptr, nullptr)) != hipSuccess) return e;
    // Key side on the matrix cores for windows 3 x 3 .. 15 x 15, and of one key where bf16 has several maps; the keys that its
    // strips leave, and those of every other call with many entries, a wave each.
    // (Windows of one key, several maps: 4 x 256 x 256, 64 channels, bf16 two maps 81 us, on lane groups 120; fp32 four maps 278,
    // on lane groups 253.)
    const int least = std::is_same<T, uint16_t>::value && p.kappa > 1 ? 0 : 1;
    if (p.b >= least && p.b <= kTileMaxB && p.nkeys > 1) {
        DiffParams pt = p;
        pt.tk = make_tiling(p.Hk, p.Wk, kTileKeys);
        const uint64_t halo = static_cast<uint64_t>(std::min(4 + 2 * p.b, p.Hk)) * std::min(4 + 2 * p.b, p.Wk);
        const uint64_t mean = static_cast<uint64_t>(p.n) * p.kappa * halo / p.keys_total;  // entries of a strip
        // (a strip of thousands of entries would run on alone; lower and higher limits were slower)
        pt.heavy_entries = static_cast<int>(std::min<uint64_t>(std::max<uint64_t>(1024, 4 * mean), INT32_MAX));
        const uint64_t strips = kStripWaves * tiling_blocks(pt.tk, S);
        auto with = [&](auto mode, auto team) {
            constexpr int MODE = decltype(mode)::value, TEAM = decltype(team)::value;
            if constexpr (std::is_same<T, float>::value)
                return launch_wave<64 * TEAM>(diff_key_strip_f32_kernel<D, MODE, TEAM>, strips, st, nullptr, nullptr, pt);
            else
                return launch_wave<64 * TEAM>(bwd_key_strip_kernel<D, MODE, DiffParams, TEAM>, strips, st, nullptr, nullptr, pt);
        };
        auto go = [&](auto mode) {
            return strips <= kTeamStrips ? with(mode, std::integral_constant<int, 4>{})
                   : strips <= 4 * kTeamStrips ? with(mode, std::integral_constant<int, 2>{})
                                               : with(mode, std::integral_constant<int, 1>{});
        };
        e = !MULTI         ? go(std::integral_constant<int, kStripPlain>{})
            : p.kappa == 1 ? go(std::integral_constant<int, kStripCausal>{})
                           : go(std::integral_constant<int, kStripMulti>{});
        if (e != hipSuccess) return e;
        return launch(diff_heavy_kernel<T, D, G, MULTI>, 1024, st, nullptr, stop, p);
    }
    if ((e = launch(diff_key_kernel<T, D, G, MULTI>, kblocks, st, nullptr, nullptr, p)) != hipSuccess) return e;
    return launch(diff_heavy_kernel<T, D, G, MULTI>, 1024, st, nullptr, stop, p);  // loops over however many there are
}

}  // namespace

size_t diff_backward_workspace_bytes(const Grid& g, int kappa)
{
    const size_t n = static_cast<size_t>(g.S) * g.Hq * g.Wq, N = static_cast<size_t>(g.S) * g.Hk * g.Wk;
    const size_t tiles = (N + kScanTile - 1) / kScanTile;
    return r256(4 * N) + r256(4 * (N + 1)) + r256(4 * (tiles + 1)) + 2 * r256(4 * n * kappa) + r256(16 * n) +
           r256(4 * (N + 1)) + r256(8 * query_blocks_most(g));
}

hipError_t launch_diff_backward(int dtype, const DiffCall& c, const void* dO, float* dQ, float* dK, float* dV, float* dlam,
                                void* workspace, hipStream_t stream, hipEvent_t start, hipEvent_t stop)
{
    DiffParams p{};
    fill_diff_params(p, c);
    p.dO = dO;
    p.dQ = dQ;
    p.dK = dK;
    p.dV = dV;
    p.dlam = dlam;
    // workspace: counts, offsets, tile sums, entries, slots, statistics, heavy keys, parts of dlam
    const size_t N = p.keys_total, total = static_cast<size_t>(p.n) * c.kappa;
    char* w = static_cast<char*>(workspace);
    auto take = [&](size_t bytes) {
        char* at = w;
        w += r256(bytes);
        return at;
    };
    int32_t* counts = reinterpret_cast<int32_t*>(take(4 * N));
    int32_t* offsets = reinterpret_cast<int32_t*>(take(4 * (N + 1)));
    int32_t* sums = reinterpret_cast<int32_t*>(take(4 * ((N + kScanTile - 1) / kScanTile + 1)));
    int32_t* entries = reinterpret_cast<int32_t*>(take(4 * total));
    p.slots = reinterpret_cast<int32_t*>(take(4 * total));
    p.stats = reinterpret_cast<float4*>(take(16 * static_cast<size_t>(p.n)));
    p.n_heavy = reinterpret_cast<int32_t*>(take(4 * (N + 1)));  // counter, then the list
    p.heavy = p.n_heavy + 1;
    p.lam_part = reinterpret_cast<double*>(w);
    p.counts = counts;
    p.offsets = offsets;
    p.entries = entries;
    return dispatch(dtype, c.g.d, [&](auto ty, auto d) {
        using T = decltype(ty);
        constexpr int D = decltype(d)::value;
        return p.kappa == 1 && !p.causal ? run_diff_backward<T, D, false>(p, counts, offsets, sums, entries, stream, start, stop)
                                         : run_diff_backward<T, D, true>(p, counts, offsets, sums, entries, stream, start, stop);
    });
}

uint64_t diff_backward_max_blocks(const Grid& g)
{
    uint64_t most = std::max<uint64_t>(4096, query_blocks_most(g));  // (4096: the grid-stride kernels of the inverse map)
    most = std::max(most, tiling_blocks(make_tiling(g.Hk, g.Wk, kTileKeys), g.S));  // key tiles on the matrix cores
    for (uint32_t items = kBlock; items >= kBlock / 16; items /= 2)
        most = std::max(most, tiling_blocks(make_tiling(g.Hk, g.Wk, items, kLaneSkew), g.S));
    return most;
}

}  // namespace scram
