// Differential attention over the match windows: forward.

#include "scram_diff_tile.h"

namespace scram {
namespace {

// Query g on a lane group, or on TEAM lane groups that share its keys and add up at the end (all lanes of the team call).
// One walk over the key set keeps two online softmaxes (base-2 domain) and their sums of values.  A key that is left out is
// not accumulated at all: whatever its rows hold stays out.
// MK = 0: one window, no mask; else up to MK windows and/or the causal mask.
template <typename T, int D, int G, int MK, int kNb, int TEAM>
__device__ __forceinline__ void diff_query(const DiffParams& p, uint32_t g, int lane, int member)
{
    constexpr bool MULTI = MK > 0;
    using RW = Row<T, D, G>;
    static_assert(RW::kCh == 2, "two chunks per lane: one of each half");
    constexpr int E = 2 * RW::kEpc;
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
        walk_window<T, D, G, kNb, MK>(p, Ks, Vs, ws, e, u, v, member, TEAM, lane, [&](const auto& ok, const auto& kr, const auto& vr) {
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
    if constexpr (TEAM > 1) {
#pragma unroll
        for (int mask = G; mask < TEAM * G; mask <<= 1) {
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

// A lane group per query, or WAVE: a wave per query, for calls of up to 4096 queries, of which lane groups or tiles would leave
// most of the machine without work.  (Kernel alone, lane groups or tiles and WAVE, bf16, 64 channels, two 5 x 5 windows: 512
// queries 15 and 7 us, 4096 18 and 14, 8192 23 and 23; two 7 x 7 20 and 15 at 4096, 28 and 25 at 8192; fp32, 64 channels, one
// 5 x 5 7 and 7 at 4096, two 7 x 7 30 and 14.  One 3 x 3 window is even at 1024 and loses at 4096, 7 and 11.)
// fp32 8 x 128 x 128 -> 192 x 192, 32 channels, two 3 x 3 windows: 36-37 us, its bytes 21 us at a copy's rate.  kNb keys at a time: three, or five for one
// 5 x 5 window, which is then five whole batches (8 x 128 x 128, 32 channels, fp32: two 3 x 3 windows with four 44 us, three
// 38, five 40; one 5 x 5 window 38, 40, 32).
template <typename T, int D, int G, int MK, int kNb, bool WAVE>
__global__ __launch_bounds__(WAVE ? 64 : kBlock) void diff_attend_kernel(DiffParams p)
{
    const int lane = threadIdx.x & (G - 1);
    if constexpr (WAVE) {
        diff_query<T, D, G, MK, kNb, 64 / G>(p, blockIdx.x, lane, threadIdx.x / G);
    } else {
        uint32_t g;
        if (tile_item<Row<T, D, G>::kQpb>(p.tq, xcd_remap(blockIdx.x, gridDim.x), threadIdx.x / G, g))
            diff_query<T, D, G, MK, kNb, 1>(p, g, lane, 0);
    }
}

// Waves per SIMD that the tile kernel's registers are sized for.
constexpr int diff_tile_waves(int D, int MK) { return D == 128 ? 2 : MK == 4 ? 3 : 4; }

// On the matrix cores (scram_diff_tile.h), bf16.  Per block of 16 keys
//   S1^T, S2^T = K_blk Q^T       keys x queries, of each half of the channels
//   P1, P2 = 2^(S scale log2 e - reference) on the query's keys, 0 elsewhere
//   O1^T += V_blk^T P1^T, O2^T += V_blk^T P2^T
// with the weights as three bf16 parts that add up to them, and at the end o = O1 / l1 - lam O2 / l2.  (What a weight loses is
// lost against O1 and O2, not against the difference: where the two maps are alike, two parts, 18 bits, show in the output.)  A
// query whose sums are
// not finite (an infinite value of the box reaches every query of its cluster through 0 * inf, a score that is not a number
// passes its mask), or whose set is empty, is computed over again on a lane group, and so are a wave's queries whose matches
// lie too far apart to share rows.
// 4 x 256 x 256, 64 channels, two 5 x 5 windows: 137-144 us (a lane group per query 175; its bytes 26 us at a copy's rate), the
// vector units and the loads' return path bound it, at 4 waves per SIMD.  The normalisers are added up by the vector units (on
// the matrix cores, as a product with ones, 141 us for 137, and spills with the causal mask).
template <int D, int W, bool CAUSAL, int MK>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(diff_tile_waves(D, MK)))) void
diff_tile_kernel(DiffParams p)
{
    using TR = TileRow<D>;
    constexpr int kOt = D / 16, kRowB = 2 * D + kRowPad;
    constexpr int G = kDiffLanes<uint16_t, D>;
    __shared__ __align__(16) unsigned char tk[16 * kRowB], tv[16 * kRowB];
    const int lane = threadIdx.x, m = lane & 15, g4 = lane >> 4;
    // a wave is a block of its own: their work is uneven, and one that is done makes room at once
    const uint32_t one = xcd_remap(blockIdx.x, gridDim.x), blk = one / 4;
    const int wave = static_cast<int>(one % 4);
    const DiffTile<MK> t = diff_tile<W, MK>(p, blk, wave, lane, p.tile_blocks);
    if (t.tc.nclu == 0) return;  // no query of this wave lies inside the grid
    uint32_t todo = 0xFFFFu;     // queries left to the lane groups
    if (t.tc.nclu > 0) {
        // every item of a tile lies in one slice, whose rows the caller keeps below 4 GiB: 32-bit offsets from a uniform base
        const size_t slice = static_cast<size_t>(__builtin_amdgcn_readfirstlane(t.s)) * p.nkeys * static_cast<size_t>(2 * D);
        const unsigned char* const Kb = static_cast<const unsigned char*>(p.K) + slice;
        const unsigned char* const Vb = static_cast<const unsigned char*>(p.V) + slice;
        HalfQueries<D> q;
        q.load(static_cast<const unsigned char*>(p.Q) + static_cast<size_t>(t.gq) * (2 * D), g4);
        MapReference ref[2];
        {
            float s0[2];
            q.own_scores(Kb + t.centre * (2u * D), g4, s0);
            const bool held = !CAUSAL || t.centre <= t.limit;
            ref[0].start(s0[0], held, p.scale_log2e);
            ref[1].start(s0[1], held, p.scale_log2e);
        }
        f32x4_t acc[2][kOt];
        float sum[2] = {0.f, 0.f};  // of the weights of this lane's keys
#pragma unroll
        for (int o = 0; o < kOt; ++o) acc[0][o] = acc[1][o] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        diff_walk<D, W, CAUSAL, MK>(p, t, Kb, Vb, tk, tv, lane, [&](f32x4_t bias) {
            f32x4_t sc[2];
            q.scores([&](int ds) { return TR::frag(tk + m * kRowB, ds, g4); }, bias, sc);
            float x[2][4];
            block_weights(ref, sc, p.scale_log2e, x, [&](int h, float f) {
                sum[h] *= f;
#pragma unroll
                for (int o = 0; o < kOt; ++o) acc[h][o] *= f;
            });
#pragma unroll
            for (int h = 0; h < 2; ++h) sum[h] += (x[h][0] + x[h][1]) + (x[h][2] + x[h][3]);
            const Parts3 w0 = parts3(x[0]), w1 = parts3(x[1]);
#pragma unroll
            for (int o = 0; o < kOt; ++o) {
                const bf16x4_t vt = column4<D>(tv, m, g4, o);
                acc[0][o] = product3(vt, w0, acc[0][o]);
                acc[1][o] = product3(vt, w1, acc[1][o]);
            }
        });
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            sum[h] += __shfl_xor(sum[h], 16);
            sum[h] += __shfl_xor(sum[h], 32);
        }
        const float i1 = 1.f / sum[0], i2 = p.lam[t.s] / sum[1];  // an empty set's are infinite
        float size = i1 + i2;
#pragma unroll
        for (int o = 0; o < kOt; ++o) {
            acc[0][o] = acc[0][o] * i1 - acc[1][o] * i2;
            size += (fabsf(acc[0][o][0]) + fabsf(acc[0][o][1])) + (fabsf(acc[0][o][2]) + fabsf(acc[0][o][3]));
        }
        const uint64_t bad = __ballot(!(fabsf(size) < INFINITY));
        todo = static_cast<uint32_t>(bad | bad >> 16 | bad >> 32 | bad >> 48) & 0xFFFFu;
        if (t.valid && !((todo >> m) & 1u)) {
            // lane holds channels 16 o + 4 g4 + i of query m
            uint16_t* const row = static_cast<uint16_t*>(p.out) + static_cast<size_t>(t.g) * D + 4 * g4;
#pragma unroll
            for (int o = 0; o < kOt; ++o)
                *reinterpret_cast<uint2*>(row + 16 * o) = make_uint2(bf16_pair(acc[0][o][0], acc[0][o][1]), bf16_pair(acc[0][o][2], acc[0][o][3]));
        }
    }
    for (int i = lane / G; i < 16; i += 64 / G) {
        uint32_t g;
        if (((todo >> i) & 1u) && tile_item<kBlock / 4>(p.tq, blk, tile_wave_item(p.tq, wave, i), g))
            diff_query<uint16_t, D, G, (CAUSAL || MK > 1 ? MK : 0), 2, 1>(p, g, lane & (G - 1), 0);
    }
}

template <int D, int W>
hipError_t run_diff_tile(const DiffParams& p, uint64_t tiles, hipStream_t st, hipEvent_t e0, hipEvent_t e1)
{
    auto with = [&](auto mk) {
        constexpr int MK = decltype(mk)::value;
        return p.causal ? launch_wave(diff_tile_kernel<D, W, true, MK>, 4 * tiles, st, e0, e1, p)
                        : launch_wave(diff_tile_kernel<D, W, false, MK>, 4 * tiles, st, e0, e1, p);
    };
    return p.kappa == 1   ? with(std::integral_constant<int, 1>{})
           : p.kappa == 2 ? with(std::integral_constant<int, 2>{})
                          : with(std::integral_constant<int, 4>{});
}

// On the matrix cores, if they take this call (false: not launched).
template <typename T, int D>
bool run_diff_tiles(const DiffParams& p0, hipStream_t st, hipEvent_t e0, hipEvent_t e1, hipError_t& err)
{
    if constexpr (std::is_same<T, uint16_t>::value && D >= 32) {
        DiffParams p = p0;
        const uint64_t tiles = diff_tiles<D>(p);
        if (tiles == 0) return false;
        err = p.b == 1   ? run_diff_tile<D, 3>(p, tiles, st, e0, e1)
              : p.b == 2 ? run_diff_tile<D, 5>(p, tiles, st, e0, e1)
              : p.b == 3 ? run_diff_tile<D, 7>(p, tiles, st, e0, e1)
                         : run_diff_tile<D, 9>(p, tiles, st, e0, e1);
        return true;
    }
    return false;
}

template <typename T, int D, int MK>
hipError_t run_diff(const DiffParams& p0, hipStream_t st, hipEvent_t e0, hipEvent_t e1)
{
    constexpr int G = kDiffLanes<T, D>;
    DiffParams p = p0;
    if (p.n <= 4096) return launch_wave(diff_attend_kernel<T, D, G, MK, 4, true>, p.n, st, e0, e1, p);
    hipError_t err = hipSuccess;
    if (run_diff_tiles<T, D>(p, st, e0, e1, err)) return err;
    p.tq = make_tiling(p.Hq, p.Wq, Row<T, D, G>::kQpb, kLaneSkew);
    const uint64_t blocks = tiling_blocks(p.tq, p.n / p.tq.plane);
    if constexpr (MK == 0)
        if (p.b == 2) return launch(diff_attend_kernel<T, D, G, MK, 5, false>, blocks, st, e0, e1, p);
    return launch(diff_attend_kernel<T, D, G, MK, 3, false>, blocks, st, e0, e1, p);
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
        // (centres of the windows in registers: 4 x 256 x 256 fp32, 64 channels, four 3 x 3 windows, sized for four 223 us, for
        // eight 257)
        return p.kappa <= 2   ? run_diff<T, D, 2>(p, stream, start, stop)
               : p.kappa <= 4 ? run_diff<T, D, 4>(p, stream, start, stop)
                              : run_diff<T, D, kMaxKappa>(p, stream, start, stop);
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
