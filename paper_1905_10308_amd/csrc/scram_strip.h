// Key side of the gradients on the matrix cores: the strips of the attend's
// (scram_backward.hip) and the differential attend's (scram_diff_backward.hip),
// and their kernel for bf16 storage.
//
// Everything here lives in an unnamed namespace, like scram_device.h.

#pragma once

#include "scram_diff.h"
#include "scram_inverse.h"
#include "scram_tile.h"

namespace scram {
namespace {

// ---------------------------------------------------------------------------
// Key side on the matrix cores (bf16 storage).  Each wave takes a strip of 16
// keys of a 64-key tile (a 4 x 4 quarter of an 8 x 8 tile; items 16 w .. 16 w
// + 15 in raster order of flatter or taller tiles) and works alone, a block
// of its own: the number of entries
// per strip is very uneven, and a wave that finishes releases its LDS at once
// instead of holding it until the slowest strip of a shared block is done.  The
// queries whose key sets reach the strip are exactly the entries whose match
// lies in the strip's halo (the strip widened by b), one contiguous entry
// range per halo row.  Per chunk of 32 of those entries, staged in the wave's
// own LDS (q and dO rows, match, log2 normaliser, D), on the matrix cores
//   S^T = Q_E K_w^T,  dP^T = dO_E V_w^T                 (entries x keys),
// in registers P = window test ? 2^(S scale log2 e - lse2) : 0 and
// dS = P (dP - D), and again on the matrix cores
//   dV_w += P dO_E,   dK_w += dS Q_E                    (keys x channels).
// The output layout of the first products (lane l: key l mod 16 and four
// entries) is the operand layout of the second, so P and dS never leave
// registers (the entries' order along the contraction only has to agree
// between the two operands).  The channel-major operands dO_E, Q_E of the
// second products come from the staged rows through the transposing LDS load.
// P and dS enter as three bf16 parts that add up to the fp32 values exactly
// (products of bf16 parts are exact); all sums are fp32.
// ---------------------------------------------------------------------------
constexpr int kTileKeys = 64;                          // keys per block, 16 per wave
constexpr int kTileMaxB = 7;                           // windows up to 15 x 15
constexpr int kStripMaxRows = 16 + 2 * kTileMaxB;      // halo rows of the tallest strip (16 x 1)
constexpr int kStripCE = 32;                           // entries per chunk: one contraction step

template <int D>
struct KeyStrip {
    static constexpr int kRowB = 2 * D + 16;           // row stride in LDS, bytes (padded)
    static constexpr int kDs = D >= 32 ? D / 32 : 1;   // 32-channel steps of the first products
    static constexpr int kOt = D / 16;                 // 16-channel tiles of dK_w, dV_w
    static constexpr int kPieces = D / 8;              // 16-byte pieces per row
};

// The strip kernel's key-set tests: the window only, the window and the causal mask (one map), or
// several windows (and the causal mask if asked for).
enum StripMode { kStripPlain = 0, kStripCausal = 1, kStripMulti = 2 };

// waves per SIMD the strip kernel's registers are sized for (64 channels of the differential attend: four spill, 16 x 128 x
// 128, two 5 x 5 maps, 407 us against 369 in all)
constexpr int strip_waves(int D, bool diff) { return D > 64 ? 2 : diff && D == 64 ? 3 : 4; }

// x = hi + mid + lo exactly, each part a bf16 value held as an fp32 bit
// pattern with a zero low half: hi keeps the top 8 significant bits of x
// (truncation), x - hi is exact in fp32 and mid keeps its top 8, and the
// remaining lo has at most 8 significant bits (x has 24).
__device__ __forceinline__ void split3(float x, uint32_t& hi, uint32_t& mid, uint32_t& lo)
{
    hi = __float_as_uint(x) & 0xFFFF0000u;
    const float r1 = x - __uint_as_float(hi);
    mid = __float_as_uint(r1) & 0xFFFF0000u;
    lo = __float_as_uint(r1 - __uint_as_float(mid));
}

__device__ __forceinline__ bf16x8_t lds_frag(const unsigned char* p)
{
    return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(p));
}

constexpr int kStripWaves = kTileKeys / 16;  // strips of a tile, one one-wave block each

// Differential attend (P = DiffParams): S^T of each half of the channels (a fragment that holds both halves enters twice, the
// other half of the keys zeroed), P = P1 - lam P2 for dV, and dS1, dS2 = - lam P2 (dP - D2) for the halves of dK.  Strips whose
// sums are not finite (a row that is not reaches all of the strip's keys through 0 * inf) and those of more entries than
// p.heavy_entries leave their keys to the list of diff_heavy_kernel.
// For which of the strip's keys an entry counts is worked out once, by the lane that stages it, as 16 bits (16 x 128 x 128, 64
// channels, two 5 x 5 windows: all of a call 319 us, with a test per key and entry 347; the strips 115-134 of it, vector units
// issuing in 52 % of the cycles, waves waiting for 34 % of theirs).
// TEAM waves share a strip, taking its chunks in turn, and their sums are added up through LDS.
template <int D, int MODE, typename P, int TEAM = 1>
__global__ __launch_bounds__(64 * TEAM) __attribute__((amdgpu_waves_per_eu(strip_waves(D, std::is_same<P, DiffParams>::value)))) void
bwd_key_strip_kernel(P p)
{
    constexpr bool DIFF = std::is_same<P, DiffParams>::value;
    constexpr bool MULTI = MODE == kStripMulti;
    constexpr bool kQueryIndex = MODE != kStripPlain;  // entries carry their window and query's raster index
    using KS = KeyStrip<D>;
    constexpr int kCE = kStripCE;
    constexpr int kW = TEAM;  // waves per block
    // q rows of the chunk, then 64 bytes of skew, then its dO rows: lanes 2t and 2t + 1 stage row t of
    // each; with the skew the eight lanes of one 128-bit access (rows t .. t + 3 of both) use disjoint
    // halves of the 32 banks, without it the two rows of each pair share banks
    __shared__ __align__(16) unsigned char s_row[kW][2 * kCE * KS::kRowB + 64];
    __shared__ int4 s_meta[kW][kCE];        // match row, match column, lse2 bits, D bits
    // several windows: the strip's keys that one of the entry query's earlier windows holds (bit k: key
    // k); causal: the query's raster index
    __shared__ int32_t s_el[kW][kQueryIndex ? kCE : 1][2];
    __shared__ int32_t s_lo[kW][kStripMaxRows], s_pre[kW][kStripMaxRows + 1];
    __shared__ float2 s_second[kW][DIFF ? kCE : 1];  // lse2, D of the second map

    const int lane = threadIdx.x & 63, wave = TEAM > 1 ? threadIdx.x >> 6 : 0;
    const int m = lane & 15, g4 = lane >> 4;
    const uint32_t blk = xcd_remap(blockIdx.x, gridDim.x);

    // the tile (th x tw keys at x0, y0 of slice s) and this wave's strip in it
    uint32_t s, k, tr, tc;
    divmod(blk / kStripWaves, p.tk.div_slice, s, k);
    tile_coords(p.tk, k, tr, tc);
    const int tw = 1 << p.tk.lw, th = kTileKeys >> p.tk.lw;
    const int x0 = static_cast<int>(tr) * th, y0 = static_cast<int>(tc) * tw;
    const int w4 = static_cast<int>(blk % kStripWaves);
    // the strip: a 4 x 4 quarter of an 8 x 8 tile (its halo holds 11 % fewer match positions than that
    // of 2 rows of 8), else items 16 w4 .. 16 w4 + 15 of the tile in raster order; key i of the strip
    const bool quad = p.tk.lw == 3 && th == 8;
    const int it0 = 16 * w4;
    const int sr0 = quad ? x0 + 4 * (w4 >> 1) : x0 + (it0 >> p.tk.lw);
    const int sr1 = quad ? sr0 + 3 : x0 + ((it0 + 15) >> p.tk.lw);
    const int sc0 = quad ? y0 + 4 * (w4 & 1) : y0 + (it0 & (tw - 1));
    const int sc1 = quad ? sc0 + 3 : sc0 + min(tw, 16) - 1;
    auto strip_key = [&](int i, int& x, int& y) {
        x = quad ? sr0 + (i >> 2) : x0 + ((it0 + i) >> p.tk.lw);
        y = quad ? sc0 + (i & 3) : y0 + ((it0 + i) & (tw - 1));
    };
    // the strip is a rectangle: key i at row sr0 + i / sC, column sc0 + i mod sC.  Bits of the keys in
    // rows rlo .. rhi, columns clo .. chi (relative to the strip's first row and column)
    const int sC = sc1 - sc0 + 1, sR = 16 / sC;
    auto strip_bits = [&](int rlo, int rhi, int clo, int chi) {
        rlo = max(rlo, 0), rhi = min(rhi, sR - 1), clo = max(clo, 0), chi = min(chi, sC - 1);
        uint32_t bits = 0u;
        if (clo <= chi) {
            const uint32_t cb = ((2u << chi) - 1u) & ~((1u << clo) - 1u);
            for (int r = rlo; r <= rhi; ++r) bits |= cb << (sC * r);
        }
        return bits;
    };
    if (sr0 >= p.Hk || sc0 >= p.Wk) return;  // the strip lies past the grid's edge
    const int hr0 = max(sr0 - p.b, 0), hr1 = min(sr1 + p.b, p.Hk - 1);
    const int hc0 = max(sc0 - p.b, 0), hc1 = min(sc1 + p.b, p.Wk - 1);
    const int nrows = hr1 - hr0 + 1;  // at most kStripMaxRows
    const int32_t* off = p.offsets + static_cast<size_t>(s) * p.nkeys;
    int32_t* const lo_w = s_lo[wave];
    int32_t* const pre_w = s_pre[wave];
    int E;
    {
        // entry count of halo row `lane`, then an inclusive scan across the wave
        int cnt = 0;
        if (lane < nrows) {
            const int r = hr0 + lane;
            const int32_t lo = off[r * p.Wk + hc0];
            lo_w[lane] = lo;
            cnt = off[r * p.Wk + hc1 + 1] - lo;
        }
        int incl = cnt;
#pragma unroll
        for (int k2 = 1; k2 < 64; k2 <<= 1) {
            const int y = __shfl_up(incl, k2, 64);
            if (lane >= k2) incl += y;
        }
        if (lane < nrows) pre_w[lane + 1] = incl;
        if (lane == 0) pre_w[0] = 0;
        E = __shfl(incl, nrows - 1, 64);
    }
    wave_lds_sync();

    // this lane's key (column of the first products): key m of the strip
    int kx, ky;
    strip_key(m, kx, ky);
    const bool key_ok = kx < p.Hk && ky < p.Wk;
    const size_t kslice = static_cast<size_t>(s) * p.nkeys;
    const size_t krow = kslice + (key_ok ? static_cast<size_t>(kx) * p.Wk + ky : static_cast<size_t>(sr0) * p.Wk + sc0);
    auto leave_keys = [&]() {
        if (key_ok && g4 == 0 && wave == 0) p.heavy[atomicAdd(p.n_heavy, 1)] = static_cast<int32_t>(krow);
    };
    if constexpr (DIFF) {
        if (E > p.heavy_entries) {
            leave_keys();
            return;
        }
    }
    bf16x8_t kf[KS::kDs], vf[KS::kDs];
#pragma unroll
    for (int ds = 0; ds < KS::kDs; ++ds) {
        const int d = 32 * ds + 8 * g4;
        uint4 kw = make_uint4(0u, 0u, 0u, 0u), vw = kw;
        if (d < D) {
            kw = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.K) + krow * D + d);
            vw = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.V) + krow * D + d);
        }
        kf[ds] = __builtin_bit_cast(bf16x8_t, kw);
        vf[ds] = __builtin_bit_cast(bf16x8_t, vw);
    }
    float lam = 0.f;
    if constexpr (DIFF) lam = p.lam[s];
    const uint32_t live = static_cast<uint32_t>(__ballot(key_ok)) & 0xFFFFu;  // keys of the strip inside the grid
    const uint32_t key_local = static_cast<uint32_t>(kx) * p.Wk + ky;  // raster index (causal test)

    // a fragment holds one half's channels, or with 16 and 32 channels both halves': the lane groups before kHalfG, and the others
    constexpr bool kMixed = KS::kDs == 1;
    constexpr int kHalfG = D / 16;
    auto half_of = [&](bf16x8_t x, int h) {
        return (g4 < kHalfG) == (h == 0) ? x : __builtin_bit_cast(bf16x8_t, make_uint4(0u, 0u, 0u, 0u));
    };
    f32x4_t dk[KS::kOt], dv[KS::kOt];
#pragma unroll
    for (int o = 0; o < KS::kOt; ++o) dk[o] = dv[o] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    // staging: lane pair (2 t, 2 t + 1) finds entry slot t; the even lane brings its statistics
    const int t = lane >> 1, hf = lane & 1;
    const uint16_t* const Qb = static_cast<const uint16_t*>(p.Q);
    const uint16_t* const Gb = static_cast<const uint16_t*>(p.dO);
    auto slot_code = [&](int c0) {
        const int v = c0 + t;
        if (v >= E) return -1;
        int lo = 0, hi = nrows - 1;  // halo row holding flat position v: the last with pre <= v
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (pre_w[mid] <= v) lo = mid; else hi = mid - 1;
        }
        return static_cast<int>(p.entries[lo_w[lo] + (v - pre_w[lo])]);
    };
    unsigned char* const rows_q = s_row[wave];
    unsigned char* const rows_g = s_row[wave] + kCE * KS::kRowB + 64;
    // B operands of the second products, channel tile o: lane (n, g4) holds entries 4 g4 .. 4 g4 + 3 and
    // 16 + 4 g4 .. 16 + 4 g4 + 3 at channel 16 o + n.  The transposing LDS load hands lane (n, g4) rows
    // 4 g4 .. 4 g4 + 3 at channel 16 o + n when it addresses row 4 g4 + n / 4 at channels 4 (n mod 4) .. + 3
    // (+ 16 o); a second load 16 rows further gives the other four.
    const int tr_off = (4 * g4 + (m >> 2)) * KS::kRowB + 8 * (m & 3);
    auto tr_pair = [&](const unsigned char* a) {
        using lds_v4 = __attribute__((address_space(3))) bf16x4_t*;
        const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_v4)(a));
        const bf16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_v4)(a + 16 * KS::kRowB));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    int code = slot_code(TEAM > 1 ? kCE * wave : 0);
    for (int c0 = TEAM > 1 ? kCE * wave : 0; c0 < E; c0 += kCE * TEAM) {
        {
            uint32_t qe = 0, qg = 0;
            if (code >= 0) divmod(static_cast<uint32_t>(code), p.div_n, qe, qg);
            int32_t match = -1, earlier = 0;
            float lse = 0.f, dq = 0.f;
            float2 second = make_float2(0.f, 0.f);
            if (hf == 0 && code >= 0) {
                match = p.J[code];
                if constexpr (DIFF) {
                    const float4 st = p.stats[qg];
                    if constexpr (MULTI) earlier = p.J[qg];
                    lse = st.x, dq = st.y;
                    second = make_float2(st.z, st.w);
                } else {
                    lse = p.lse2[qg];
                    dq = p.Dq[qg];
                }
            }
            // the chunk's q and dO rows, kLR consecutive lanes per row (whole spans per load): lane l
            // brings pieces l mod kLR (+ kLR ...) of entry slots l / kLR + kRpi j; entry slot e's query
            // comes from lane 2 e (-1: past the entries, a zero row keeps the operands finite)
            constexpr int kLR = KS::kPieces < 8 ? KS::kPieces : 8;  // lanes per row
            constexpr int kRpi = 64 / kLR;                          // rows per load instruction
            constexpr int kRep = kCE / kRpi;                        // load instructions per row set
            constexpr int kPpl = KS::kPieces / kLR;                 // pieces per lane and row
            const int er = lane / kLR, ep = lane % kLR;
            const int my_q = code >= 0 ? static_cast<int>(qg) : -1;
            uint4 val[2][kRep][kPpl];
#pragma unroll
            for (int j = 0; j < kRep; ++j) {
                const int qj = __shfl(my_q, 2 * (er + kRpi * j), 64);
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                    const uint16_t* const row = (a ? Gb : Qb) + static_cast<size_t>(max(qj, 0)) * D;
                    const uint4* src = reinterpret_cast<const uint4*>(row);
#pragma unroll
                    for (int k = 0; k < kPpl; ++k)
                        val[a][j][k] = qj >= 0 ? src[ep + kLR * k] : make_uint4(0u, 0u, 0u, 0u);
                }
            }
#pragma unroll
            for (int j = 0; j < kRep; ++j)
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int k = 0; k < kPpl; ++k)
                        *reinterpret_cast<uint4*>((a ? rows_g : rows_q) + (er + kRpi * j) * KS::kRowB +
                                                  (ep + kLR * k) * 16) = val[a][j][k];
            if (hf == 0) {
                int4 meta = make_int4(DIFF ? 0 : -(1 << 30), -(1 << 30), 0, 0);  // no key is near this match
                if constexpr (kQueryIndex) s_el[wave][t][0] = s_el[wave][t][1] = 0;
                if (code >= 0) {
                    uint32_t mu, mv;
                    divmod(static_cast<uint32_t>(clamp_index(match, p.nkeys)), p.div_wk, mu, mv);
                    meta = make_int4(static_cast<int>(mu), static_cast<int>(mv), __float_as_int(lse),
                                     __float_as_int(dq));
                    if constexpr (kQueryIndex) {
                        uint32_t sl, local;
                        divmod(qg, p.div_plane, sl, local);
                        if constexpr (DIFF) local = causal_limit(p, sl, local);
                        s_el[wave][t][1] = static_cast<int32_t>(local);
                    }
                    if constexpr (DIFF) {
                        // the strip's keys that the entry counts for, once for all: in its window, not after the query, in
                        // none of the query's earlier windows
                        const int ru = static_cast<int>(mu) - sr0, cv = static_cast<int>(mv) - sc0;
                        uint32_t in = strip_bits(ru - p.b, ru + p.b, cv - p.b, cv + p.b) & live;
                        if (kQueryIndex && p.causal) {
                            uint32_t lr, lc;
                            divmod(static_cast<uint32_t>(s_el[wave][t][1]), p.div_wk, lr, lc);
                            const int last = static_cast<int>(lr) - sr0;
                            in &= strip_bits(0, last - 1, 0, 15) | strip_bits(last, last, 0, static_cast<int>(lc) - sc0);
                        }
                        if constexpr (MULTI) {
                            for (int f = 0; f < static_cast<int>(qe); ++f) {
                                uint32_t fu, fv;
                                const int32_t at = f == 0 ? earlier : p.J[static_cast<size_t>(f) * p.n + qg];
                                divmod(static_cast<uint32_t>(clamp_index(at, p.nkeys)), p.div_wk, fu, fv);
                                const int hu = static_cast<int>(fu) - sr0, hv = static_cast<int>(fv) - sc0;
                                in &= ~strip_bits(hu - p.b, hu + p.b, hv - p.b, hv + p.b);
                            }
                        }
                        // (a set of one key: its weights count, its score's gradients do not)
                        if (!kQueryIndex || __float_as_uint(second.y) != kOneKey) in |= in << 16;
                        meta.x = static_cast<int>(in);
                    } else if constexpr (MULTI) {
                        // the centres of the query's windows 0 .. e-1 (loaded together), then the strip's
                        // keys their (2 b + 1)^2 neighbourhoods hold
                        int32_t pc[kMaxKappa - 1];
#pragma unroll
                        for (int f = 0; f < kMaxKappa - 1; ++f)
                            pc[f] = f < static_cast<int>(qe) ? p.J[static_cast<size_t>(f) * p.n + qg] : 0;
                        uint32_t held = 0u;
#pragma unroll
                        for (int f = 0; f < kMaxKappa - 1; ++f) {
                            if (f < static_cast<int>(qe)) {
                                uint32_t fu, fv;
                                divmod(static_cast<uint32_t>(clamp_index(pc[f], p.nkeys)), p.div_wk, fu, fv);
                                const int ru = static_cast<int>(fu) - sr0, cv = static_cast<int>(fv) - sc0;
                                held |= strip_bits(ru - p.b, ru + p.b, cv - p.b, cv + p.b);
                            }
                        }
                        s_el[wave][t][0] = static_cast<int32_t>(held);
                    }
                }
                s_meta[wave][t] = meta;
                if constexpr (DIFF) s_second[wave][t] = second;
            }
        }
        code = slot_code(c0 + kCE * TEAM);  // the next chunk's entries load during the products
        wave_lds_sync();

        // S^T, dP^T for entries 16 et + (0..15) of the chunk against the strip's 16 keys
        f32x4_t sc[2], dp[2], sc2[2];
#pragma unroll
        for (int et = 0; et < 2; ++et) {
            sc[et] = dp[et] = sc2[et] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            const int er = et * 16 + m;
#pragma unroll
            for (int ds = 0; ds < KS::kDs; ++ds) {
                const int d = 32 * ds + 8 * g4;
                bf16x8_t aq = __builtin_bit_cast(bf16x8_t, make_uint4(0u, 0u, 0u, 0u)), ag = aq;
                if (d < D) {
                    aq = lds_frag(rows_q + er * KS::kRowB + d * 2);
                    ag = lds_frag(rows_g + er * KS::kRowB + d * 2);
                }
                if constexpr (!DIFF) {
                    sc[et] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aq, kf[ds], sc[et], 0, 0, 0);
                } else if constexpr (kMixed) {
                    sc[et] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aq, half_of(kf[ds], 0), sc[et], 0, 0, 0);
                    sc2[et] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aq, half_of(kf[ds], 1), sc2[et], 0, 0, 0);
                } else if (ds < KS::kDs / 2) {
                    sc[et] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aq, kf[ds], sc[et], 0, 0, 0);
                } else {
                    sc2[et] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aq, kf[ds], sc2[et], 0, 0, 0);
                }
                dp[et] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ag, vf[ds], dp[et], 0, 0, 0);
            }
        }
        // P and dS of (key m, entry 16 et + 4 g4 + r): operand slot 4 et + r of this lane, in three parts
        uint32_t ph[8], pm[8], pl[8], sh[8], sm[8], sl[8];
        float wd[8], d1[8], d2[8];  // differential: P, dS1, dS2, split when they enter
#pragma unroll
        for (int et = 0; et < 2; ++et) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int te = et * 16 + 4 * g4 + r;
                const int4 mt = s_meta[wave][te];
                if constexpr (DIFF) {
                    const float2 st = s_second[wave][te];
                    const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[et][r], p.scale_log2e, -__int_as_float(mt.z)));
                    const float p2 = lam * __builtin_amdgcn_exp2f(fmaf(sc2[et][r], p.scale_log2e, -st.x));
                    // (selected by bits: a key that is left out may hold anything)
                    auto kept = [](float x, int in) { return __uint_as_float(__float_as_uint(x) & static_cast<uint32_t>(in)); };
                    const int in = __builtin_amdgcn_sbfe(mt.x, m, 1), in_ds = kQueryIndex ? __builtin_amdgcn_sbfe(mt.x, m + 16, 1) : in;
                    wd[4 * et + r] = kept(p1 - p2, in);
                    d1[4 * et + r] = kept(p1 * (dp[et][r] - __int_as_float(mt.w)), in_ds);
                    d2[4 * et + r] = kept(p2 * (st.y - dp[et][r]), in_ds);
                    continue;
                }
                bool ok = key_ok && abs(mt.x - kx) <= p.b && abs(mt.y - ky) <= p.b;
                if constexpr (MULTI) {
                    // not when an earlier window of the query holds this key (key m of the strip)
                    ok = ok && !((static_cast<uint32_t>(s_el[wave][te][0]) >> m) & 1u);
                    if (p.causal) ok = ok && key_local <= static_cast<uint32_t>(s_el[wave][te][1]);
                } else if constexpr (MODE == kStripCausal) {
                    ok = ok && key_local <= static_cast<uint32_t>(s_el[wave][te][1]);
                }
                const float pr = ok ? __builtin_amdgcn_exp2f(sc[et][r] * p.scale_log2e - __int_as_float(mt.z)) : 0.f;
                const float dsr = pr * (dp[et][r] - __int_as_float(mt.w));
                split3(pr, ph[4 * et + r], pm[4 * et + r], pl[4 * et + r]);
                split3(dsr, sh[4 * et + r], sm[4 * et + r], sl[4 * et + r]);
            }
        }
        auto operand = [](const uint32_t (&v)[8]) {
            return __builtin_bit_cast(bf16x8_t, make_uint4(hi16_pair(v[0], v[1]), hi16_pair(v[2], v[3]),
                                                           hi16_pair(v[4], v[5]), hi16_pair(v[6], v[7])));
        };
        if constexpr (DIFF) {
            // acc[o] += x rows for the channel tiles first .. last - 1; keep: which channels of a tile count (0: all, 1: m < 8, 2: the others)
            auto add = [&](const float (&x)[8], f32x4_t (&acc)[KS::kOt], const unsigned char* rows, int first, int last, int keep) {
#pragma unroll
                for (int i = 0; i < 8; ++i) split3(x[i], ph[i], pm[i], pl[i]);
                const bf16x8_t ah = operand(ph), am = operand(pm), al = operand(pl);
#pragma unroll
                for (int o = 0; o < KS::kOt; ++o) {
                    if (o < first || o >= last) continue;
                    bf16x8_t b = tr_pair(rows + tr_off + 32 * o);
                    if (keep) b = (m < 8) == (keep == 1) ? b : __builtin_bit_cast(bf16x8_t, make_uint4(0u, 0u, 0u, 0u));
                    acc[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ah, b, acc[o], 0, 0, 0);
                    acc[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(am, b, acc[o], 0, 0, 0);
                    acc[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(al, b, acc[o], 0, 0, 0);
                }
            };
            constexpr bool kOne = KS::kOt == 1;  // 16 channels: both halves in one tile
            add(wd, dv, rows_g, 0, KS::kOt, 0);
            add(d1, dk, rows_q, 0, kOne ? 1 : KS::kOt / 2, kOne ? 1 : 0);
            add(d2, dk, rows_q, kOne ? 0 : KS::kOt / 2, KS::kOt, kOne ? 2 : 0);
            wave_lds_sync();  // this chunk's LDS reads come before the next chunk's writes
            continue;
        }
        const bf16x8_t aph = operand(ph), apm = operand(pm), apl = operand(pl);
        const bf16x8_t ash = operand(sh), asm_ = operand(sm), asl = operand(sl);
        // dV_w += P dO_E, dK_w += dS Q_E per 16-channel tile o
#pragma unroll
        for (int o = 0; o < KS::kOt; ++o) {
            const bf16x8_t bq = tr_pair(rows_q + tr_off + 32 * o), bg = tr_pair(rows_g + tr_off + 32 * o);
            dv[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aph, bg, dv[o], 0, 0, 0);
            dv[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(apm, bg, dv[o], 0, 0, 0);
            dv[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(apl, bg, dv[o], 0, 0, 0);
            dk[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ash, bq, dk[o], 0, 0, 0);
            dk[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(asm_, bq, dk[o], 0, 0, 0);
            dk[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(asl, bq, dk[o], 0, 0, 0);
        }
        wave_lds_sync();  // this chunk's LDS reads come before the next chunk's writes
    }

    if constexpr (TEAM > 1) {
        // the other waves' sums, from their staging areas (16 keys' two gradient rows fit those of 32 entries)
        f32x4_t* const mine = reinterpret_cast<f32x4_t*>(s_row[wave]) + lane;
        if (wave > 0) {
#pragma unroll
            for (int o = 0; o < KS::kOt; ++o) mine[128 * o] = dk[o], mine[128 * o + 64] = dv[o];
        }
        __syncthreads();
        if (wave > 0) return;
        for (int w = 1; w < TEAM; ++w) {
            const f32x4_t* const other = reinterpret_cast<const f32x4_t*>(s_row[w]) + lane;
#pragma unroll
            for (int o = 0; o < KS::kOt; ++o) dk[o] += other[128 * o], dv[o] += other[128 * o + 64];
        }
    }
    if constexpr (DIFF) {
        float sum = 0.f;
#pragma unroll
        for (int o = 0; o < KS::kOt; ++o)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += fabsf(dk[o][r]) + fabsf(dv[o][r]);
        if (__any(!(sum < INFINITY))) {
            leave_keys();
            return;
        }
    }
    // lane holds keys 4 g4 + r of the strip, channel 16 o + m
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        int ox, oy;
        strip_key(4 * g4 + r, ox, oy);
        if (ox >= p.Hk || oy >= p.Wk) continue;
        const size_t row = (kslice + static_cast<size_t>(ox) * p.Wk + oy) * D;
#pragma unroll
        for (int o = 0; o < KS::kOt; ++o) {
            p.dK[row + 16 * o + m] = dk[o][r] * p.scale;
            p.dV[row + 16 * o + m] = dv[o][r];
        }
    }
}

// ---------------------------------------------------------------------------
// Pieces of the strips with fp32 storage.
// ---------------------------------------------------------------------------
constexpr int kStripFE = 16;  // entries per chunk

template <int N>
__device__ __forceinline__ void load_floats(float (&v)[N], const float* a)
{
    if constexpr (N >= 4) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const f32x4_t x = *reinterpret_cast<const f32x4_t*>(a + i);
            v[i] = x[0], v[i + 1] = x[1], v[i + 2] = x[2], v[i + 3] = x[3];
        }
    } else if constexpr (N == 2) {
        const f32x2_t x = *reinterpret_cast<const f32x2_t*>(a);
        v[0] = x[0], v[1] = x[1];
    } else {
        v[0] = a[0];
    }
}

template <int N>
__device__ __forceinline__ void store_floats(float* a, const float (&v)[N])
{
    if constexpr (N >= 4) {
#pragma unroll
        for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4_t*>(a + i) = f32x4_t{v[i], v[i + 1], v[i + 2], v[i + 3]};
    } else if constexpr (N == 2) {
        *reinterpret_cast<f32x2_t*>(a) = f32x2_t{v[0], v[1]};
    } else {
        a[0] = v[0];
    }
}

// The 16 keys of a one-wave block, as in the bf16 kernel: rows sr0 .. sr1, columns sc0 .. sc1 of slice s.
struct KeyStripF {
    uint32_t s;
    int lw, x0, y0, it0, sr0, sr1, sc0, sc1;
    bool quad;

    __device__ __forceinline__ KeyStripF(const Tiling& tk, uint32_t strip)
    {
        uint32_t k, tr, tc;
        divmod(strip / kStripWaves, tk.div_slice, s, k);
        tile_coords(tk, k, tr, tc);
        lw = tk.lw;
        const int tw = 1 << lw, th = kTileKeys >> lw;
        x0 = static_cast<int>(tr) * th, y0 = static_cast<int>(tc) * tw;
        const int w4 = static_cast<int>(strip % kStripWaves);
        quad = lw == 3 && th == 8;
        it0 = 16 * w4;
        sr0 = quad ? x0 + 4 * (w4 >> 1) : x0 + (it0 >> lw);
        sr1 = quad ? sr0 + 3 : x0 + ((it0 + 15) >> lw);
        sc0 = quad ? y0 + 4 * (w4 & 1) : y0 + (it0 & (tw - 1));
        sc1 = quad ? sc0 + 3 : sc0 + min(tw, 16) - 1;
    }
    __device__ __forceinline__ void key(int i, int& x, int& y) const
    {
        x = quad ? sr0 + (i >> 2) : x0 + ((it0 + i) >> lw);
        y = quad ? sc0 + (i & 3) : y0 + ((it0 + i) & ((1 << lw) - 1));
    }
    // bits of the keys in rows rlo .. rhi, columns clo .. chi (relative to the strip's first)
    __device__ __forceinline__ uint32_t bits(int rlo, int rhi, int clo, int chi) const
    {
        const int sC = sc1 - sc0 + 1, sR = 16 / sC;
        rlo = max(rlo, 0), rhi = min(rhi, sR - 1), clo = max(clo, 0), chi = min(chi, sC - 1);
        uint32_t set = 0u;
        if (clo <= chi) {
            const uint32_t cb = ((2u << chi) - 1u) & ~((1u << clo) - 1u);
            for (int r = rlo; r <= rhi; ++r) set |= cb << (sC * r);
        }
        return set;
    }
};

// The entries of a strip's halo: their ranges into lo, pre; returns their number.
template <typename Lds>
__device__ __forceinline__ int strip_entries(const BwdParams& p, const KeyStripF& t, Lds& lds, int lane, int& nrows)
{
    const int hr0 = max(t.sr0 - p.b, 0), hr1 = min(t.sr1 + p.b, p.Hk - 1);
    const int hc0 = max(t.sc0 - p.b, 0), hc1 = min(t.sc1 + p.b, p.Wk - 1);
    nrows = hr1 - hr0 + 1;  // at most kStripMaxRows
    const int32_t* const off = p.offsets + static_cast<size_t>(t.s) * p.nkeys;
    int cnt = 0;
    if (lane < nrows) {
        const int r = hr0 + lane;
        const int32_t lo = off[r * p.Wk + hc0];
        lds.lo[lane] = lo;
        cnt = off[r * p.Wk + hc1 + 1] - lo;
    }
    int incl = cnt;
#pragma unroll
    for (int k2 = 1; k2 < 64; k2 <<= 1) {
        const int y = __shfl_up(incl, k2, 64);
        if (lane >= k2) incl += y;
    }
    if (lane < nrows) lds.pre[lane + 1] = incl;
    if (lane == 0) lds.pre[0] = 0;
    const int E = __shfl(incl, nrows - 1, 64);
    wave_lds_sync();
    return E;
}

}  // namespace
}  // namespace scram
