// Differential attention on the matrix cores for bf16 storage: the pieces that
// the forward (scram_diff.hip) and the gradients' query side
// (scram_diff_backward.hip) share.
//
// A wave takes 16 neighbouring queries and visits the keys of their windows in
// the clusters and key boxes of scram_tile.h, a block of 16 keys at a time:
// the blocks' key and value rows are gathered a row per 4 consecutive lanes,
// staged in the wave's LDS tiles and read back as the products' operands,
// while the next block's rows load.  All windows of the queries are clustered
// together; a query keeps the slots of window e in the cluster that holds that
// window's centre, less the keys of its windows 0 .. e - 1 and, with the causal
// mask, those after its limit, so every key of its set enters once.
//
// Everything here lives in an unnamed namespace, like scram_device.h.

#pragma once

#include "scram_diff.h"
#include "scram_tile.h"

namespace scram {
namespace {

constexpr int kRowPad = 16;  // bytes behind each LDS row: spreads a column read over the banks

// Where a wave's queries lie and what they attend to.
template <int MK>
struct DiffTile {
    uint32_t g, gq;      // this lane's query m, and the same with a query inside the grid for those outside
    uint32_t s;          // its slice (the tile's)
    bool valid;
    uint32_t centre;     // its first match
    int u[MK], v[MK];    // its windows' centres
    int mine[MK];        // the clusters that hold them (-1: no such window)
    uint32_t limit;      // causal: raster index of its last key
    TileClusters tc;
};

// The 16 queries of a wave (lane (m, g4) works on query m) and their clusters; tc.nclu == 0: none lies inside the grid,
// < 0: the boxes hold more than `most` blocks of 16 keys.
template <int W, int MK>
__device__ __forceinline__ DiffTile<MK> diff_tile(const DiffParams& p, uint32_t blk, int wave, int lane, int most)
{
    constexpr int NJ = MK == 4 ? 4 : 2;
    const int m = lane & 15, g4 = lane >> 4;
    DiffTile<MK> t;
    uint32_t g0, rem;
    t.valid = tile_item<kBlock / 4>(p.tq, blk, tile_wave_item(p.tq, wave, m), t.g);
    tile_item<kBlock / 4>(p.tq, blk, 0, g0);  // item 0 of a tile is always inside the grid
    t.gq = t.valid ? t.g : g0;
    divmod(t.gq, p.div_plane, t.s, rem);
    t.limit = p.causal ? causal_limit(p, t.s, rem) : 0u;
    const int ew = g4 & (NJ - 1);  // the window whose centre this lane clusters
    int iu = 0, iv = 0;
#pragma unroll
    for (int e = 0; e < MK; ++e) {
        const int f = e < p.kappa ? e : 0;  // a window past kappa repeats the first and is not clustered
        const uint32_t at = static_cast<uint32_t>(clamp_index(p.J[static_cast<size_t>(f) * p.n + t.gq], p.nkeys));
        if (e == 0) t.centre = at;
        uint32_t uu, vv;
        divmod(at, p.div_wk, uu, vv);
        t.u[e] = static_cast<int>(uu), t.v[e] = static_cast<int>(vv);
        iu = e == 0 || ew == e ? t.u[e] : iu, iv = e == 0 || ew == e ? t.v[e] : iv;
    }
    t.tc = tile_clusters_joint<W / 2, NJ, true>(t.valid && ew < p.kappa, iu, iv, lane, tile_radius(W), p.Hk, p.Wk, most);
#pragma unroll
    for (int e = 0; e < MK; ++e) t.mine[e] = __shfl(t.tc.mine, m + 16 * e);
    return t;
}

// A cluster's box as blocks of 16 slots, 4 groups of 4 neighbouring columns of one box row: the box is widened to whole
// groups (columns past it belong to no window).  Lane group g4 has group 4 k + g4 of the box in raster order, for the rows it
// brings and for the scores it holds.
struct DiffBox {
    int r0, c0, h, gw, nb, q, r;   // rows, groups of a row, blocks; a step of 4 groups: q rows and r groups
    uint32_t step, wrap, last;     // the key index' change in a step, more where it wraps; the box's last key
};

__device__ __forceinline__ DiffBox diff_box(const TileClusters& tc, int cl, int Wk, uint32_t nkeys)
{
    DiffBox b;
    b.r0 = __builtin_amdgcn_readlane(tc.t_r0, cl);
    b.c0 = __builtin_amdgcn_readlane(tc.t_c0, cl);
    b.h = __builtin_amdgcn_readlane(tc.t_h, cl);
    b.gw = (__builtin_amdgcn_readlane(tc.t_bw, cl) + 3) >> 2;  // at most 7
    b.nb = (b.h * b.gw + 3) >> 2;
    b.q = b.gw == 1 ? 4 : b.gw == 2 ? 2 : b.gw <= 4 ? 1 : 0;
    b.r = 4 - b.q * b.gw;
    b.step = static_cast<uint32_t>(b.q * Wk + 4 * b.r);
    b.wrap = static_cast<uint32_t>(Wk - 4 * b.gw);
    b.last = min(static_cast<uint32_t>((b.r0 + b.h - 1) * Wk + b.c0 + 4 * b.gw - 1), nkeys - 1u);
    return b;
}

// A lane's pieces of the key or value rows in flight: a whole row by consecutive lanes (spans of 128 bytes and more take the
// memory pipe half the time that spans of 64 do), neighbouring slots by the same lanes.  (Named members: an array loaded on two
// paths of a loop ends in scratch memory.)
template <int D>
struct DiffRows {
    static constexpr int kLanes = D / 8;     // of a row, 16 bytes each
    static constexpr int kRows = D / 32;     // rows per lane: kRows (lane / kLanes) and the next ones
    u32x4_t a, b, c, d;

    __device__ __forceinline__ void load(const unsigned char* rows, const uint32_t (&off)[kRows])
    {
        a = *reinterpret_cast<const u32x4_t*>(rows + off[0]);
        if constexpr (kRows > 1) b = *reinterpret_cast<const u32x4_t*>(rows + off[1]);
        if constexpr (kRows > 2) {
            c = *reinterpret_cast<const u32x4_t*>(rows + off[2]);
            d = *reinterpret_cast<const u32x4_t*>(rows + off[3]);
        }
    }

    __device__ __forceinline__ void store(unsigned char* to, int row_bytes) const
    {
        *reinterpret_cast<u32x4_t*>(to) = a;
        if constexpr (kRows > 1) *reinterpret_cast<u32x4_t*>(to + row_bytes) = b;
        if constexpr (kRows > 2) {
            *reinterpret_cast<u32x4_t*>(to + 2 * row_bytes) = c;
            *reinterpret_cast<u32x4_t*>(to + 3 * row_bytes) = d;
        }
    }
};

// Walks the boxes of the wave's clusters (at least one).  block(bias): a block's rows are staged at tk and tv (row r at
// r * (2 D + kRowPad)); bias[i], the start of a score's sum, is 0 if slot 4 g4 + i belongs to query m here, else -inf.
template <int D, int W, bool CAUSAL, int MK, typename Block>
__device__ __forceinline__ void diff_walk(const DiffParams& p, const DiffTile<MK>& t, const unsigned char* Kb, const unsigned char* Vb,
                                          unsigned char* tk, unsigned char* tv, int lane, Block&& block)
{
    using Rows = DiffRows<D>;
    constexpr int B = W / 2;
    constexpr int kRowB = 2 * D + kRowPad;
    const int g4 = lane >> 4;
    // the lane brings piece lpiece of slots lslot .. lslot + kRows - 1, all in group g4
    const int lslot = Rows::kRows * (lane / Rows::kLanes), lpiece = lane % Rows::kLanes;
    int qx = 0, qy = 0;
    if constexpr (CAUSAL) {
        uint32_t xx, yy;
        divmod(t.limit, p.div_wk, xx, yy);
        qx = static_cast<int>(xx), qy = static_cast<int>(yy);
    }
    // bit positions 0..3 as values the compiler cannot see: one bit-field extract per slot below
    int bit_at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("s_mov_b32 %0, %1" : "=s"(bit_at[i]) : "i"(i));

    Rows kr, vr;
    auto load = [&](uint32_t key, uint32_t last) {  // a slot past the box's last row reads its last key's row
        uint32_t off[Rows::kRows];
#pragma unroll
        for (int j = 0; j < Rows::kRows; ++j) off[j] = min(key + j, last) * (2u * D) + 16u * lpiece;
        kr.load(Kb, off);
        vr.load(Vb, off);
    };
    auto stage = [&]() {
        const int off = lslot * kRowB + 16 * lpiece;
        kr.store(tk + off, kRowB);
        vr.store(tv + off, kRowB);
    };
    // the lane group's place in a box: row and group, and the key of the first slot that the lane brings
    struct Place {
        int row, grp;
        uint32_t key;
    };
    auto first = [&](const DiffBox& b) {
        Place a;
        a.row = (g4 >= b.gw) + (g4 >= 2 * b.gw) + (g4 >= 3 * b.gw);
        a.grp = g4 - a.row * b.gw;
        a.key = static_cast<uint32_t>((b.r0 + a.row) * p.Wk + b.c0 + 4 * a.grp + (lslot & 3));
        return a;
    };
    auto advance = [](const DiffBox& b, Place& a) {
        a.grp += b.r;
        a.row += b.q;
        a.key += b.step;
        const bool carry = a.grp >= b.gw;
        a.grp -= carry ? b.gw : 0;
        a.row += carry ? 1 : 0;
        a.key += carry ? b.wrap : 0u;
    };

    DiffBox bx = diff_box(t.tc, 0, p.Wk, p.nkeys);
    Place next = first(bx);  // of the block whose rows load
    load(next.key, bx.last);
    for (int c = 0;;) {
        // window e of query m in this box: its first row, its rows less one, its columns; none where its centre is elsewhere
        int jd[MK], jn[MK];
        uint32_t jx[MK];
        bool mine[MK];
#pragma unroll
        for (int e = 0; e < MK; ++e) {
            jd[e] = t.u[e] - B - bx.r0;
            jn[e] = min(2 * B, bx.h - 1 - jd[e]);
            const int lo = max(t.v[e] - B - bx.c0, 0), hi = min(min(t.v[e] + B, p.Wk - 1) - bx.c0, 31);
            // no columns for a window beside or wholly below the box (its row count would be negative) or past kappa
            const int n = jn[e] >= 0 && (MK == 1 || e < p.kappa) ? max(hi - lo + 1, 0) : 0;
            jx[e] = ((1u << n) - 1u) << (lo & 31);
            mine[e] = c == t.mine[e];
        }
        int cr = 0;        // causal: the limit's row as a box row
        uint32_t cc = 0u;  // and the box columns up to its column
        if constexpr (CAUSAL) {
            cr = qx - bx.r0;
            const int qc = qy - bx.c0;
            cc = qc < 0 ? 0u : qc >= 30 ? 0x7FFFFFFFu : (2u << qc) - 1u;
        }
        Place at = next;  // of the block that is computed
        auto one = [&]() {
            uint32_t bits = 0u, earlier = 0u;
#pragma unroll
            for (int e = 0; e < MK; ++e) {
                const uint32_t w = static_cast<unsigned>(at.row - jd[e]) <= static_cast<unsigned>(jn[e]) ? jx[e] : 0u;
                bits |= mine[e] ? w & ~earlier : 0u;
                earlier |= w;
            }
            if constexpr (CAUSAL) bits &= at.row < cr ? ~0u : at.row == cr ? cc : 0u;
            bits = ~(bits >> (4 * at.grp));
            f32x4_t bias;
#pragma unroll
            for (int i = 0; i < 4; ++i)  // 0xFF800000 is -inf
                bias[i] = __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_sbfe(static_cast<int>(bits), bit_at[i], 1)) << 23);
            block(bias);
        };
        for (int k = 1; k < bx.nb; ++k) {
            stage();
            advance(bx, next);
            load(next.key, bx.last);
            wave_lds_sync();
            one();
            at = next;
            wave_lds_sync();  // this block's LDS reads come before the next block's writes
        }
        stage();
        const bool more = c + 1 < t.tc.nclu;
        DiffBox nx = bx;
        if (more) {
            nx = diff_box(t.tc, c + 1, p.Wk, p.nkeys);
            next = first(nx);
            load(next.key, nx.last);
        }
        wave_lds_sync();
        one();
        if (!more) break;
        bx = nx;
        ++c;
        wave_lds_sync();
    }
}

// The scores of 16 staged keys with query m, of each half of the channels.  qf: query m's fragments; a fragment that holds
// both halves (32 channels) enters twice, the other half's lane groups zeroed in q1, q2.
template <int D>
struct HalfQueries {
    using TR = TileRow<D>;
    typename TR::Frag f[TR::kDs], g[TR::kDs];  // g: 32 channels only, the last half; f is then the first

    __device__ __forceinline__ void load(const unsigned char* row, int g4)
    {
#pragma unroll
        for (int ds = 0; ds < TR::kDs; ++ds) f[ds] = TR::frag(row, ds, g4);
        if constexpr (TR::kDs == 1) {
            const typename TR::Frag whole = f[0], none = {};
            f[0] = g4 < 2 ? whole : none;
            g[0] = g4 < 2 ? none : whole;
        }
    }

    // scores with the rows whose fragment ds is key(ds), on top of bias
    template <typename Key>
    __device__ __forceinline__ void scores(Key&& key, f32x4_t bias, f32x4_t (&sc)[2]) const
    {
        sc[0] = sc[1] = bias;
#pragma unroll
        for (int ds = 0; ds < TR::kDs; ++ds) {
            const typename TR::Frag k = key(ds);
            if constexpr (TR::kDs == 1) {
                sc[0] = TR::product(k, f[0], sc[0]);
                sc[1] = TR::product(k, g[0], sc[1]);
            } else if (ds < TR::kDs / 2) {
                sc[0] = TR::product(k, f[ds], sc[0]);
            } else {
                sc[1] = TR::product(k, f[ds], sc[1]);
            }
        }
    }

    // query m's own scores with one row, on all of its lanes
    __device__ __forceinline__ void own_scores(const unsigned char* row, int g4, float (&s)[2]) const
    {
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int ds = 0; ds < TR::kDs; ++ds) {
            const typename TR::Frag k = TR::frag(row, ds, g4);
            if constexpr (TR::kDs == 1) {
                s[0] = TR::dot(f[0], k, s[0]);
                s[1] = TR::dot(g[0], k, s[1]);
            } else {
                s[ds < TR::kDs / 2 ? 0 : 1] = TR::dot(f[ds], k, s[ds < TR::kDs / 2 ? 0 : 1]);
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s[h] += __shfl_xor(s[h], 16);
            s[h] += __shfl_xor(s[h], 32);
        }
    }
};

// One map's online softmax reference of query m (base-2 domain).  It starts at the score of the query's first match, a key
// of its set, and is raised when a weight passes 2^kRescaleSlack.  Under the causal mask the match may lie after the query:
// the first kept key's weight then comes out infinite against kNoReference and sets the reference.
constexpr float kNoReference = -1e30f;

struct MapReference {
    float ref;

    __device__ __forceinline__ void start(float score, bool held, float scale) { ref = held ? score * scale : kNoReference; }

    // the weights of scores that are -inf where a slot is left out
    __device__ __forceinline__ void weights(const f32x4_t& sc, float scale, float (&w)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], scale, -ref));
    }

    // raises the reference to the largest score where that passes it by more than kRescaleSlack; the factor of the sums so far
    // (1: not raised)
    __device__ __forceinline__ float raise(const f32x4_t& sc, float scale)
    {
        float mx = fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3])) * scale;
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        if (!(mx > ref + kRescaleSlack)) return 1.f;
        const float factor = __builtin_amdgcn_exp2f(ref - mx);
        ref = mx;
        return factor;
    }
};

// The weights of both maps for a block; scale_sums(h, f) where map h's reference is raised.
template <typename Scale>
__device__ __forceinline__ void block_weights(MapReference (&ref)[2], const f32x4_t (&sc)[2], float scale, float (&w)[2][4],
                                              Scale&& scale_sums)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) ref[h].weights(sc[h], scale, w[h]);
    const float m0 = fmaxf(fmaxf(w[0][0], w[0][1]), fmaxf(w[0][2], w[0][3]));
    const float m1 = fmaxf(fmaxf(w[1][0], w[1][1]), fmaxf(w[1][2], w[1][3]));
    if (__ballot(fmaxf(m0, m1) > 256.f)) {  // 2^kRescaleSlack
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            scale_sums(h, ref[h].raise(sc[h], scale));
            ref[h].weights(sc[h], scale, w[h]);
        }
    }
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{a, b}, bf16x2_t));
}

// Four fp32 values as three bf16 parts that add up to them: two rounded to nearest, the rest fits the third.  The first two
// enter one 16x16x32 product whose other operand is doubled, the last a 16x16x16 one.
struct Parts3 {
    bf16x8_t upper;
    bf16x4_t last;
};

__device__ __forceinline__ Parts3 parts3(const float (&x)[4])
{
    const uint32_t h0 = bf16_pair(x[0], x[1]), h1 = bf16_pair(x[2], x[3]);
    const float r[4] = {x[0] - __uint_as_float(h0 << 16), x[1] - __uint_as_float(h0 & 0xFFFF0000u),
                        x[2] - __uint_as_float(h1 << 16), x[3] - __uint_as_float(h1 & 0xFFFF0000u)};
    const uint32_t m0 = bf16_pair(r[0], r[1]), m1 = bf16_pair(r[2], r[3]);
    const uint32_t l0 = bf16_pair(r[0] - __uint_as_float(m0 << 16), r[1] - __uint_as_float(m0 & 0xFFFF0000u));
    const uint32_t l1 = bf16_pair(r[2] - __uint_as_float(m1 << 16), r[3] - __uint_as_float(m1 & 0xFFFF0000u));
    return Parts3{__builtin_bit_cast(bf16x8_t, make_uint4(h0, h1, m0, m1)), __builtin_bit_cast(bf16x4_t, make_uint2(l0, l1))};
}

// c + a b over the block's 16 keys: a 4 keys of each lane group, b in parts
__device__ __forceinline__ f32x4_t product3(bf16x4_t a, const Parts3& b, f32x4_t c)
{
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_shufflevector(a, a, 0, 1, 2, 3, 4, 5, 6, 7), b.upper, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, b.last, c, 0, 0, 0);
}

// Rows 4 g4 .. 4 g4 + 3 of a staged block at channel 16 o + m: the transposing load hands lane i of each 16 the element e of
// the 8 bytes that lane 4 e + i / 4 addresses.
template <int D>
__device__ __forceinline__ bf16x4_t column4(const unsigned char* tile, int m, int g4, int o)
{
    const unsigned char* const at = tile + (4 * g4 + (m >> 2)) * (2 * D + kRowPad) + 8 * (m & 3) + 32 * o;
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4_t*)(at));
}

// Host: whether the matrix cores take this call -- up to four windows of side 3, 5, 7 or 9, a positive scale, slices of at most
// 4 GiB of key rows (bf16 rows of 32 to 128 channels).  Sets the tiling and the blocks up to which a wave walks its boxes;
// returns the tiles of 64 queries, 0: not taken.
template <int D>
uint64_t diff_tiles(DiffParams& p)
{
    if (p.kappa > 4 || p.b < 1 || p.b > 4 || !(p.scale_log2e > 0.f) || static_cast<uint64_t>(p.nkeys) * (2 * D) > 0xFFFFFFFFull)
        return 0;
    p.tq = make_tiling(p.Hq, p.Wq, kBlock / 4);
    const uint64_t tiles = tiling_blocks(p.tq, p.n / p.tq.plane);
    // A lane group takes kappa w^2 keys of its query, one after another.  4 x 256 x 256, smooth displacements, limits of 5/8, 1
    // and 12/8 as many blocks: 64 channels, two 5 x 5 windows 135, 144, 144 us, four 206, 196, 196, two of 128 channels (192 x
    // 192) 148, 139, 139; one 3 x 3 window 39, 40, 51, two 71, 73, 93; on matches of noise 12/8 cost half as much again.
    const int side = 2 * p.b + 1;
    p.tile_blocks = p.kappa * side * side * (side == 3 ? 5 : 8) / 8;
    return tiles > kMaxBlocks / 4 ? 0 : tiles;
}

}  // namespace
}  // namespace scram
