// The inverse of the match maps, shared by the gradients of the attend
// (scram_backward.hip) and of the differential attend (scram_diff_backward.hip):
// the (query, match) entries sorted by match key.  A counting sort: the query
// kernels count each match key's entries and record each entry's slot among
// them, a scan turns the counts into offsets, and the fill puts every entry at
// its key's offset plus its slot, without atomics.
//
// Everything here lives in an unnamed namespace, like scram_device.h.

#pragma once

#include "scram_grad.h"

namespace scram {
namespace {

constexpr int kScanItems = 8;                          // counts per thread in the scan
constexpr int kScanTile = kBlock * kScanItems;         // counts per scan block

// Host: blocks of a grid-stride kernel over `items`.
inline uint32_t stride_blocks(size_t items)
{
    const size_t b = (items + kBlock - 1) / kBlock;
    return static_cast<uint32_t>(b < 1 ? 1 : (b > 4096 ? 4096 : b));
}

// a[0 .. count) = 0 and, when given, *word = 0
__global__ __launch_bounds__(kBlock) void zero_i32_kernel(int32_t* a, size_t count, int32_t* word)
{
    for (size_t i = static_cast<size_t>(blockIdx.x) * kBlock + threadIdx.x; i < count;
         i += static_cast<size_t>(gridDim.x) * kBlock)
        a[i] = 0;
    if (word != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *word = 0;
}

// Exclusive scan of in[0 .. count) by one block, count <= kScanTile, into
// out (which may be in, in global or shared memory); returns the total to
// thread kBlock - 1.  wave_tot: kBlock / 64 ints of shared memory.
__device__ int32_t block_exclusive_scan(const int32_t* in, int32_t* out, size_t count, int32_t* wave_tot)
{
    const size_t base = static_cast<size_t>(threadIdx.x) * kScanItems;
    int32_t v[kScanItems];
    int32_t run = 0;
#pragma unroll
    for (int i = 0; i < kScanItems; ++i) {
        v[i] = base + i < count ? in[base + i] : 0;
        const int32_t x = v[i];
        v[i] = run;  // exclusive within the thread
        run += x;
    }
    // exclusive prefix of the thread totals: within the wave, then across waves
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t incl = run;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const int32_t y = __shfl_up(incl, k, 64);
        if (lane >= k) incl += y;
    }
    if (lane == 63) wave_tot[wave] = incl;
    __syncthreads();
    int32_t before = incl - run;
    for (int w = 0; w < wave; ++w) before += wave_tot[w];
#pragma unroll
    for (int i = 0; i < kScanItems; ++i)
        if (base + i < count) out[base + i] = before + v[i];
    return before + run;
}

// Exclusive scan, step 1: each block scans a tile of kScanTile counts into
// out (tile-local prefixes; out may be in) and writes the tile's total to
// sums[tile].
__global__ __launch_bounds__(kBlock) void scan_tiles_kernel(const int32_t* in, int32_t* out, int32_t* sums,
                                                            size_t count)
{
    __shared__ int32_t wave_tot[kBlock / 64];
    const size_t base = static_cast<size_t>(blockIdx.x) * kScanTile;
    const int32_t tot = block_exclusive_scan(in + base, out + base, count - base < kScanTile ? count - base : kScanTile,
                                             wave_tot);
    if (threadIdx.x == kBlock - 1) sums[blockIdx.x] = tot;
}

// Exclusive scan, step 2 (one block): sums[0..tiles) in place, total in sums[tiles].
__global__ __launch_bounds__(kBlock) void scan_sums_kernel(int32_t* sums, uint32_t tiles)
{
    __shared__ int32_t wave_tot[kBlock / 64];
    __shared__ int32_t carry_s;
    if (threadIdx.x == 0) carry_s = 0;
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (uint32_t c0 = 0; c0 < tiles; c0 += kBlock) {
        const uint32_t i = c0 + threadIdx.x;
        const int32_t x = i < tiles ? sums[i] : 0;
        int32_t incl = x;
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) {
            const int32_t y = __shfl_up(incl, k, 64);
            if (lane >= k) incl += y;
        }
        if (lane == 63) wave_tot[wave] = incl;
        __syncthreads();
        int32_t before = carry_s + incl - x;
        for (int w = 0; w < wave; ++w) before += wave_tot[w];
        if (i < tiles) sums[i] = before;
        __syncthreads();  // every thread has read carry_s and wave_tot
        if (threadIdx.x == kBlock - 1) carry_s = before + x;
        __syncthreads();
    }
    if (threadIdx.x == 0) sums[tiles] = carry_s;
}

// The inverse map from the scan: key k's entries start at
// offsets[k] = local[k] + pre[k / kScanTile] (local: tile-local exclusive
// prefixes of the counts, pre: exclusive prefixes of the tile totals, the
// grand total in pre[tiles]), and entry x goes to its key's start plus the
// slot the count recorded for it.  OWN_SCAN (tiles <= kScanTile): sums holds
// the raw tile totals and every block scans them into shared memory itself;
// otherwise scan_sums_kernel has turned sums into pre.
template <bool OWN_SCAN>
__global__ __launch_bounds__(kBlock) void bwd_fill_kernel(BwdParams p, const int32_t* local, const int32_t* sums,
                                                          uint32_t tiles, int32_t* offsets, int32_t* entries)
{
    __shared__ int32_t s_pre[OWN_SCAN ? kScanTile + 1 : 1];
    __shared__ int32_t wave_tot[kBlock / 64];
    const int32_t* pre = sums;
    if constexpr (OWN_SCAN) {
        const int32_t tot = block_exclusive_scan(sums, s_pre, tiles, wave_tot);
        if (threadIdx.x == kBlock - 1) s_pre[tiles] = tot;
        __syncthreads();
        pre = s_pre;
    }
    const size_t stride = static_cast<size_t>(gridDim.x) * kBlock;
    const size_t first = static_cast<size_t>(blockIdx.x) * kBlock + threadIdx.x;
    const size_t total = static_cast<size_t>(p.kappa) * p.n;
    for (size_t x = first; x < total; x += stride) {
        const uint32_t g = static_cast<uint32_t>(x % p.n);
        uint32_t s, rem;
        divmod(g, p.div_plane, s, rem);
        const size_t key = static_cast<size_t>(s) * p.nkeys + clamp_index(p.J[x], p.nkeys);
        entries[local[key] + pre[key / kScanTile] + p.slots[x]] = static_cast<int32_t>(x);
    }
    for (size_t k = first; k < p.keys_total; k += stride) offsets[k] = local[k] + pre[k / kScanTile];
    if (first == 0) offsets[p.keys_total] = pre[tiles];
}

// Neighbourhoods of up to this many rows are walked as one flat list.
constexpr int kMaxRows = 8;

// The entry ranges of the neighbourhood rows r0..r1 of key j: row i covers
// entries [lo[i], lo[i] + pre[i+1] - pre[i]); pre[] is the running count.
struct Neighbourhood {
    int lo[kMaxRows];
    int pre[kMaxRows + 1];
    int total;
};

__device__ __forceinline__ Neighbourhood load_neighbourhood(const int32_t* off, int Wk, int r0, int r1, int c0, int c1)
{
    Neighbourhood nb;
    nb.pre[0] = 0;
#pragma unroll
    for (int i = 0; i < kMaxRows; ++i) {
        int lo = 0, len = 0;
        if (r0 + i <= r1) {
            lo = off[(r0 + i) * Wk + c0];
            len = off[(r0 + i) * Wk + c1 + 1] - lo;
        }
        nb.lo[i] = lo;
        nb.pre[i + 1] = nb.pre[i] + len;
    }
    nb.total = nb.pre[kMaxRows];
    return nb;
}

// Entry slot of flat position v (0 <= v < total): the last row with pre <= v.
__device__ __forceinline__ int flat_slot(const Neighbourhood& nb, int v)
{
    int x = nb.lo[0] + v;
#pragma unroll
    for (int i = 1; i < kMaxRows; ++i)
        if (v >= nb.pre[i]) x = nb.lo[i] + (v - nb.pre[i]);
    return x;
}

struct KeyPos {
    uint32_t s, j, ju, jv;
    int r0, r1, c0, c1;
};

__device__ __forceinline__ KeyPos key_pos(const BwdParams& p, uint32_t kg)
{
    KeyPos k;
    divmod(kg, p.div_keys, k.s, k.j);
    divmod(k.j, p.div_wk, k.ju, k.jv);
    k.r0 = max(static_cast<int>(k.ju) - p.b, 0);
    k.r1 = min(static_cast<int>(k.ju) + p.b, p.Hk - 1);
    k.c0 = max(static_cast<int>(k.jv) - p.b, 0);
    k.c1 = min(static_cast<int>(k.jv) + p.b, p.Wk - 1);
    return k;
}

// Host: scan and fill, after the query kernel has counted.  counts: [N], scanned in place; sums: [tiles + 1].
inline hipError_t run_inverse(const BwdParams& p, int32_t* counts, int32_t* offsets, int32_t* sums, int32_t* entries,
                              hipStream_t stream, hipEvent_t start, hipEvent_t stop)
{
    const size_t N = p.keys_total, total = static_cast<size_t>(p.n) * p.kappa;
    const uint32_t tiles = static_cast<uint32_t>((N + kScanTile - 1) / kScanTile);
    hipError_t r;
    if ((r = launch(scan_tiles_kernel, tiles, stream, start, nullptr, static_cast<const int32_t*>(counts), counts, sums,
                    N)) != hipSuccess)
        return r;
    const uint32_t fill_blocks = stride_blocks(total > N ? total : N + 1);
    if (tiles <= static_cast<uint32_t>(kScanTile))
        return launch(bwd_fill_kernel<true>, fill_blocks, stream, nullptr, stop, p, static_cast<const int32_t*>(counts),
                      static_cast<const int32_t*>(sums), tiles, offsets, entries);
    if ((r = launch(scan_sums_kernel, 1u, stream, nullptr, nullptr, sums, tiles)) != hipSuccess) return r;
    return launch(bwd_fill_kernel<false>, fill_blocks, stream, nullptr, stop, p, static_cast<const int32_t*>(counts),
                  static_cast<const int32_t*>(sums), tiles, offsets, entries);
}

}  // namespace
}  // namespace scram
