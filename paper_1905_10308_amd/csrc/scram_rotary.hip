// Rotary positions on a grid: every channel pair of a row is turned by an
// angle that grows along one axis of the grid (time, height or width).
//
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = position * frequency
//
// The gradient is the rotation by -t.  One pass, read and written once: bound
// by memory (Q and K of 4 x 256 x 256, 64 channels, bf16: 134 MB in 24-28 us;
// 6 x 16 x 45 x 80, 100 channels, fp32: 276 MB in 56-61; a copy moves 5.15 TB/s).  The
// angles of a pixel's pairs are the same in every slice and tensor, so a thread
// computes those of its pairs once and walks the slices.

#include <algorithm>

#include "scram_rows.h"

namespace scram {
namespace {

constexpr int kMaxPairs = 128;

struct RotaryParams {
    const void* src[4];
    void* dst[4];
    uint32_t slices[4];
    int count;
    uint32_t most;          // most slices of a tensor
    uint32_t total;         // work items of one slice
    int T, H, W;
    int d, group, pairs, chunks;  // row width, channels and pairs of a group, work items of a group
    Div div_row, div_chunks, div_w, div_h;
    int axis1, axis2;       // first pair of the height, of the width
    const int32_t* origin;
    int per_slice;          // an origin per slice
    int first[3];
    uint32_t per_block;     // slices per block row
    uint64_t turn[kMaxPairs];  // turns per step, as a fraction of 2^64 (negated for the inverse)
};

// cos and sin of a whole turn's fraction x / 2^64.  The nearest quarter turn
// is taken off exactly; the rest, at most an eighth of a turn, goes through the
// Taylor series of sin and cos (first left-out terms below 2e-9 and 2e-9 there).
__device__ __forceinline__ void turn_cos_sin(uint64_t x, float& c, float& s)
{
    const uint32_t hi = static_cast<uint32_t>(x >> 32), lo = static_cast<uint32_t>(x);
    const uint32_t quarter = (hi + 0x20000000u) >> 30;
    const int32_t rest = static_cast<int32_t>(hi - (quarter << 30));
    const float a = fmaf(static_cast<float>(lo), 0x1p-32f, static_cast<float>(rest)) * 1.4629180792671596e-9f;  // 2 pi / 2^32
    const float z = a * a;
    float ps = fmaf(z, 1.f / 362880.f, -1.f / 5040.f);
    ps = fmaf(z, ps, 1.f / 120.f);
    ps = fmaf(z, ps, -1.f / 6.f);
    const float sn = fmaf(a * z, ps, a);
    float pc = fmaf(z, -1.f / 3628800.f, 1.f / 40320.f);
    pc = fmaf(z, pc, -1.f / 720.f);
    pc = fmaf(z, pc, 1.f / 24.f);
    pc = fmaf(z, pc, -0.5f);
    const float cs = fmaf(z, pc, 1.f);
    const float x0 = quarter & 1u ? sn : cs, x1 = quarter & 1u ? cs : sn;
    c = ((quarter + 1u) & 2u) ? -x0 : x0;
    s = quarter & 2u ? -x1 : x1;
}

// A thread takes V pairs of one group of one pixel's row, two vectors of V
// channels (the pairs' first and second channels, or 2 V neighbouring ones when
// INTER), or one vector of the channels that are not turned; in the slices of
// its block row.  MANY: a slice has fewer work items than half a block's threads,
// and several threads of an item take those slices by turns (the form's cost
// where a thread takes them all: Q and K of 4 x 256 x 256, bf16, 30 us, without it 28).
template <typename T, int V, bool INTER, bool MANY>
__global__ __launch_bounds__(kBlock) void rotary_kernel(RotaryParams p)
{
    using Vec = vec<T, V>;
    const uint32_t i = blockIdx.x * (MANY ? blockDim.x : kBlock) + threadIdx.x;
    if (i >= p.total) return;
    uint32_t pixel, in_row, grp, chunk;
    divmod(i, p.div_row, pixel, in_row);
    divmod(in_row, p.div_chunks, grp, chunk);
    const int pair0 = static_cast<int>(chunk) * V;
    const bool turned = pair0 < p.pairs;
    int at0, at1;  // channels of the two vectors
    if (turned) {
        at0 = INTER ? 2 * pair0 : pair0;
        at1 = INTER ? 2 * pair0 + V : pair0 + p.pairs;
    } else {
        at0 = at1 = pair0 + p.pairs;  // pair0 = pairs, pairs + V, ...: channels 2 pairs ...
    }
    const size_t row = static_cast<size_t>(pixel) * p.d + static_cast<size_t>(grp) * p.group;
    const size_t slice = static_cast<size_t>(p.T) * p.H * p.W * p.d;
    uint32_t tt, yy, xx, rest;
    divmod(pixel, p.div_w, rest, xx);
    divmod(rest, p.div_h, tt, yy);
    float cs[V], sn[V];
    auto angles = [&](int t0, int y0, int x0) {
        const int64_t pos[3] = {int64_t(t0) + tt, int64_t(y0) + yy, int64_t(x0) + xx};
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int k = min(pair0 + j, p.pairs - 1);
            const int64_t at = k >= p.axis2 ? pos[2] : k >= p.axis1 ? pos[1] : pos[0];
            turn_cos_sin(static_cast<uint64_t>(at) * p.turn[k], cs[j], sn[j]);
        }
    };
    if (turned && !p.per_slice) {
        if (p.origin != nullptr)
            angles(p.origin[0], p.origin[1], p.origin[2]);
        else
            angles(p.first[0], p.first[1], p.first[2]);
    }
    const uint32_t s0 = blockIdx.y * p.per_block, s1 = s0 + min(p.per_block, p.most - s0);
    for (uint32_t s = s0 + (MANY ? threadIdx.y : 0u); s < s1; s += MANY ? blockDim.y : 1u) {
        if (turned && p.per_slice) {
            const int32_t* const at = p.origin + 3 * static_cast<size_t>(s);
            angles(at[0], at[1], at[2]);
        }
        for (int t = 0; t < p.count; ++t) {
            if (s >= p.slices[t]) continue;
            const T* const from = static_cast<const T*>(p.src[t]) + s * slice + row;
            T* const to = static_cast<T*>(p.dst[t]) + s * slice + row;
            Vec a = *reinterpret_cast<const Vec*>(from + at0);
            if (!turned) {
                *reinterpret_cast<Vec*>(to + at0) = a;
                continue;
            }
            Vec b = *reinterpret_cast<const Vec*>(from + at1);
            T in[2 * V], out[2 * V];
#pragma unroll
            for (int j = 0; j < V; ++j) in[j] = a[j], in[V + j] = b[j];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int i0 = INTER ? 2 * j : j, i1 = INTER ? 2 * j + 1 : V + j;
                const float x = to_float(in[i0]), y = to_float(in[i1]);
                out[i0] = from_float<T>(fmaf(x, cs[j], -(y * sn[j])));
                out[i1] = from_float<T>(fmaf(x, sn[j], y * cs[j]));
            }
#pragma unroll
            for (int j = 0; j < V; ++j) a[j] = out[j], b[j] = out[V + j];
            *reinterpret_cast<Vec*>(to + at0) = a;
            *reinterpret_cast<Vec*>(to + at1) = b;
        }
    }
}

// Channels per vector: the most, up to 16 bytes, that divide the turned pairs and the group.  (Whole vectors of 16 bytes with a
// last one in pieces were slower: 6 x 16 x 45 x 80, 46 pairs of 100 fp32 channels, vectors of 8 bytes 56 us, 16 with a rest 65.
// An odd number of pairs goes a channel at a time: two tensors of 4 x 256 x 256, bf16, 23 pairs of 46 channels 27 us, 18.7 at a
// copy's rate; 24 of 48, in vectors of 16 bytes, 21 and 19.5.)
int rotary_vector(int elem, const RotaryCall& c)
{
    const int group = c.d / c.groups, pairs = c.pairs[0] + c.pairs[1] + c.pairs[2];
    int v = 16 / elem;
    while (group % v || pairs % v) v /= 2;
    return v;
}

}  // namespace

uint64_t rotary_items(int dtype, const RotaryCall& c)
{
    const int group = c.d / c.groups, pairs = c.pairs[0] + c.pairs[1] + c.pairs[2];
    return uint64_t(c.T) * c.H * c.W * c.groups * ((group - pairs) / rotary_vector(dtype == SCRAM_BF16 ? 2 : 4, c));
}

hipError_t launch_rotary(int dtype, const RotaryCall& c, hipStream_t stream)
{
    const int v = rotary_vector(dtype == SCRAM_BF16 ? 2 : 4, c);
    RotaryParams p{};
    p.count = c.count;
    for (int t = 0; t < c.count; ++t) {
        p.src[t] = c.src[t];
        p.dst[t] = c.dst[t];
        p.slices[t] = c.slices[t];
        p.most = p.slices[t] > p.most ? p.slices[t] : p.most;
    }
    p.T = c.T;
    p.H = c.H;
    p.W = c.W;
    p.d = c.d;
    p.group = c.d / c.groups;
    p.pairs = c.pairs[0] + c.pairs[1] + c.pairs[2];
    p.chunks = (p.group - p.pairs) / v;
    p.total = static_cast<uint32_t>(rotary_items(dtype, c));
    p.div_row = make_div(static_cast<uint32_t>(c.groups) * p.chunks);
    p.div_chunks = make_div(p.chunks);
    p.div_w = make_div(c.W);
    p.div_h = make_div(c.H);
    p.axis1 = c.pairs[0];
    p.axis2 = c.pairs[0] + c.pairs[1];
    p.origin = c.origin;
    p.per_slice = c.origin_rows > 1 ? 1 : 0;
    for (int a = 0; a < 3; ++a) p.first[a] = c.first[a];
    for (int k = 0; k < p.pairs; ++k) {
        // whole turns do not count: the fraction, rounded to 2^-64 turns (of the value without its sign: a small negative one
        // would lose its low bits in 1 - x)
        const double turns = fabs(c.freq[k]) / 6.283185307179586476925;
        const uint64_t f = static_cast<uint64_t>(rint(ldexp(turns - floor(turns), 64)));  // (less than 1 by 2^-53 at least)
        p.turn[k] = c.inverse != (c.freq[k] < 0.0) ? 0u - f : f;
    }
    dim3 threads(kBlock, 1);
    while (threads.x / 2 >= p.total) threads.x /= 2, threads.y *= 2;
    const uint32_t blocks = (p.total + threads.x - 1) / threads.x;
    const uint32_t want = (2048 + blocks - 1) / blocks;  // block rows: enough blocks to fill the machine
    p.per_block = std::max((p.most + want - 1) / want, threads.y);
    const dim3 grid(blocks, (p.most + p.per_block - 1) / p.per_block);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, threads, 0, stream, p);
        return hipGetLastError();
    };
    auto with = [&](auto type, auto width) {
        using T = decltype(type);
        constexpr int V = decltype(width)::value;
        if (threads.y > 1) return c.interleaved ? go(rotary_kernel<T, V, true, true>) : go(rotary_kernel<T, V, false, true>);
        return c.interleaved ? go(rotary_kernel<T, V, true, false>) : go(rotary_kernel<T, V, false, false>);
    };
    using std::integral_constant;
    if (dtype == SCRAM_BF16) {
        if (v == 8) return with(uint16_t{}, integral_constant<int, 8>{});
        if (v == 4) return with(uint16_t{}, integral_constant<int, 4>{});
        if (v == 2) return with(uint16_t{}, integral_constant<int, 2>{});
        return with(uint16_t{}, integral_constant<int, 1>{});
    }
    if (v == 4) return with(float{}, integral_constant<int, 4>{});
    if (v == 2) return with(float{}, integral_constant<int, 2>{});
    return with(float{}, integral_constant<int, 1>{});
}

}  // namespace scram
