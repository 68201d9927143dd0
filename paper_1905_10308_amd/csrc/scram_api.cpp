// C-ABI front end of the SCRAM library: argument validation (host only, no
// HIP call before every check has passed), ping-pong buffer planning for the
// Jacobi sweeps, and the launches.  The contract is documented in scram.h.

#include <math.h>
#include <stdint.h>
#include <string.h>

#include <hip/hip_runtime.h>

#include "scram.h"
#include "scram_launch.h"

namespace {

constexpr int64_t kMaxSide = int64_t(1) << 30;
constexpr int64_t kMaxCount = int64_t(1) << 31;
constexpr uint64_t kMaxBlocks = 0xFFFFFFFFull / 256;  // one dispatch: at most 2^32 - 1 work-items

size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

struct Range {
    uintptr_t lo, hi;  // [lo, hi)
};

Range range(const void* p, size_t bytes)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    return Range{a, a + bytes};
}

bool overlap(const Range& a, const Range& b)
{
    return a.lo != a.hi && b.lo != b.hi && a.lo < b.hi && b.lo < a.hi;
}

bool supported_width(int d) { return d == 16 || d == 32 || d == 64 || d == 128; }

size_t elem_bytes(int dtype) { return dtype == SCRAM_BF16 ? 2 : 4; }

int check_grid(int S, int Hq, int Wq, int Hk, int Wk)
{
    if (S <= 0 || Hq <= 0 || Wq <= 0 || Hk <= 0 || Wk <= 0) return SCRAM_ERR_SHAPE;
    if (Hq > kMaxSide || Wq > kMaxSide || Hk > kMaxSide || Wk > kMaxSide) return SCRAM_ERR_SHAPE;
    if (int64_t(S) * Hq * Wq >= kMaxCount || int64_t(Hk) * Wk >= kMaxCount) return SCRAM_ERR_SHAPE;
    return SCRAM_OK;
}

int check_type(int dtype, int d)
{
    if (dtype != SCRAM_F32 && dtype != SCRAM_BF16) return SCRAM_ERR_UNSUPPORTED;
    if (!supported_width(d)) return SCRAM_ERR_UNSUPPORTED;
    return SCRAM_OK;
}

// Arguments that the differential attend and its gradients share, but for pointers.
int check_differential(int dtype, const scram::Grid& g, int kappa, int dv, int window, float scale, uint32_t flags, int first,
                       const int32_t* origin)
{
    int rc = check_grid(g.S, g.Hq, g.Wq, g.Hk, g.Wk);
    if (rc) return rc;
    if (window < 1 || window % 2 == 0 || window > 32767) return SCRAM_ERR_SHAPE;
    if (kappa < 1 || kappa > SCRAM_MAX_KAPPA) return SCRAM_ERR_SHAPE;
    if (!isfinite(scale)) return SCRAM_ERR_SHAPE;
    if ((rc = check_type(dtype, g.d))) return rc;
    if (dv != g.d) return SCRAM_ERR_UNSUPPORTED;
    if (flags & ~uint32_t(SCRAM_CAUSAL)) return SCRAM_ERR_UNSUPPORTED;
    const int64_t nq = int64_t(g.Hq) * g.Wq, nk = int64_t(g.Hk) * g.Wk;
    if (!(flags & SCRAM_CAUSAL)) return first != 0 || origin ? SCRAM_ERR_SHAPE : SCRAM_OK;
    // the queries are a run of the keys' raster: whole rows, or a part of it as one row
    if (g.Hq != 1 && g.Wq != g.Wk) return SCRAM_ERR_SHAPE;
    if (first < 0 || (origin && first != 0) || first + nq > nk) return SCRAM_ERR_SHAPE;
    return SCRAM_OK;
}

// The kernels count rows in steps of up to 512: a step behind the last row is a number too.
int check_dense_grid(int S, int key_slices, int Hq, int Wq, int Hk, int Wk)
{
    const int rc = check_grid(S, Hq, Wq, Hk, Wk);
    if (rc) return rc;
    const int64_t most = kMaxCount - 1024;
    if (int64_t(S) * Hq * Wq >= most || int64_t(Hk) * Wk >= most) return SCRAM_ERR_SHAPE;
    return key_slices < 1 || S % key_slices ? SCRAM_ERR_SHAPE : SCRAM_OK;
}

// Arguments that the dense attend and its gradients share, but for pointers.
int check_dense(int dtype, const scram::DenseCall& c, int dv, uint32_t flags)
{
    const scram::Grid& g = c.g;
    int rc = check_dense_grid(g.S, c.key_slices, g.Hq, g.Wq, g.Hk, g.Wk);
    if (rc) return rc;
    if (!isfinite(c.scale)) return SCRAM_ERR_SHAPE;
    if ((rc = check_type(dtype, g.d))) return rc;
    if (dv != g.d) return SCRAM_ERR_UNSUPPORTED;
    if (flags & ~uint32_t(SCRAM_CAUSAL)) return SCRAM_ERR_UNSUPPORTED;
    const int64_t nq = int64_t(g.Hq) * g.Wq, nk = int64_t(g.Hk) * g.Wk;
    if (c.bias) {
        if (c.bias_rows < 1 || g.S % c.bias_rows) return SCRAM_ERR_SHAPE;
        if ((2 * int64_t(g.Hk) - 1) * (2 * int64_t(g.Wk) - 1) >= kMaxCount) return SCRAM_ERR_SHAPE;
        if (scram::dense_bias_window(g.Hk, g.Wk) > scram::kBiasWindowMost) return SCRAM_ERR_SHAPE;
    }
    if (!(flags & SCRAM_CAUSAL) && !c.bias) return c.first != 0 || c.origin ? SCRAM_ERR_SHAPE : SCRAM_OK;
    // the queries are a run of the keys' raster: whole rows, or a part of it as one row
    if (g.Hq != 1 && g.Wq != g.Wk) return SCRAM_ERR_SHAPE;
    if (c.first < 0 || (c.origin && c.first != 0) || c.first + nq > nk) return SCRAM_ERR_SHAPE;
    return SCRAM_OK;
}

scram::DenseCall dense_call(const void* Q, const void* K, const void* V, const void* bias, int bias_rows, const int32_t* lengths,
                            int S, int key_slices, int Hq, int Wq, int Hk, int Wk, int d, float scale, uint32_t flags, int first,
                            const int32_t* origin)
{
    return scram::DenseCall{Q,     K,      V, bias, bias ? bias_rows : 0, lengths, scram::Grid{S, Hq, Wq, Hk, Wk, d}, key_slices, scale,
                            (flags & SCRAM_CAUSAL) != 0, first, origin};
}

bool fits(const scram::DenseNeeds& n) { return n.blocks <= kMaxBlocks && n.lds <= scram::kLdsMost; }

size_t bias_bytes(const scram::DenseCall& c, size_t eb)
{
    return c.bias ? size_t(c.bias_rows) * (2 * size_t(c.g.Hk) - 1) * (2 * size_t(c.g.Wk) - 1) * eb : 0;
}

int check_relative(int dtype, int heads, int H, int W, const int* edges_y, int my, const int* edges_x, int mx)
{
    if (heads < 1 || H < 1 || W < 1 || H > kMaxSide || W > kMaxSide) return SCRAM_ERR_SHAPE;
    const int64_t plane = (2 * int64_t(H) - 1) * (2 * int64_t(W) - 1);
    if (plane >= kMaxCount || heads >= (int64_t(1) << 40) / plane) return SCRAM_ERR_SHAPE;
    if (my < 0 || mx < 0 || my > SCRAM_BIAS_MAX_EDGES || mx > SCRAM_BIAS_MAX_EDGES) return SCRAM_ERR_SHAPE;
    if ((my && !edges_y) || (mx && !edges_x)) return SCRAM_ERR_NULL;
    for (int k = 0; k < my; ++k)
        if (edges_y[k] <= (k ? edges_y[k - 1] : 0)) return SCRAM_ERR_SHAPE;
    for (int k = 0; k < mx; ++k)
        if (edges_x[k] <= (k ? edges_x[k - 1] : 0)) return SCRAM_ERR_SHAPE;
    return dtype == SCRAM_F32 || dtype == SCRAM_BF16 ? SCRAM_OK : SCRAM_ERR_UNSUPPORTED;
}

int check_group(int64_t images, int64_t pixels, int channels, int groups, int dtype, int weight_dtype, int activation)
{
    const int64_t most = int64_t(1) << 40;
    if (images < 1 || pixels < 1 || channels < 1 || channels > scram::kNormMaxChannels) return SCRAM_ERR_SHAPE;
    if (images >= most || pixels >= most / images || images * pixels >= most / channels) return SCRAM_ERR_SHAPE;
    if (groups < 1 || channels % groups || images >= kMaxCount / groups) return SCRAM_ERR_SHAPE;
    if (dtype != SCRAM_F32 && dtype != SCRAM_BF16) return SCRAM_ERR_UNSUPPORTED;
    if (weight_dtype != dtype && weight_dtype != SCRAM_F32) return SCRAM_ERR_UNSUPPORTED;
    if (activation != SCRAM_ACT_NONE && activation != SCRAM_ACT_SILU) return SCRAM_ERR_UNSUPPORTED;
    return SCRAM_OK;
}

int check_norm(int64_t rows, int channels, int dtype, int weight_dtype)
{
    if (rows < 1 || rows >= (int64_t(1) << 40) || channels < 1 || channels > scram::kNormMaxChannels) return SCRAM_ERR_SHAPE;
    if (dtype != SCRAM_F32 && dtype != SCRAM_BF16) return SCRAM_ERR_UNSUPPORTED;
    if (weight_dtype != dtype && weight_dtype != SCRAM_F32) return SCRAM_ERR_UNSUPPORTED;
    return SCRAM_OK;
}

}  // namespace

namespace scram {

// Every check of scram_patchmatch's arguments, on the host (no HIP call).  A
// null workspace is the library's own scratch (scram_patchmatch_noalloc):
// its presence, size and overlap are then not checked here.
int patchmatch_check(const void* Q, const void* K, int dtype, int S, int Hq, int Wq, int Hk, int Wk, int d,
                     int iters, const int32_t* init, const float* init_score, int t0, uint32_t flags,
                     const int32_t* prev, int n_prev, int sep, const int32_t* argmax_out, const float* score_out,
                     const void* workspace, size_t workspace_bytes)
{
    if (!Q || !K || !argmax_out) return SCRAM_ERR_NULL;
    if (n_prev > 0 && !prev) return SCRAM_ERR_NULL;
    int rc = check_grid(S, Hq, Wq, Hk, Wk);
    if (rc) return rc;
    if (iters < 0 || t0 < 1 || int64_t(t0) + iters > int64_t(0xFFFFFFFFu)) return SCRAM_ERR_SHAPE;
    if (n_prev < 0 || n_prev > SCRAM_MAX_PREV || sep < 1) return SCRAM_ERR_SHAPE;
    if ((rc = check_type(dtype, d))) return rc;
    if (patchmatch_max_blocks(dtype, Grid{S, Hq, Wq, Hk, Wk, d}) > kMaxBlocks) return SCRAM_ERR_SHAPE;
    if (flags & ~uint32_t(SCRAM_PM_NO_PROPAGATION | SCRAM_PM_NO_RANDOM_SEARCH | SCRAM_CAUSAL))
        return SCRAM_ERR_UNSUPPORTED;
    const bool causal = (flags & SCRAM_CAUSAL) != 0;
    if (causal && (Hq != Hk || Wq != Wk)) return SCRAM_ERR_SHAPE;
    if (!init) init_score = nullptr;
    if (n_prev == 0) prev = nullptr;
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(argmax_out, 4) || (workspace && !aligned(workspace, 256)) ||
        (score_out && !aligned(score_out, 4)) || (init && !aligned(init, 4)) ||
        (init_score && !aligned(init_score, 4)) || (prev && !aligned(prev, 4)))
        return SCRAM_ERR_ALIGN;
    const size_t n = size_t(S) * Hq * Wq;
    const size_t need = scram_patchmatch_workspace_bytes(S, Hq, Wq);
    if (workspace && workspace_bytes < need) return SCRAM_ERR_WORKSPACE;

    const size_t eb = elem_bytes(dtype);
    const Range rQ = range(Q, n * d * eb), rK = range(K, size_t(S) * Hk * Wk * d * eb);
    const Range rJ = range(argmax_out, 4 * n), rW = workspace ? range(workspace, need) : Range{0, 0};
    const Range rS = score_out ? range(score_out, 4 * n) : Range{0, 0};
    const Range rI = init ? range(init, 4 * n) : Range{0, 0};
    const Range rIS = init_score ? range(init_score, 4 * n) : Range{0, 0};
    const Range rP = prev ? range(prev, 4 * n * size_t(n_prev)) : Range{0, 0};
    for (const Range& out : {rJ, rS, rW}) {
        for (const Range& other : {rQ, rK, rI, rIS, rP}) {
            if (overlap(out, other)) return SCRAM_ERR_ALIAS;
        }
    }
    if (overlap(rJ, rS) || overlap(rJ, rW) || overlap(rS, rW)) return SCRAM_ERR_ALIAS;
    return SCRAM_OK;
}

}  // namespace scram

extern "C" {

size_t scram_patchmatch_workspace_bytes(int S, int Hq, int Wq)
{
    if (S <= 0 || Hq <= 0 || Wq <= 0) return 0;
    const size_t n = size_t(S) * size_t(Hq) * size_t(Wq);
    return 3 * round256(4 * n);
}

int scram_patchmatch(const void* Q, const void* K, int dtype, int S, int Hq, int Wq, int Hk, int Wk,
                     int d, int iters, uint64_t seed, const int32_t* init, const float* init_score,
                     int t0, uint32_t flags, const int32_t* prev, int n_prev, int sep, int32_t* argmax_out,
                     float* score_out, void* workspace, size_t workspace_bytes, hipEvent_t* events,
                     hipStream_t stream)
{
    // ---- validation (no HIP call above this line) ----
    if (Q && K && argmax_out && !(n_prev > 0 && !prev) && !workspace) return SCRAM_ERR_WORKSPACE;
    int rc = scram::patchmatch_check(Q, K, dtype, S, Hq, Wq, Hk, Wk, d, iters, init, init_score, t0, flags, prev,
                                     n_prev, sep, argmax_out, score_out, workspace, workspace_bytes);
    if (rc) return rc;
    const bool causal = (flags & SCRAM_CAUSAL) != 0;
    if (!init) init_score = nullptr;
    if (n_prev == 0) prev = nullptr;
    const size_t n = size_t(S) * Hq * Wq;

    // ---- plan the ping-pong buffers ----
    // The map after sweep k (k = 0 is the initial map) lives in buffer
    // (iters - k) % 2, so the last sweep writes buffer 0 = the caller's
    // outputs and no sweep reads the buffer it writes.
    char* ws = static_cast<char*>(workspace);
    int32_t* Jbuf[2] = {argmax_out, reinterpret_cast<int32_t*>(ws)};
    float* s_ws0 = reinterpret_cast<float*>(ws + round256(4 * n));
    float* s_ws1 = reinterpret_cast<float*>(ws + 2 * round256(4 * n));
    float* sbuf[2] = {score_out ? score_out : s_ws0, s_ws1};
    const scram::Grid grid{S, Hq, Wq, Hk, Wk, d};
    const scram::RunSpec run{prev, n_prev, sep, causal};
    flags &= ~uint32_t(SCRAM_CAUSAL);

    const int p0 = iters % 2;
    const int32_t* Jcur;
    const float* scur;
    hipEvent_t* ev = events;  // 2 per launch: start, stop
    hipError_t e = hipSuccess;
    if (init) {
        Jcur = init;
        if (init_score) {
            scur = init_score;
            if (ev) {  // nothing to launch: the first pair brackets no work
                e = hipEventRecord(ev[0], stream);
                if (e == hipSuccess) e = hipEventRecord(ev[1], stream);
            }
        } else {
            e = scram::launch_pm_init(dtype, Q, K, grid, seed, run, init, nullptr, sbuf[p0], stream,
                                      ev ? ev[0] : nullptr, ev ? ev[1] : nullptr);
            scur = sbuf[p0];
        }
        if (e == hipSuccess && iters == 0) {
            e = hipMemcpyAsync(argmax_out, init, 4 * n, hipMemcpyDeviceToDevice, stream);
            if (e == hipSuccess && score_out && init_score)
                e = hipMemcpyAsync(score_out, init_score, 4 * n, hipMemcpyDeviceToDevice, stream);
        }
    } else if (iters > 0 && flags == 0) {
        // the first sweep recomputes the random initial field itself: no
        // init launch, and the init's event pair brackets no work
        Jcur = nullptr;
        scur = nullptr;
        if (ev) {
            e = hipEventRecord(ev[0], stream);
            if (e == hipSuccess) e = hipEventRecord(ev[1], stream);
        }
    } else {
        e = scram::launch_pm_init(dtype, Q, K, grid, seed, run, nullptr, Jbuf[p0], sbuf[p0], stream,
                                  ev ? ev[0] : nullptr, ev ? ev[1] : nullptr);
        Jcur = Jbuf[p0];
        scur = sbuf[p0];
    }
    for (int k = 1; k <= iters && e == hipSuccess; ++k) {
        const int pk = (iters - k) % 2;
        // maps between two sweeps of this call carry the stable-entry mark;
        // the caller's init and the final map do not
        e = scram::launch_pm_iter(dtype, Q, K, grid, seed, run, uint32_t(t0 + k - 1), flags, Jcur, scur, k > 1,
                                  k < iters, Jbuf[pk], sbuf[pk], stream, ev ? ev[2 * k] : nullptr,
                                  ev ? ev[2 * k + 1] : nullptr);
        Jcur = Jbuf[pk];
        scur = sbuf[pk];
    }
    return e == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

int scram_sparse_attend(const void* Q, const void* K, const void* V, int dtype, const int32_t* argmax, int kappa,
                        int S, int Hq, int Wq, int Hk, int Wk, int d, int dv, int window, float scale,
                        uint32_t flags, void* out, hipEvent_t* events, hipStream_t stream)
{
    if (!Q || !K || !V || !argmax || !out) return SCRAM_ERR_NULL;
    int rc = check_grid(S, Hq, Wq, Hk, Wk);
    if (rc) return rc;
    if (window < 1 || window % 2 == 0 || window > 32767) return SCRAM_ERR_SHAPE;
    if (kappa < 1 || kappa > SCRAM_MAX_KAPPA) return SCRAM_ERR_SHAPE;
    if (!isfinite(scale)) return SCRAM_ERR_SHAPE;
    if ((rc = check_type(dtype, d))) return rc;
    if (scram::attend_max_blocks(dtype, scram::Grid{S, Hq, Wq, Hk, Wk, d}) > kMaxBlocks) return SCRAM_ERR_SHAPE;
    if (dv != d) return SCRAM_ERR_UNSUPPORTED;
    if (flags & ~uint32_t(SCRAM_CAUSAL)) return SCRAM_ERR_UNSUPPORTED;
    const bool causal = (flags & SCRAM_CAUSAL) != 0;
    if (causal && (Hq != Hk || Wq != Wk)) return SCRAM_ERR_SHAPE;
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(out, 16) || !aligned(argmax, 4))
        return SCRAM_ERR_ALIGN;
    const size_t n = size_t(S) * Hq * Wq, eb = elem_bytes(dtype);
    const Range rO = range(out, n * dv * eb);
    for (const Range& other : {range(Q, n * d * eb), range(K, size_t(S) * Hk * Wk * d * eb),
                               range(V, size_t(S) * Hk * Wk * dv * eb), range(argmax, 4 * n * size_t(kappa))}) {
        if (overlap(rO, other)) return SCRAM_ERR_ALIAS;
    }
    const scram::Grid grid{S, Hq, Wq, Hk, Wk, d};
    const hipError_t e = scram::launch_attend(dtype, Q, K, V, argmax, kappa, grid, window, scale, causal, out, stream,
                                              events ? events[0] : nullptr, events ? events[1] : nullptr);
    return e == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

size_t scram_sparse_attend_backward_workspace_bytes(int S, int Hq, int Wq, int Hk, int Wk, int d, int dtype,
                                                    int kappa)
{
    if (check_grid(S, Hq, Wq, Hk, Wk) || kappa < 1 || kappa > SCRAM_MAX_KAPPA || check_type(dtype, d)) return 0;
    return scram::attend_backward_workspace_bytes(S, Hq, Wq, Hk, Wk, d, dtype, kappa);
}

int scram_sparse_attend_backward(const void* Q, const void* K, const void* V, int dtype, const int32_t* argmax,
                                 int kappa, int S, int Hq, int Wq, int Hk, int Wk, int d, int dv, int window,
                                 float scale, uint32_t flags, const void* dO, float* dQ, float* dK, float* dV,
                                 void* workspace, size_t workspace_bytes, hipEvent_t* events, hipStream_t stream)
{
    if (!Q || !K || !V || !argmax || !dO || !dQ || !dK || !dV) return SCRAM_ERR_NULL;
    int rc = check_grid(S, Hq, Wq, Hk, Wk);
    if (rc) return rc;
    // the inverse map codes (match, query) pairs as e * n + i in an int32, and
    // keys are numbered across slices (s * Hk * Wk + j)
    if (int64_t(S) * Hq * Wq * (kappa < 1 ? 1 : kappa) >= kMaxCount) return SCRAM_ERR_SHAPE;
    if (int64_t(S) * Hk * Wk >= kMaxCount) return SCRAM_ERR_SHAPE;
    if (window < 1 || window % 2 == 0 || window > 32767) return SCRAM_ERR_SHAPE;
    if (kappa < 1 || kappa > SCRAM_MAX_KAPPA) return SCRAM_ERR_SHAPE;
    if (!isfinite(scale)) return SCRAM_ERR_SHAPE;
    if ((rc = check_type(dtype, d))) return rc;
    if (scram::attend_backward_max_blocks(dtype, scram::Grid{S, Hq, Wq, Hk, Wk, d}, kappa) > kMaxBlocks)
        return SCRAM_ERR_SHAPE;
    if (dv != d) return SCRAM_ERR_UNSUPPORTED;
    if (flags & ~uint32_t(SCRAM_CAUSAL)) return SCRAM_ERR_UNSUPPORTED;
    const bool causal = (flags & SCRAM_CAUSAL) != 0;
    if (causal && (Hq != Hk || Wq != Wk)) return SCRAM_ERR_SHAPE;
    if (!workspace) return SCRAM_ERR_WORKSPACE;
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(dO, 16) || !aligned(argmax, 4) ||
        !aligned(dQ, 16) || !aligned(dK, 16) || !aligned(dV, 16) || !aligned(workspace, 256))
        return SCRAM_ERR_ALIGN;
    const size_t need = scram::attend_backward_workspace_bytes(S, Hq, Wq, Hk, Wk, d, dtype, kappa);
    if (workspace_bytes < need) return SCRAM_ERR_WORKSPACE;
    const size_t n = size_t(S) * Hq * Wq, nk = size_t(S) * Hk * Wk, eb = elem_bytes(dtype);
    const Range rQ = range(dQ, 4 * n * d), rK = range(dK, 4 * nk * d), rV = range(dV, 4 * nk * dv);
    const Range rW = range(workspace, need);
    for (const Range& o : {rQ, rK, rV, rW}) {
        for (const Range& other : {range(Q, n * d * eb), range(K, nk * d * eb), range(V, nk * dv * eb),
                                   range(argmax, 4 * n * size_t(kappa)), range(dO, n * dv * eb)}) {
            if (overlap(o, other)) return SCRAM_ERR_ALIAS;
        }
    }
    if (overlap(rQ, rK) || overlap(rQ, rV) || overlap(rK, rV) || overlap(rW, rQ) || overlap(rW, rK) ||
        overlap(rW, rV))
        return SCRAM_ERR_ALIAS;
    const scram::Grid grid{S, Hq, Wq, Hk, Wk, d};
    const hipError_t e = scram::launch_attend_backward(dtype, Q, K, V, argmax, kappa, grid, window, scale, causal, dO,
                                                       dQ, dK, dV, workspace, stream, events);
    return e == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

int scram_snis_attend(const void* Q, const void* K, const void* V, int dtype, const int32_t* modes, int kappa, int S,
                      int Hq, int Wq, int Hk, int Wk, int d, int dv, int samples, float alpha, int radius, float scale,
                      uint64_t seed, uint32_t flags, void* out, float* ess_out, float* var_out, hipEvent_t* events,
                      hipStream_t stream)
{
    if (!Q || !K || !V || !modes || !out) return SCRAM_ERR_NULL;
    int rc = check_grid(S, Hq, Wq, Hk, Wk);
    if (rc) return rc;
    if (kappa < 1 || kappa > SCRAM_MAX_KAPPA) return SCRAM_ERR_SHAPE;
    if (samples < 1 || samples > SCRAM_SNIS_MAX_SAMPLES) return SCRAM_ERR_SHAPE;
    if (!(alpha >= 0.f && alpha <= 1.f)) return SCRAM_ERR_SHAPE;  // also rejects NaN
    if (radius < 0 || radius > SCRAM_SNIS_MAX_RADIUS) return SCRAM_ERR_SHAPE;
    if (!isfinite(scale)) return SCRAM_ERR_SHAPE;
    if ((rc = check_type(dtype, d))) return rc;
    if (scram::snis_max_blocks(dtype, scram::Grid{S, Hq, Wq, Hk, Wk, d}) > kMaxBlocks) return SCRAM_ERR_SHAPE;
    if (dv != d) return SCRAM_ERR_UNSUPPORTED;
    if (flags & ~uint32_t(SCRAM_CAUSAL)) return SCRAM_ERR_UNSUPPORTED;
    const bool causal = (flags & SCRAM_CAUSAL) != 0;
    if (causal && (Hq != Hk || Wq != Wk)) return SCRAM_ERR_SHAPE;
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(out, 16) || !aligned(modes, 4) ||
        (ess_out && !aligned(ess_out, 4)) || (var_out && !aligned(var_out, 16)))
        return SCRAM_ERR_ALIGN;
    const size_t n = size_t(S) * Hq * Wq, eb = elem_bytes(dtype);
    const Range rO = range(out, n * dv * eb);
    const Range rE = ess_out ? range(ess_out, 4 * n) : Range{0, 0};
    const Range rV = var_out ? range(var_out, 4 * n * dv) : Range{0, 0};
    for (const Range& o : {rO, rE, rV}) {
        for (const Range& other : {range(Q, n * d * eb), range(K, size_t(S) * Hk * Wk * d * eb),
                                   range(V, size_t(S) * Hk * Wk * dv * eb), range(modes, 4 * n * size_t(kappa))}) {
            if (overlap(o, other)) return SCRAM_ERR_ALIAS;
        }
    }
    if (overlap(rO, rE) || overlap(rO, rV) || overlap(rE, rV)) return SCRAM_ERR_ALIAS;
    const scram::Grid grid{S, Hq, Wq, Hk, Wk, d};
    const scram::SnisSpec spec{samples, alpha, radius, scale, seed};
    const hipError_t e = scram::launch_snis(dtype, Q, K, V, modes, kappa, grid, spec, causal, out, ess_out, var_out,
                                            stream, events ? events[0] : nullptr, events ? events[1] : nullptr);
    return e == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

int scram_pad_channels(int count, const void* const* src, void* const* dst, const int64_t* rows, const int* widths,
                       int width, int elem_bytes, int unpad, hipStream_t stream)
{
    if (!src || !dst || !rows || !widths) return SCRAM_ERR_NULL;
    if (count < 1 || count > 4) return SCRAM_ERR_SHAPE;
    if (!supported_width(width) || (elem_bytes != 2 && elem_bytes != 4)) return SCRAM_ERR_UNSUPPORTED;
    scram::PadTensor t[4];
    for (int i = 0; i < count; ++i) {
        if (!src[i] || !dst[i]) return SCRAM_ERR_NULL;
        if (rows[i] < 1 || rows[i] >= (int64_t(1) << 40) / width || widths[i] < 1 || widths[i] > width)
            return SCRAM_ERR_SHAPE;
        const void* wide = unpad ? src[i] : dst[i];
        const void* narrow = unpad ? dst[i] : src[i];
        if (!aligned(wide, 16) || !aligned(narrow, elem_bytes)) return SCRAM_ERR_ALIGN;
        const size_t row = size_t(rows[i]) * elem_bytes;
        if (overlap(range(wide, row * width), range(narrow, row * widths[i]))) return SCRAM_ERR_ALIAS;
        t[i] = scram::PadTensor{src[i], dst[i], rows[i], widths[i]};
    }
    const hipError_t e = scram::launch_pad(t, count, width, elem_bytes, unpad != 0, stream);
    return e == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

int scram_differential_attend(const void* Q, const void* K, const void* V, int dtype, const int32_t* argmax, int kappa,
                              const float* lam, int S, int Hq, int Wq, int Hk, int Wk, int d, int dv, int window, float scale,
                              uint32_t flags, int first, const int32_t* origin, void* out, hipEvent_t* events,
                              hipStream_t stream)
{
    if (!Q || !K || !V || !argmax || !lam || !out) return SCRAM_ERR_NULL;
    const scram::Grid grid{S, Hq, Wq, Hk, Wk, d};
    int rc = check_differential(dtype, grid, kappa, dv, window, scale, flags, first, origin);
    if (rc) return rc;
    if (scram::diff_attend_max_blocks(dtype, grid) > kMaxBlocks) return SCRAM_ERR_SHAPE;
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(out, 16) || !aligned(argmax, 4) || !aligned(lam, 4) ||
        !aligned(origin, 4))
        return SCRAM_ERR_ALIGN;
    const size_t n = size_t(S) * Hq * Wq, nk = size_t(S) * Hk * Wk, eb = elem_bytes(dtype);
    const Range rO = range(out, n * dv * eb);
    for (const Range& other : {range(Q, n * d * eb), range(K, nk * d * eb), range(V, nk * dv * eb),
                               range(argmax, 4 * n * size_t(kappa)), range(lam, 4 * size_t(S)),
                               range(origin, origin ? 4 * size_t(S) : 0)}) {
        if (overlap(rO, other)) return SCRAM_ERR_ALIAS;
    }
    const scram::DiffCall call{Q, K, V, argmax, kappa, lam, grid, window, scale, (flags & SCRAM_CAUSAL) != 0, first, origin};
    const hipError_t e = scram::launch_diff_attend(dtype, call, out, stream, events ? events[0] : nullptr,
                                                   events ? events[1] : nullptr);
    return e == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

size_t scram_differential_attend_backward_workspace_bytes(int S, int Hq, int Wq, int Hk, int Wk, int d, int dtype, int kappa)
{
    if (check_grid(S, Hq, Wq, Hk, Wk) || kappa < 1 || kappa > SCRAM_MAX_KAPPA || check_type(dtype, d)) return 0;
    return scram::diff_backward_workspace_bytes(scram::Grid{S, Hq, Wq, Hk, Wk, d}, kappa);
}

int scram_differential_attend_backward(const void* Q, const void* K, const void* V, int dtype, const int32_t* argmax,
                                       int kappa, const float* lam, int S, int Hq, int Wq, int Hk, int Wk, int d, int dv,
                                       int window, float scale, uint32_t flags, int first, const int32_t* origin,
                                       const void* dO, float* dQ, float* dK, float* dV, float* dlam, void* workspace,
                                       size_t workspace_bytes, hipEvent_t* events, hipStream_t stream)
{
    if (!Q || !K || !V || !argmax || !lam || !dO || !dQ || !dK || !dV || !dlam) return SCRAM_ERR_NULL;
    const scram::Grid grid{S, Hq, Wq, Hk, Wk, d};
    int rc = check_differential(dtype, grid, kappa, dv, window, scale, flags, first, origin);
    if (rc) return rc;
    // the inverse map codes (match, query) pairs as e * n + i in an int32, and keys are numbered across slices
    if (int64_t(S) * Hq * Wq * kappa >= kMaxCount || int64_t(S) * Hk * Wk >= kMaxCount) return SCRAM_ERR_SHAPE;
    if (scram::diff_backward_max_blocks(grid) > kMaxBlocks) return SCRAM_ERR_SHAPE;
    if (!workspace) return SCRAM_ERR_WORKSPACE;
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(dO, 16) || !aligned(argmax, 4) || !aligned(lam, 4) ||
        !aligned(origin, 4) || !aligned(dQ, 16) || !aligned(dK, 16) || !aligned(dV, 16) || !aligned(dlam, 4) ||
        !aligned(workspace, 256))
        return SCRAM_ERR_ALIGN;
    const size_t need = scram::diff_backward_workspace_bytes(grid, kappa);
    if (workspace_bytes < need) return SCRAM_ERR_WORKSPACE;
    const size_t n = size_t(S) * Hq * Wq, nk = size_t(S) * Hk * Wk, eb = elem_bytes(dtype);
    const Range outs[] = {range(dQ, 4 * n * d), range(dK, 4 * nk * d), range(dV, 4 * nk * dv), range(dlam, 4 * size_t(S)),
                          range(workspace, need)};
    for (const Range& o : outs) {
        for (const Range& other : {range(Q, n * d * eb), range(K, nk * d * eb), range(V, nk * dv * eb),
                                   range(argmax, 4 * n * size_t(kappa)), range(dO, n * dv * eb), range(lam, 4 * size_t(S)),
                                   range(origin, origin ? 4 * size_t(S) : 0)}) {
            if (overlap(o, other)) return SCRAM_ERR_ALIAS;
        }
        for (const Range& other : outs) {
            if (&o != &other && overlap(o, other)) return SCRAM_ERR_ALIAS;
        }
    }
    const scram::DiffCall call{Q, K, V, argmax, kappa, lam, grid, window, scale, (flags & SCRAM_CAUSAL) != 0, first, origin};
    const hipError_t e = scram::launch_diff_backward(dtype, call, dO, dQ, dK, dV, dlam, workspace, stream,
                                                     events ? events[0] : nullptr, events ? events[1] : nullptr);
    return e == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

int scram_rotary(int count, const void* const* src, void* const* dst, const int* slices, int dtype, int T, int H, int W, int d,
                 int groups, const int* sections, const double* freqs, const int* first, const int32_t* origin, int origin_rows,
                 uint32_t flags, hipStream_t stream)
{
    if (!src || !dst || !slices || !sections || !freqs) return SCRAM_ERR_NULL;
    if (origin ? origin_rows < 1 : !first) return SCRAM_ERR_NULL;
    if (count < 1 || count > 4) return SCRAM_ERR_SHAPE;
    if (dtype != SCRAM_F32 && dtype != SCRAM_BF16) return SCRAM_ERR_UNSUPPORTED;
    if (flags & ~uint32_t(SCRAM_ROTARY_INTERLEAVED | SCRAM_ROTARY_INVERSE)) return SCRAM_ERR_UNSUPPORTED;
    if (T < 1 || H < 1 || W < 1 || T > kMaxSide || H > kMaxSide || W > kMaxSide) return SCRAM_ERR_SHAPE;
    if (int64_t(H) * W >= kMaxCount || int64_t(T) * (int64_t(H) * W) >= kMaxCount) return SCRAM_ERR_SHAPE;
    if (groups < 1 || d < 2 || d > 65536 || d % groups) return SCRAM_ERR_SHAPE;
    int64_t pairs = 0;
    for (int a = 0; a < 3; ++a) {
        if (sections[a] < 0) return SCRAM_ERR_SHAPE;
        pairs += sections[a];
    }
    if (pairs < 1 || pairs > SCRAM_ROTARY_MAX_PAIRS || 2 * pairs > d / groups) return SCRAM_ERR_SHAPE;
    for (int64_t k = 0; k < pairs; ++k)
        if (!isfinite(freqs[k])) return SCRAM_ERR_SHAPE;
    scram::RotaryCall c{};
    const size_t eb = elem_bytes(dtype), plane = size_t(T) * H * W * d * eb;
    c.count = count;
    for (int i = 0; i < count; ++i) {
        if (!src[i] || !dst[i]) return SCRAM_ERR_NULL;
        if (slices[i] < 1 || (origin && origin_rows > 1 && slices[i] != origin_rows)) return SCRAM_ERR_SHAPE;
        if (!aligned(src[i], eb) || !aligned(dst[i], eb)) return SCRAM_ERR_ALIGN;
        c.src[i] = src[i];
        c.dst[i] = dst[i];
        c.slices[i] = slices[i];
    }
    if (!aligned(origin, 4)) return SCRAM_ERR_ALIGN;
    for (int i = 0; i < count; ++i) {
        const Range o = range(dst[i], plane * slices[i]);
        if (overlap(o, range(origin, origin ? 12 * size_t(origin_rows) : 0))) return SCRAM_ERR_ALIAS;
        for (int j = 0; j < count; ++j) {
            // a tensor may be turned in place, and overlaps nothing otherwise
            if (!(i == j && src[j] == dst[i]) && overlap(o, range(src[j], plane * slices[j]))) return SCRAM_ERR_ALIAS;
            if (i != j && overlap(o, range(dst[j], plane * slices[j]))) return SCRAM_ERR_ALIAS;
        }
    }
    c.T = T;
    c.H = H;
    c.W = W;
    c.d = d;
    c.groups = groups;
    for (int a = 0; a < 3; ++a) {
        c.pairs[a] = sections[a];
        c.first[a] = origin ? 0 : first[a];
    }
    c.freq = freqs;
    c.origin = origin;
    c.origin_rows = origin_rows;
    c.interleaved = (flags & SCRAM_ROTARY_INTERLEAVED) != 0;
    c.inverse = (flags & SCRAM_ROTARY_INVERSE) != 0;
    if (scram::rotary_items(dtype, c) >= uint64_t(kMaxCount)) return SCRAM_ERR_SHAPE;
    return scram::launch_rotary(dtype, c, stream) == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

int scram_layer_norm(const void* X, int dtype, const void* weight, const void* bias, int weight_dtype, int64_t rows, int channels,
                     float eps, void* Y, float* mean, float* rstd, hipStream_t stream)
{
    if (!X || !Y || !mean != !rstd) return SCRAM_ERR_NULL;
    int rc = check_norm(rows, channels, dtype, weight_dtype);
    if (rc) return rc;
    if (!(eps >= 0.f) || !isfinite(eps)) return SCRAM_ERR_SHAPE;
    const size_t eb = elem_bytes(dtype), wb = elem_bytes(weight_dtype);
    if (!aligned(X, eb) || !aligned(Y, eb) || !aligned(weight, wb) || !aligned(bias, wb) || !aligned(mean, 4) || !aligned(rstd, 4))
        return SCRAM_ERR_ALIGN;
    const size_t n = size_t(rows) * channels, stat = mean ? 4 * size_t(rows) : 0;
    const Range outs[] = {range(Y, n * eb), range(mean, stat), range(rstd, stat)};
    for (const Range& o : outs) {
        // Y may be X: a row is read before it is written
        if (overlap(o, range(X, n * eb)) && !(&o == &outs[0] && Y == X)) return SCRAM_ERR_ALIAS;
        if (overlap(o, range(weight, weight ? wb * channels : 0)) || overlap(o, range(bias, bias ? wb * channels : 0)))
            return SCRAM_ERR_ALIAS;
        for (const Range& other : outs) {
            if (&o != &other && overlap(o, other)) return SCRAM_ERR_ALIAS;
        }
    }
    const scram::NormCall c{rows, channels, dtype, dtype, weight_dtype, X, weight, bias, nullptr, eps};
    return scram::launch_norm(c, Y, mean, rstd, stream) == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

size_t scram_layer_norm_backward_workspace_bytes(int64_t rows, int channels)
{
    if (check_norm(rows, channels, SCRAM_F32, SCRAM_F32)) return 0;
    return scram::norm_backward_workspace_bytes(rows, channels);
}

int scram_layer_norm_backward(const void* dY, int grad_dtype, const void* X, int dtype, const float* mean, const float* rstd,
                              const void* weight, int weight_dtype, int64_t rows, int channels, void* dX, float* dweight,
                              float* dbias, void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    if (!dY || !X || !mean || !rstd || !dX || !dweight || !dbias) return SCRAM_ERR_NULL;
    int rc = check_norm(rows, channels, dtype, weight_dtype);
    if (rc) return rc;
    if (grad_dtype != dtype && grad_dtype != SCRAM_F32) return SCRAM_ERR_UNSUPPORTED;
    if (!workspace) return SCRAM_ERR_WORKSPACE;
    const size_t eb = elem_bytes(dtype), gb = elem_bytes(grad_dtype), wb = elem_bytes(weight_dtype);
    if (!aligned(X, eb) || !aligned(dY, gb) || !aligned(dX, gb) || !aligned(weight, wb) || !aligned(mean, 4) || !aligned(rstd, 4) ||
        !aligned(dweight, 4) || !aligned(dbias, 4) || !aligned(workspace, 256))
        return SCRAM_ERR_ALIGN;
    const size_t need = scram::norm_backward_workspace_bytes(rows, channels);
    if (workspace_bytes < need) return SCRAM_ERR_WORKSPACE;
    const size_t n = size_t(rows) * channels;
    const Range outs[] = {range(dX, n * gb), range(dweight, 4 * size_t(channels)), range(dbias, 4 * size_t(channels)),
                          range(workspace, need)};
    for (const Range& o : outs) {
        // dX may be dY: a row is read before it is written
        if (overlap(o, range(dY, n * gb)) && !(&o == &outs[0] && dX == dY)) return SCRAM_ERR_ALIAS;
        for (const Range& other : {range(X, n * eb), range(mean, 4 * size_t(rows)), range(rstd, 4 * size_t(rows)),
                                   range(weight, weight ? wb * channels : 0)}) {
            if (overlap(o, other)) return SCRAM_ERR_ALIAS;
        }
        for (const Range& other : outs) {
            if (&o != &other && overlap(o, other)) return SCRAM_ERR_ALIAS;
        }
    }
    const scram::NormCall c{rows, channels, dtype, grad_dtype, weight_dtype, X, weight, nullptr, dY, 0.f};
    return scram::launch_norm_backward(c, mean, rstd, dX, dweight, dbias, workspace, stream) == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

size_t scram_dense_attend_workspace_bytes(int S, int key_slices, int Hq, int Wq, int Hk, int Wk, int d, int dtype, int biased)
{
    if (check_dense_grid(S, key_slices, Hq, Wq, Hk, Wk) || check_type(dtype, d)) return 0;
    return scram::dense_workspace_bytes(dtype, dense_call(nullptr, nullptr, nullptr, biased ? "" : nullptr, 1, nullptr, S, key_slices, Hq, Wq,
                                                   Hk, Wk, d, 1.f, 0, 0, nullptr));
}

int scram_dense_attend(const void* Q, const void* K, const void* V, int dtype, const void* bias, int bias_rows,
                       const int32_t* lengths, int S, int key_slices, int Hq, int Wq, int Hk, int Wk, int d, int dv, float scale,
                       uint32_t flags, int first, const int32_t* origin, void* out, void* workspace, size_t workspace_bytes,
                       hipEvent_t* events, hipStream_t stream)
{
    if (!Q || !K || !V || !out) return SCRAM_ERR_NULL;
    const scram::DenseCall call =
        dense_call(Q, K, V, bias, bias_rows, lengths, S, key_slices, Hq, Wq, Hk, Wk, d, scale, flags, first, origin);
    int rc = check_dense(dtype, call, dv, flags);
    if (rc) return rc;
    if (!fits(scram::dense_needs(dtype, call))) return SCRAM_ERR_SHAPE;
    const size_t eb = elem_bytes(dtype), need = scram::dense_workspace_bytes(dtype, call);
    if (need && !workspace) return SCRAM_ERR_WORKSPACE;
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(out, 16) || !aligned(bias, eb) || !aligned(lengths, 4) ||
        !aligned(origin, 4) || (need && !aligned(workspace, 256)))
        return SCRAM_ERR_ALIGN;
    if (workspace_bytes < need) return SCRAM_ERR_WORKSPACE;
    const size_t n = size_t(S) * Hq * Wq, nk = size_t(key_slices) * Hk * Wk;
    const Range outs[] = {range(out, n * dv * eb), range(workspace, need)};
    for (const Range& o : outs) {
        for (const Range& other : {range(Q, n * d * eb), range(K, nk * d * eb), range(V, nk * dv * eb), range(bias, bias_bytes(call, eb)),
                                   range(lengths, lengths ? 4 * size_t(key_slices) : 0), range(origin, origin ? 4 * size_t(S) : 0)}) {
            if (overlap(o, other)) return SCRAM_ERR_ALIAS;
        }
    }
    if (overlap(outs[0], outs[1])) return SCRAM_ERR_ALIAS;
    const hipError_t e = scram::launch_dense(dtype, call, out, workspace, stream, events ? events[0] : nullptr,
                                             events ? events[1] : nullptr);
    return e == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

size_t scram_dense_attend_backward_workspace_bytes(int S, int key_slices, int Hq, int Wq, int Hk, int Wk, int d, int dtype,
                                                   int bias_rows)
{
    if (check_dense_grid(S, key_slices, Hq, Wq, Hk, Wk) || check_type(dtype, d)) return 0;
    if (bias_rows < 0 || (bias_rows && S % bias_rows)) return 0;
    return scram::dense_backward_workspace_bytes(dtype, dense_call(nullptr, nullptr, nullptr, bias_rows ? "" : nullptr, bias_rows, nullptr, S,
                                                            key_slices, Hq, Wq, Hk, Wk, d, 1.f, 0, 0, nullptr));
}

int scram_dense_attend_backward(const void* Q, const void* K, const void* V, int dtype, const void* bias, int bias_rows,
                                const int32_t* lengths, int S, int key_slices, int Hq, int Wq, int Hk, int Wk, int d, int dv,
                                float scale, uint32_t flags, int first, const int32_t* origin, const void* dO, void* dQ, void* dK,
                                void* dV, void* dbias, void* workspace, size_t workspace_bytes, hipEvent_t* events,
                                hipStream_t stream)
{
    if (!Q || !K || !V || !dO || !dQ || !dK || !dV) return SCRAM_ERR_NULL;
    if (dbias && !bias) return SCRAM_ERR_NULL;
    const scram::DenseCall call =
        dense_call(Q, K, V, bias, bias_rows, lengths, S, key_slices, Hq, Wq, Hk, Wk, d, scale, flags, first, origin);
    int rc = check_dense(dtype, call, dv, flags);
    if (rc) return rc;
    if (!fits(scram::dense_backward_needs(dtype, call))) return SCRAM_ERR_SHAPE;
    if (!workspace) return SCRAM_ERR_WORKSPACE;
    const size_t eb = elem_bytes(dtype), need = scram::dense_backward_workspace_bytes(dtype, call);
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(dO, 16) || !aligned(bias, eb) || !aligned(lengths, 4) ||
        !aligned(origin, 4) || !aligned(dQ, 16) || !aligned(dK, 16) || !aligned(dV, 16) || !aligned(dbias, eb) ||
        !aligned(workspace, 256))
        return SCRAM_ERR_ALIGN;
    if (workspace_bytes < need) return SCRAM_ERR_WORKSPACE;
    const size_t n = size_t(S) * Hq * Wq, nk = size_t(key_slices) * Hk * Wk, bb = bias_bytes(call, eb);
    const Range outs[] = {range(dQ, n * d * eb), range(dK, nk * d * eb), range(dV, nk * dv * eb), range(dbias, dbias ? bb : 0),
                          range(workspace, need)};
    for (const Range& o : outs) {
        for (const Range& other : {range(Q, n * d * eb), range(K, nk * d * eb), range(V, nk * dv * eb), range(dO, n * dv * eb),
                                   range(bias, bb), range(lengths, lengths ? 4 * size_t(key_slices) : 0),
                                   range(origin, origin ? 4 * size_t(S) : 0)}) {
            if (overlap(o, other)) return SCRAM_ERR_ALIAS;
        }
        for (const Range& other : outs) {
            if (&o != &other && overlap(o, other)) return SCRAM_ERR_ALIAS;
        }
    }
    const hipError_t e = scram::launch_dense_backward(dtype, call, dO, dQ, dK, dV, dbias, workspace, stream,
                                                      events ? events[0] : nullptr, events ? events[1] : nullptr);
    return e == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

int scram_relative_bias(const void* table, int dtype, int heads, int H, int W, const int* edges_y, int my, const int* edges_x, int mx,
                        void* bias, hipStream_t stream)
{
    if (!table || !bias) return SCRAM_ERR_NULL;
    int rc = check_relative(dtype, heads, H, W, edges_y, my, edges_x, mx);
    if (rc) return rc;
    const size_t eb = elem_bytes(dtype);
    if (!aligned(table, eb) || !aligned(bias, eb)) return SCRAM_ERR_ALIGN;
    if (overlap(range(bias, size_t(heads) * (2 * size_t(H) - 1) * (2 * size_t(W) - 1) * eb),
                range(table, size_t(heads) * (2 * my + 1) * (2 * mx + 1) * eb)))
        return SCRAM_ERR_ALIAS;
    const scram::BiasCall c{dtype, heads, H, W, {my, mx}, {edges_y, edges_x}};
    return scram::launch_relative_bias(c, table, bias, stream) == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

size_t scram_relative_bias_backward_workspace_bytes(int heads, int H, int W, int mx)
{
    if (mx < 0 || mx > SCRAM_BIAS_MAX_EDGES || check_relative(SCRAM_F32, heads, H, W, nullptr, 0, nullptr, 0)) return 0;
    return scram::relative_bias_backward_workspace_bytes(scram::BiasCall{SCRAM_F32, heads, H, W, {0, mx}, {nullptr, nullptr}});
}

int scram_relative_bias_backward(const void* dbias, int dtype, int heads, int H, int W, const int* edges_y, int my, const int* edges_x,
                                 int mx, void* dtable, void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    if (!dbias || !dtable) return SCRAM_ERR_NULL;
    int rc = check_relative(dtype, heads, H, W, edges_y, my, edges_x, mx);
    if (rc) return rc;
    if (!workspace) return SCRAM_ERR_WORKSPACE;
    const size_t eb = elem_bytes(dtype);
    if (!aligned(dbias, eb) || !aligned(dtable, eb) || !aligned(workspace, 256)) return SCRAM_ERR_ALIGN;
    const scram::BiasCall c{dtype, heads, H, W, {my, mx}, {edges_y, edges_x}};
    const size_t need = scram::relative_bias_backward_workspace_bytes(c);
    if (workspace_bytes < need) return SCRAM_ERR_WORKSPACE;
    const Range in = range(dbias, size_t(heads) * (2 * size_t(H) - 1) * (2 * size_t(W) - 1) * eb);
    const Range out = range(dtable, size_t(heads) * (2 * my + 1) * (2 * mx + 1) * eb), ws = range(workspace, need);
    if (overlap(in, out) || overlap(in, ws) || overlap(out, ws)) return SCRAM_ERR_ALIAS;
    return scram::launch_relative_bias_backward(c, dbias, dtable, workspace, stream) == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

size_t scram_group_norm_workspace_bytes(int64_t images, int64_t pixels, int channels, int groups, int dtype)
{
    if (check_group(images, pixels, channels, groups, dtype, dtype, SCRAM_ACT_NONE)) return 0;
    return scram::group_norm_workspace_bytes(
        scram::GroupCall{images, pixels, channels, groups, dtype, dtype, dtype, 0, nullptr, nullptr, nullptr, nullptr, 0.f});
}

int scram_group_norm(const void* X, int dtype, const void* weight, const void* bias, int weight_dtype, int64_t images, int64_t pixels,
                     int channels, int groups, float eps, int activation, void* Y, float* mean, float* rstd, void* workspace,
                     size_t workspace_bytes, hipStream_t stream)
{
    if (!X || !Y || !mean != !rstd) return SCRAM_ERR_NULL;
    int rc = check_group(images, pixels, channels, groups, dtype, weight_dtype, activation);
    if (rc) return rc;
    if (!(eps >= 0.f) || !isfinite(eps)) return SCRAM_ERR_SHAPE;
    const size_t eb = elem_bytes(dtype), wb = elem_bytes(weight_dtype);
    const scram::GroupCall c{images, pixels, channels, groups, dtype, dtype, weight_dtype, activation, X, weight, bias, nullptr, eps};
    const size_t need = scram::group_norm_workspace_bytes(c);
    if (need && !workspace) return SCRAM_ERR_WORKSPACE;
    if (!aligned(X, eb) || !aligned(Y, eb) || !aligned(weight, wb) || !aligned(bias, wb) || !aligned(mean, 4) || !aligned(rstd, 4) ||
        (need && !aligned(workspace, 256)))
        return SCRAM_ERR_ALIGN;
    if (workspace_bytes < need) return SCRAM_ERR_WORKSPACE;
    const size_t n = size_t(images) * pixels * channels, stat = mean ? 4 * size_t(images) * groups : 0;
    const Range outs[] = {range(Y, n * eb), range(mean, stat), range(rstd, stat), range(workspace, need)};
    for (const Range& o : outs) {
        // Y may be X: an element is read before it is written, and after the statistics
        if (overlap(o, range(X, n * eb)) && !(&o == &outs[0] && Y == X)) return SCRAM_ERR_ALIAS;
        if (overlap(o, range(weight, weight ? wb * channels : 0)) || overlap(o, range(bias, bias ? wb * channels : 0)))
            return SCRAM_ERR_ALIAS;
        for (const Range& other : outs) {
            if (&o != &other && overlap(o, other)) return SCRAM_ERR_ALIAS;
        }
    }
    return scram::launch_group_norm(c, Y, mean, rstd, workspace, stream) == hipSuccess ? SCRAM_OK : SCRAM_ERR_HIP;
}

size_t scram_group_norm_backward_workspace_bytes(int64_t images, int64_t pixels, int channels, int groups, int dtype)
{
    if (check_group(images, pixels, channels, groups, dtype, dtype, SCRAM_ACT_NONE)) return 0;
    return scram::group_norm_backward_workspace_bytes(
        scram::GroupCall{images, pixels, channels, groups, dtype, dtype, dtype, 0, nullptr, nullptr, nullptr, nullptr, 0.f});
}

int scram_group_norm_backward(const void* dY, int grad_dtype, const void* X, int dtype, const float* mean, const float* rstd,
                              const void* weight, const void* bias, int weight_dtype, int64_t images, int64_t pixels, int channels,
                              int groups, int activation, void* dX, float* dweight, float* dbias, void* workspace,
                              size_t workspace_bytes, hipStream_t stream)
{
    if (!dY || !X || !mean || !rstd || !dX || !dweight || !dbias) return SCRAM_ERR_NULL;
    int rc = check_group(images, pixels, channels, groups, dtype, weight_dtype, activation);
    if (rc) return rc;
    if (grad_dtype != dtype && grad_dtype != SCRAM_F32) return SCRAM_ERR_UNSUPPORTED;
    if (!workspace) return SCRAM_ERR_WORKSPACE;
    const size_t eb = elem_bytes(dtype), gb = elem_bytes(grad_dtype), wb = elem_bytes(weight_dtype);
    if (!aligned(X, eb) || !aligned(dY, gb) || !aligned(dX, gb) || !aligned(weight, wb) || !aligned(bias, wb) || !aligned(mean, 4) ||
        !aligned(rstd, 4) || !aligned(dweight, 4) || !aligned(dbias, 4) || !aligned(workspace, 256))
        return SCRAM_ERR_ALIGN;
    const scram::GroupCall c{images, pixels, channels, groups, dtype, grad_dtype, weight_dtype, activation, X, weight, bias, dY, 0.f};
    const size_t need = scram::group_norm_backward_workspace_bytes(c);
    if (workspace_bytes < need) return SCRAM_ERR_WORKSPACE;
    const size_t n = size_t(images) * pixels * channels, stat = 4 * size_t(images) * groups;
    const Range outs[] = {range(dX, n * gb), range(dweight, 4 * size_t(channels)), range(dbias, 4 * size_t(channels)),
                          range(workspace, need)};
    for (const Range& o : outs) {
        // dX may be dY: an element is read before it is written, and after the sums
        if (overlap(o, range(dY, n * gb)) && !(&o == &outs[0] && dX == dY)) return SCRAM_ERR_ALIAS;
        for (const Range& other : {range(X, n * eb), range(mean, stat), range(rstd, stat), range(weight, weight ? wb * channels : 0),
                                   range(bias, bias ? wb * channels : 0)}) {
            if (overlap(o, other)) return SCRAM_ERR_ALIAS;
        }
        for (const Range& other : outs) {
            if (&o != &other && overlap(o, other)) return SCRAM_ERR_ALIAS;
        }
    }
    return scram::launch_group_norm_backward(c, mean, rstd, dX, dweight, dbias, workspace, stream) == hipSuccess ? SCRAM_OK
                                                                                                                 : SCRAM_ERR_HIP;
}

const char* scram_status_string(int status)
{
    switch (status) {
        case SCRAM_OK: return "ok";
        case SCRAM_ERR_NULL: return "a required pointer is NULL";
        case SCRAM_ERR_SHAPE: return "a size or count is out of range";
        case SCRAM_ERR_UNSUPPORTED: return "unsupported dtype, channel count or flag";
        case SCRAM_ERR_ALIGN: return "a pointer is not aligned as required";
        case SCRAM_ERR_ALIAS: return "an output overlaps an input or another output";
        case SCRAM_ERR_HIP: return "a HIP launch or copy failed";
        case SCRAM_ERR_WORKSPACE: return "workspace missing or too small";
        case SCRAM_ERR_SCRATCH: return "more queries than the no-allocation entry point's fixed scratch holds";
        default: return "unknown status";
    }
}

int scram_abi_version(void) { return SCRAM_ABI_VERSION; }

}  // extern "C"
