// Parameters of the kernels that compute the attend's gradients, by kernel
// value; the differential attend's (scram_diff.h) extend them.
//
// Everything here lives in an unnamed namespace, like scram_device.h.

#pragma once

#include "scram_wave.h"

namespace scram {
namespace {

struct BwdParams {
    const void* Q;
    const void* K;
    const void* V;
    const int32_t* J;      // [kappa, n]
    const void* dO;
    float* dQ;
    float* dK;
    float* dV;
    float* lse2;           // [n] max + log2(normaliser), base-2 scores
    float* Dq;             // [n] D_i
    const int32_t* offsets;  // [S * nkeys + 1] start of each key's entries
    const int32_t* entries;  // [kappa * n] e * n + i, grouped by match key
    int32_t* counts;         // [S * nkeys] entries per match key (zeroed before the query kernel)
    int32_t* slots;          // [kappa * n] each entry's slot among its key's entries
    int32_t* heavy;          // [S * nkeys] keys left to bwd_heavy_kernel (fp32 strips: to bwd_strip_team_f32_kernel)
    int32_t* n_heavy;        // their count
    int heavy_entries;       // fp32 strips: most entries of a strip that one wave sums
    void* qs;                // [kappa * n, D] q_i of each entry, in entry order
    void* gs;                // [kappa * n, D] dO_i of each entry, in entry order
    float2* st;              // [kappa * n] (log2 normaliser, D_i) of each entry
    uint32_t n;
    uint32_t keys_total;   // S * nkeys
    Tiling tq, tk;         // blocks -> tiles of the query grid (query kernel), the key grid (key kernel)
    int Hq, Wq, Hk, Wk;
    uint32_t nkeys;
    Div div_plane, div_wk, div_n, div_keys;
    int b;
    float scale;
    float scale_log2e;
    int kappa;
    int causal;
    int rc;                // cluster radius of the matrix-core query kernel
};

}  // namespace
}  // namespace scram
