// Host-side interface between the entry points of acp_ops.h and their launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "acp_internal.h"
#include "acp_ops.h"

namespace acp {

struct Strides {              // elements, {batch, head, position}
    int64_t b, h, l;
};

struct NormArgs {
    const void* x;
    const void* dy;           // backward only
    Strides xs, dys, dxs;
    const void* weight;
    const void* bias;         // forward only, or null
    bool bf16, wbf16;
    int B, H, L, n;
    bool per_head, center;
    float eps;
    void* y;                  // forward: [B, H, L, n]; backward: dx
    float* mean;              // [B, H, L], or null
    float* rstd;
    float* dweight;           // [groups, n]
    float* dbias;             // or null
    float* part;              // [2 (with dbias)][groups][norm_parts][n]
};

struct RotaryArgs {
    const void* x[2];         // q, k (null: absent)
    void* y[2];
    Strides xs[2], ys[2];
    int heads[2];
    bool bf16;
    int B, L, d, rot;
    bool interleaved, inverse;
    float amplitude;
    const double* turns;      // [rot / 2]
    const void* pos;
    int pos_bytes;
    int64_t pos_b, pos_l, start;
};

struct PagedArgs {
    bool bf16;
    int T, N, W, P, H, Hk, d;
    const int* cu;
    const int* past;
    const int* table;
    void* kp;                 // [P, Hk, 64, d]
    void* vp;
    double* cp;               // [P, H, 64]
    int* flags;               // [N, H] or null
    // append
    const void* k;
    const void* v;
    const float* log_f;
    int64_t kt, kh, vt, vh, ft, fh;   // strides {token, head}
    // attention
    const void* q;
    int64_t qt, qh;
    const float* gamma_q;
    const float* gamma_k;
    double log_lmax_over_eps; // +inf for eps = 0
    bool fill;                // rows that nothing attends for: O = 0, lse = -inf
    int max_new;
    int64_t max_len;
    void* O;
    float* lse;
    float* part;
};

size_t norm_workspace(int B, int H, int L, int n, bool per_head);
size_t paged_workspace(const PagedArgs& a);
hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t s);
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t s);
hipError_t launch_paged_append(const PagedArgs& a, hipStream_t s);
hipError_t launch_paged_attend(const PagedArgs& a, hipStream_t s);

}  // namespace acp
