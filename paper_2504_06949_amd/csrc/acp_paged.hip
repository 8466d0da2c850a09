// New tokens into the pages of a cache: keys and values to their slots, and the cumulative
// gates on top of those held.
//
// One launch holds two kinds of workgroups that touch different memory: the first ones sum
// the gates of a sequence (8 heads each), the others copy the rows of a few tokens.  Bound
// by memory: each row is read and written once.
#include "acp_paged.h"

namespace acp {
namespace {

constexpr int kThreads = 1024;
constexpr int kGateHeads = 8;                        // heads per workgroup of the sums
constexpr int kGateLanes = kThreads / kGateHeads;    // runs that a head's tokens are cut into

// c of the new positions of sequence s, heads h0 .. h0 + 7: every thread sums a run of one
// head's tokens in float64, the runs are scanned, and the run is gone through again.  The
// sums are exact, whatever their order, while they span less than 53 bits.
__device__ void append_gates(const PagedArgs& a, int s, int h0, double* scan) {
    const Seq q = seq_of(a, s);
    const int hl = threadIdx.x % kGateHeads, ln = threadIdx.x / kGateHeads;
    const int h = h0 + hl;
    const bool on = h < a.H;
    const int per = (q.n + kGateLanes - 1) / kGateLanes;
    const int r0 = min(ln * per, q.n), r1 = min(r0 + per, q.n);
    const float* f = a.log_f + (int64_t)q.row0 * a.ft + (on ? h : 0) * a.fh;

    int flags = 0;
    double sum = 0.0;
    for (int r = r0; r < r1; ++r) {
        const float v = f[(int64_t)r * a.ft];
        if (!__builtin_isfinite(v)) flags |= 2;
        else if (v > 0.0f) flags |= 1;
        sum += (double)v;
    }
    scan[threadIdx.x] = sum;
    __syncthreads();
    for (int o = 1; o < kGateLanes; o <<= 1) {
        const double t = ln >= o ? scan[threadIdx.x - o * kGateHeads] : 0.0;
        __syncthreads();
        scan[threadIdx.x] += t;
        __syncthreads();
    }
    double c = ln > 0 ? scan[threadIdx.x - kGateHeads] : 0.0;
    if (on) {
        if (q.past > 0 && q.n > 0) {
            const int p = page_of(a, s, (q.past - 1) >> 6);
            if (p >= 0) c += gates_of(a, p, h)[(q.past - 1) & 63];
            else flags |= kFlagPage;
        }
        double* dst = nullptr;
        int held = -1;                                // page of the table that dst is of
        for (int r = r0; r < r1; ++r) {
            c += (double)f[(int64_t)r * a.ft];
            const int pos = q.past + r;
            if ((pos >> 6) != held) {
                held = pos >> 6;
                const int p = page_of(a, s, held);
                if (p < 0) flags |= kFlagPage;
                dst = p < 0 ? nullptr : a.cp + ((int64_t)p * a.H + h) * 64;
            }
            if (dst) dst[pos & 63] = c;
        }
    }
    if (a.flags == nullptr) return;
    int* fl = reinterpret_cast<int*>(scan);
    __syncthreads();
    if (threadIdx.x < kGateHeads) fl[threadIdx.x] = 0;
    __syncthreads();
    if (flags) atomicOr(&fl[hl], flags);
    __syncthreads();
    if (threadIdx.x < kGateHeads && on) a.flags[(int64_t)s * a.H + h] = fl[hl];
}

// The sequence that holds packed row t, or -1: the last one that starts at or before it
__device__ __forceinline__ int sequence_of(const PagedArgs& a, int t) {
    int lo = 0, hi = a.N;                             // first s with cu[s + 1] > t
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.cu[mid + 1] > t) hi = mid;
        else lo = mid + 1;
    }
    return lo < a.N && a.cu[lo] <= t ? lo : -1;
}

template <typename T>
__device__ void append_rows(const PagedArgs& a, int t0, int tokens, int64_t* slot) {
    constexpr int VEC = 16 / (int)sizeof(T);
    if ((int)threadIdx.x < tokens) {
        const int t = t0 + threadIdx.x;
        int64_t at = -1;
        const int s = t < a.T ? sequence_of(a, t) : -1;
        if (s >= 0) {
            const Seq q = seq_of(a, s);
            const int r = t - q.row0;
            if (r >= 0 && r < q.n) {
                const int pos = q.past + r;
                const int p = page_of(a, s, pos >> 6);
                if (p >= 0) at = ((int64_t)p * a.Hk * 64 + (pos & 63)) * a.d;
            }
        }
        slot[threadIdx.x] = at;
    }
    __syncthreads();
    const int row = a.d / VEC, per = a.Hk * row;      // 16-byte pieces of a row, a token
    for (int i = threadIdx.x; i < tokens * per * 2; i += kThreads) {
        const int kv = i / (tokens * per), j = i - kv * tokens * per;
        const int tl = j / per, e = j - tl * per;
        const int64_t at = slot[tl];
        if (at < 0) continue;
        const int h = e / row, f = (e - h * row) * VEC;
        const int64_t t = t0 + tl;
        const T* src = kv ? (const T*)a.v + t * a.vt + h * a.vh : (const T*)a.k + t * a.kt + h * a.kh;
        T* dst = (T*)(kv ? a.vp : a.kp) + at + (int64_t)h * 64 * a.d;
        *reinterpret_cast<uint4*>(dst + f) = *reinterpret_cast<const uint4*>(src + f);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(PagedArgs a, int gate_wgs,
                                                                int groups, int tokens) {
    __shared__ double scan[kThreads];
    const int b = blockIdx.x;
    if (b < gate_wgs) append_gates(a, b / groups, (b % groups) * kGateHeads, scan);
    else append_rows<T>(a, (b - gate_wgs) * tokens, tokens, reinterpret_cast<int64_t*>(scan));
}

}  // namespace

hipError_t launch_paged_append(const PagedArgs& a, hipStream_t s) {
    trace_begin(ACP_K_COUNT + ACP_OP_APPEND, s);
    const int groups = (a.H + kGateHeads - 1) / kGateHeads;
    const int gate_wgs = a.N * groups;
    // tokens per copying workgroup: 4 pieces of 16 bytes per thread, at least one token
    const int pieces = 2 * a.Hk * a.d / (a.bf16 ? 8 : 4);
    int tokens = 4 * kThreads / pieces;
    tokens = tokens < 1 ? 1 : tokens > 64 ? 64 : tokens;
    while (tokens > 1 && (a.T + tokens - 1) / tokens < 512) tokens /= 2;
    const int copy_wgs = (a.T + tokens - 1) / tokens;
    if (a.bf16)
        hipLaunchKernelGGL(paged_append_kernel<__bf16>, dim3(gate_wgs + copy_wgs), dim3(kThreads), 0, s,
                           a, gate_wgs, groups, tokens);
    else
        hipLaunchKernelGGL(paged_append_kernel<float>, dim3(gate_wgs + copy_wgs), dim3(kThreads), 0, s,
                           a, gate_wgs, groups, tokens);
    const hipError_t e = hipGetLastError();
    trace_end(ACP_K_COUNT + ACP_OP_APPEND, s);
    return e;
}

}  // namespace acp
