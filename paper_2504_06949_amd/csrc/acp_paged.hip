// New tokens into the pages of a cache: keys and values to their slots, and the cumulative
// gates on top of those held.
//
// One launch holds two kinds of workgroups that touch different memory: the first ones sum
// the gates of a sequence (a few heads each), the others copy the rows of a few tokens.  Bound
// by memory: each row is read and written once.  Ragged 32k tokens of 12 heads (d = 64,
// bfloat16): 35 to 44 us for 206 MB.
#include "acp_paged.h"
#include "acp_scan.h"

namespace acp {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kFewTokens = 16;                       // summed one after the other
// Heads per workgroup of the sums: one where sequences are long (issue on the one CU that
// holds a workgroup bounds them: four heads took 60 us where one was hidden behind the 50 us
// that the copies then took, ragged 32k tokens of 12 heads), four where there are more
// sequences than CUs
constexpr int kGateHeadsLong = 1, kGateHeadsShort = 4;
static_assert(kWaves * kGateHeadsShort == 64, "a total per lane");

// Flags of a log gate x and of the sum c that it leads to (which may hold the infinity or NaN of
// a gate of an earlier call)
__device__ __forceinline__ int gate_flags(float x, double c) {
    int f = !__builtin_isfinite(x) ? 2 : x > 0.0f ? 1 : 0;
    const double size = __builtin_fabs(c);
    if (!(size <= 0x1.fffffep127)) f |= 2;
    if (size >= 0x1p32 && size < INFINITY) f |= 4;
    return f;
}

struct GateSmem {
    double total[2][kWaves * kGateHeadsShort];       // [head][wave] of the pages of a step, in turn
    int flags[kGateHeadsShort];
};

// c of a few new positions of sequence s: a thread per head
__device__ __forceinline__ void append_few_gates(const PagedArgs& a, int s, const Seq& q) {
    const int before = q.past > 0 && q.n > 0 ? page_of(a, s, (q.past - 1) >> 6) : 0;
    for (int h = threadIdx.x; h < a.H; h += kThreads) {
        int flags = before < 0 ? kFlagPage : 0;
        double c = q.past > 0 && q.n > 0 && before >= 0 ? gates_of(a, before, h)[(q.past - 1) & 63] : 0.0;
        const float* f = a.log_f + (int64_t)q.row0 * a.ft + h * a.fh;
#pragma unroll 4
        for (int r = 0; r < q.n; ++r) {
            const float x = f[(int64_t)r * a.ft];
            c += (double)x;
            flags |= gate_flags(x, c);
            const int pos = q.past + r, p = page_of(a, s, pos >> 6);
            if (p < 0) flags |= kFlagPage;
            else a.cp[((int64_t)p * a.H + h) * 64 + (pos & 63)] = c;
        }
        if (a.flags) a.flags[(int64_t)s * a.H + h] = flags;
    }
}

// c of the new positions of sequence s, heads h0 .. h0 + kGateHeads - 1, in steps of 1024
// positions: each wave scans a page of the heads in float64 (a lane per position), the pages'
// totals go through LDS, and every wave scans these.  The sums are exact, whatever their
// order, while they span less than 53 bits.
template <int kGateHeads>
__device__ __forceinline__ void append_gates(const PagedArgs& a, int s, int h0, GateSmem& sm) {
    const Seq q = seq_of(a, s);
    if (q.n <= kFewTokens) {
        if (h0 == 0) append_few_gates(a, s, q);
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int first = q.past & ~63;                   // steps are counted from a page's start
    const int skip = q.past & 63, rows = skip + q.n;  // positions from there on, new ones last
    const float* f = a.log_f + (int64_t)q.row0 * a.ft;

    if (threadIdx.x < kGateHeads) sm.flags[threadIdx.x] = 0;
    // gates and pages of kAhead steps are asked for while the kAhead before are worked on (the
    // copies saturate the memory meanwhile, and a load takes microseconds)
    constexpr int kAhead = 2, kStep = 64 * kWaves;
    float next[kAhead][kGateHeads];
    int page_next = -1;                               // lane j: this wave's page of step j
    double c[kGateHeads];
    int flags[kGateHeads];
    auto bring = [&](int t0) __attribute__((always_inline)) {
        page_next = page_of(a, s, (first + min(t0 + kStep * min(lane, kAhead - 1) + 64 * wave, rows - 1)) >> 6);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int r = t0 + kStep * j + 64 * wave + lane - skip;
            const float* fr = f + (int64_t)min(max(r, 0), q.n - 1) * a.ft;
#pragma unroll
            for (int k = 0; k < kGateHeads; ++k) next[j][k] = fr[min(h0 + k, a.H - 1) * a.fh];
        }
    };
#pragma unroll
    for (int k = 0; k < kGateHeads; ++k) {
        c[k] = 0.0;
        flags[k] = 0;
    }
    bring(0);
    if (q.past > 0) {
        const int p = page_of(a, s, (q.past - 1) >> 6);
#pragma unroll
        for (int k = 0; k < kGateHeads; ++k) {
            if (p < 0) flags[k] |= kFlagPage;
            else c[k] = gates_of(a, p, min(h0 + k, a.H - 1))[(q.past - 1) & 63];
        }
    }
    int turn = 0;
    for (int t0 = 0; t0 < rows; t0 += kAhead * kStep) {
        float x[kAhead][kGateHeads];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
#pragma unroll
            for (int k = 0; k < kGateHeads; ++k) x[j][k] = next[j][k];
        const int pages = page_next;
        if (t0 + kAhead * kStep < rows) bring(t0 + kAhead * kStep);
#pragma unroll
        for (int j = 0; j < kAhead; ++j, turn ^= 1) {
            if (t0 + kStep * j >= rows) break;
            const int t = t0 + kStep * j + 64 * wave, r = t + lane - skip;
            const bool is_new = r >= 0 && r < q.n;
            const int p = __builtin_amdgcn_readlane(pages, j);
            double incl[kGateHeads];
#pragma unroll
            for (int k = 0; k < kGateHeads; ++k) {
                incl[k] = wave_inclusive_scan_f64(is_new ? (double)x[j][k] : 0.0);
            }
            if (lane == 63)
#pragma unroll
                for (int k = 0; k < kGateHeads; ++k) sm.total[turn][kWaves * k + wave] = incl[k];
            lds_barrier();
            // lane 16 k + w: the totals of head k's pages up to wave w (k < kGateHeads)
            double tot = sm.total[turn][lane & (kWaves * kGateHeads - 1)];
            tot += dpp_f64_or_zero<0x111>(tot);
            tot += dpp_f64_or_zero<0x112>(tot);
            tot += dpp_f64_or_zero<0x114>(tot);
            tot += dpp_f64_or_zero<0x118>(tot);
            if (t < rows && p < 0) flags[0] |= kFlagPage;
#pragma unroll
            for (int k = 0; k < kGateHeads; ++k) {
                const double before = wave > 0 ? readlane_f64(tot, 16 * k + max(wave - 1, 0)) : 0.0;
                const double sum = c[k] + (before + incl[k]);
                if (is_new) flags[k] |= gate_flags(x[j][k], sum);
                if (is_new && p >= 0 && h0 + k < a.H) a.cp[((int64_t)p * a.H + h0 + k) * 64 + lane] = sum;
                c[k] += readlane_f64(tot, 16 * k + kWaves - 1);
            }
        }
    }
    if (a.flags == nullptr) return;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kGateHeads; ++k) {
        const int fk = flags[k] | (flags[0] & kFlagPage);
        if (fk) atomicOr(&sm.flags[k], fk);
    }
    __syncthreads();
    if (threadIdx.x < kGateHeads && h0 + (int)threadIdx.x < a.H)
        a.flags[(int64_t)s * a.H + h0 + threadIdx.x] = sm.flags[threadIdx.x];
}

template <typename T>
__device__ __forceinline__ void append_rows(const PagedArgs& a, int t0, int tokens, int64_t* slot) {
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
    // 16-byte pieces: kBatch of both tensors per thread are requested before one is stored
    constexpr int kBatch = 2;
    const int shift = 31 - __builtin_clz(a.d / VEC);  // pieces of a row: a power of two
    const int per = a.Hk << shift, n = tokens * per;
    for (int j0 = threadIdx.x; j0 < n; j0 += kBatch * kThreads) {
        u32x4 kv[kBatch], vv[kBatch];
        int64_t dst[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            // (past the last piece, that piece again; a token past the call's, its last one)
            const int j = min(j0 + b * kThreads, n - 1), tl = j / per, e = j - tl * per;
            const int h = e >> shift, f = (e - (h << shift)) * VEC;
            const int64_t at = slot[tl], t = min(t0 + tl, a.T - 1);
            dst[b] = at < 0 || j0 + b * kThreads >= n ? -1 : at + (int64_t)h * 64 * a.d + f;
            kv[b] = *reinterpret_cast<const u32x4*>((const T*)a.k + t * a.kt + h * a.kh + f);
            vv[b] = *reinterpret_cast<const u32x4*>((const T*)a.v + t * a.vt + h * a.vh + f);
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (dst[b] >= 0) {
                *reinterpret_cast<u32x4*>((T*)a.kp + dst[b]) = kv[b];
                *reinterpret_cast<u32x4*>((T*)a.vp + dst[b]) = vv[b];
            }
        }
    }
}

template <typename T, int HG>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(PagedArgs a, int gate_wgs, int groups,
                                                                int tokens) {
    __shared__ union {
        GateSmem gates;
        int64_t slot[64];
    } sm;
    const int b = blockIdx.x;
    if (b < gate_wgs) append_gates<HG>(a, b / groups, (b % groups) * HG, sm.gates);
    else append_rows<T>(a, (b - gate_wgs) * tokens, tokens, sm.slot);
}

}  // namespace

hipError_t launch_paged_append(const PagedArgs& a, hipStream_t s) {
    trace_begin(ACP_K_COUNT + ACP_OP_APPEND, s);
    const bool is_long = a.T > 64 * (int64_t)a.N;
    const int hg = is_long ? kGateHeadsLong : kGateHeadsShort;
    const int groups = (a.H + hg - 1) / hg;
    const int gate_wgs = a.N * groups;
    // tokens per copying workgroup: 2 pieces of 16 bytes of each tensor per thread, at least
    // one token
    const int pieces = a.Hk * a.d / (a.bf16 ? 8 : 4);
    int tokens = 2 * kThreads / pieces;
    tokens = tokens < 1 ? 1 : tokens > 64 ? 64 : tokens;
    while (tokens > 1 && (a.T + tokens - 1) / tokens < 512) tokens /= 2;
    const int copy_wgs = (a.T + tokens - 1) / tokens;
    const auto kernel = a.bf16 ? (is_long ? paged_append_kernel<__bf16, kGateHeadsLong>
                                          : paged_append_kernel<__bf16, kGateHeadsShort>)
                               : (is_long ? paged_append_kernel<float, kGateHeadsLong>
                                          : paged_append_kernel<float, kGateHeadsShort>);
    hipLaunchKernelGGL(kernel, dim3(gate_wgs + copy_wgs), dim3(kThreads), 0, s, a, gate_wgs, groups, tokens);
    const hipError_t e = hipGetLastError();
    trace_end(ACP_K_COUNT + ACP_OP_APPEND, s);
    return e;
}

}  // namespace acp
