// Layer norm and RMS norm of rows, forward and backward.
//
// A row is held in registers by the threads that share it (8 lanes to 1024 threads, each
// with up to 4 pieces of 16 bytes), so that it is read once and the mean is known before
// the squares of the centred row are summed.  Both passes are bound by memory: forward
// reads x and writes y, backward reads x and dy and writes dx.  The weight's gradient
// stays in registers while a workgroup goes through its rows; it leaves one row of
// partial sums per workgroup, and a second launch adds these in a fixed order.
#include "acp_device.h"
#include "acp_ops_internal.h"

namespace acp {
namespace {

constexpr int kMaxBlocksNorm = 1024;   // workgroups of a backward pass, at most

struct NormGeom {
    Strides xs, dys, dxs;
    int H, L, n;
    int groups;              // weight rows: H (per head) or 1
    int rows;                // rows per weight row
};

// Row r of group g as (batch, head, position)
struct RowAt {
    int64_t b, h, l;
};
__device__ __forceinline__ RowAt row_at(const NormGeom& q, int g, int r) {
    RowAt a;
    if (q.groups > 1) {
        const int b = r / q.L;
        a.b = b; a.h = g; a.l = r - b * q.L;
    } else {
        const int bh = r / q.L, b = bh / q.H;
        a.b = b; a.h = bh - b * q.H; a.l = r - bh * q.L;
    }
    return a;
}
__device__ __forceinline__ int64_t at(const Strides& s, const RowAt& a) {
    return a.b * s.b + a.h * s.h + a.l * s.l;
}

// VEC consecutive elements from p (aligned to the element only; gfx950 loads them in one
// instruction all the same), `left` of them inside the row
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T* p, int left, float (&v)[VEC]) {
    if (left >= VEC) {
        T t[VEC];
        __builtin_memcpy(t, p, sizeof(t));
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = to_f32(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = i < left ? to_f32(p[i]) : 0.f;
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T* p, int left, const float (&v)[VEC]) {
    if (left >= VEC) {
        T t[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) t[i] = from_f32<T>(v[i]);
        __builtin_memcpy(p, t, sizeof(t));
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < left) p[i] = from_f32<T>(v[i]);
    }
}

// Sums over the LPR threads that share a row (LPR > 64: the workgroup).  `red` has two
// copies used in turn, so that one barrier per sum is enough.
template <int LPR>
struct RowSum {
    float2* red;     // [2][LPR / 64]
    int turn = 0;
    __device__ __forceinline__ float2 operator()(float a, float b) {
        constexpr int kIn = LPR < 64 ? LPR : 64;
#pragma unroll
        for (int o = 1; o < kIn; o <<= 1) {
            a += __shfl_xor(a, o);
            b += __shfl_xor(b, o);
        }
        if constexpr (LPR > 64) {
            constexpr int kW = LPR / 64;
            float2* r = red + turn * kW;
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = make_float2(a, b);
            __syncthreads();
            float2 t = r[0];
#pragma unroll
            for (int w = 1; w < kW; ++w) {
                t.x += r[w].x;
                t.y += r[w].y;
            }
            return t;
        }
        return make_float2(a, b);
    }
};

template <int LPR> constexpr int norm_threads() { return LPR > 256 ? LPR : 256; }

// LPR threads per row, K pieces each: piece j of a thread starts at (j LPR + lane) VEC.
template <typename T, int LPR, int K, bool CENTER>
__global__ __launch_bounds__(norm_threads<LPR>()) void norm_fwd_kernel(
    const T* __restrict__ x, const void* __restrict__ w, const void* __restrict__ bias, bool wbf16,
    NormGeom q, float eps, T* __restrict__ y, float* __restrict__ mean_out,
    float* __restrict__ rstd_out) {
    constexpr int VEC = 16 / (int)sizeof(T);
    constexpr int kRowsWg = norm_threads<LPR>() / LPR;
    __shared__ float2 red[2 * (LPR > 64 ? LPR / 64 : 1)];
    RowSum<LPR> sum{red};
    const int g = blockIdx.y, lane = threadIdx.x % LPR;
    const float inv_n = 1.0f / (float)q.n;

    float wv[K][VEC], bv[K][VEC];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const int c = (j * LPR + lane) * VEC, left = q.n - c;
        const int64_t o = (int64_t)g * q.n + c;
#pragma unroll
        for (int i = 0; i < VEC; ++i) bv[j][i] = 0.f;
        if (wbf16) {
            load_vec<__bf16, VEC>((const __bf16*)w + o, left, wv[j]);
            if (bias) load_vec<__bf16, VEC>((const __bf16*)bias + o, left, bv[j]);
        } else {
            load_vec<float, VEC>((const float*)w + o, left, wv[j]);
            if (bias) load_vec<float, VEC>((const float*)bias + o, left, bv[j]);
        }
    }
    // every thread of a wave goes through the same number of rows (the sums are over lanes)
    const int step = gridDim.x * kRowsWg;
    for (int r0 = blockIdx.x * kRowsWg; r0 < q.rows; r0 += step) {
        const int r = r0 + (int)threadIdx.x / LPR;
        const bool on = r < q.rows;
        const RowAt a = row_at(q, g, on ? r : q.rows - 1);
        const T* xr = x + at(q.xs, a);
        float v[K][VEC];
        float s1 = 0.f;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int c = (j * LPR + lane) * VEC;
            load_vec<T, VEC>(xr + c, q.n - c, v[j]);
        }
        float m = 0.f;
        if constexpr (CENTER) {
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) s1 += v[j][i];
            m = sum(s1, 0.f).x * inv_n;
        }
        float s2 = 0.f;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int left = q.n - (j * LPR + lane) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v[j][i] -= m;
                // (features past the row's end must not count)
                s2 += CENTER && i >= left ? 0.f : v[j][i] * v[j][i];
            }
        }
        const float rstd = 1.0f / sqrtf(sum(s2, 0.f).x * inv_n + eps);
        if (on) {
            const int64_t row = (a.b * q.H + a.h) * q.L + a.l;
            T* yr = y + row * q.n;
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const int c = (j * LPR + lane) * VEC;
                float o[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) o[i] = __builtin_fmaf(v[j][i] * rstd, wv[j][i], bv[j][i]);
                store_vec<T, VEC>(yr + c, q.n - c, o);
            }
            if (lane == 0 && rstd_out) {
                rstd_out[row] = rstd;
                if (CENTER) mean_out[row] = m;
            }
        }
    }
}

template <typename T, int LPR, int K, bool CENTER>
__global__ __launch_bounds__(norm_threads<LPR>()) void norm_bwd_kernel(
    const T* dy, const T* __restrict__ x, const void* __restrict__ w, bool wbf16,
    NormGeom q, const float* __restrict__ mean, const float* __restrict__ rstd, T* dx,
    float* __restrict__ part_w, float* __restrict__ part_b) {
    constexpr int VEC = 16 / (int)sizeof(T);
    constexpr int kThreads = norm_threads<LPR>();
    constexpr int kRowsWg = kThreads / LPR;
    __shared__ float2 red[2 * (LPR > 64 ? LPR / 64 : 1)];
    __shared__ float2 acc_s[LPR > 64 ? 1 : kThreads * K * VEC];
    RowSum<LPR> sum{red};
    const int g = blockIdx.y, lane = threadIdx.x % LPR;
    const float inv_n = 1.0f / (float)q.n;

    float wv[K][VEC], aw[K][VEC], ab[K][VEC];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const int c = (j * LPR + lane) * VEC, left = q.n - c;
        const int64_t o = (int64_t)g * q.n + c;
        if (wbf16) load_vec<__bf16, VEC>((const __bf16*)w + o, left, wv[j]);
        else load_vec<float, VEC>((const float*)w + o, left, wv[j]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) aw[j][i] = ab[j][i] = 0.f;
    }
    const int step = gridDim.x * kRowsWg;
    for (int r0 = blockIdx.x * kRowsWg; r0 < q.rows; r0 += step) {
        const int r = r0 + (int)threadIdx.x / LPR;
        const bool on = r < q.rows;
        const RowAt a = row_at(q, g, on ? r : q.rows - 1);
        const int64_t row = (a.b * q.H + a.h) * q.L + a.l;
        const T* xr = x + at(q.xs, a);
        const T* dyr = dy + at(q.dys, a);
        float xv[K][VEC], gv[K][VEC];
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int c = (j * LPR + lane) * VEC;
            load_vec<T, VEC>(xr + c, q.n - c, xv[j]);
            load_vec<T, VEC>(dyr + c, q.n - c, gv[j]);
        }
        const float m = CENTER ? mean[row] : 0.f, rs = rstd[row];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int left = q.n - (j * LPR + lane) * VEC;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                // (past the row's end dy and w are zero; xh must be too, m may be not finite)
                const float xh = i < left ? (xv[j][i] - m) * rs : 0.f;
                xv[j][i] = xh;
                if (on) {
                    aw[j][i] = __builtin_fmaf(gv[j][i], xh, aw[j][i]);
                    ab[j][i] += gv[j][i];
                }
                gv[j][i] *= wv[j][i];
                s1 += gv[j][i];
                s2 = __builtin_fmaf(gv[j][i], xh, s2);
            }
        }
        const float2 t = sum(CENTER ? s1 : 0.f, s2);
        const float m1 = CENTER ? t.x * inv_n : 0.f, m2 = t.y * inv_n;
        if (on) {
            T* dxr = dx + at(q.dxs, a);
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const int c = (j * LPR + lane) * VEC;
                float o[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    o[i] = rs * (gv[j][i] - m1 - xv[j][i] * m2);
                store_vec<T, VEC>(dxr + c, q.n - c, o);
            }
        }
    }
    // the workgroup's sums over its rows: [group][workgroup][n]
    const int64_t out = ((int64_t)g * gridDim.x + blockIdx.x) * q.n;
    if constexpr (LPR > 64) {
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int c = (j * LPR + lane) * VEC;
            store_vec<float, VEC>(part_w + out + c, q.n - c, aw[j]);
            if (part_b) store_vec<float, VEC>(part_b + out + c, q.n - c, ab[j]);
        }
    } else {
        const int sub = threadIdx.x / LPR;
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                acc_s[(sub * K * VEC + j * VEC + i) * LPR + lane] = make_float2(aw[j][i], ab[j][i]);
        __syncthreads();
        for (int e = threadIdx.x; e < K * VEC * LPR; e += kThreads) {
            const int ji = e / LPR, ln = e % LPR;
            const int col = ((ji / VEC) * LPR + ln) * VEC + ji % VEC;
            if (col >= q.n) continue;
            float2 t = acc_s[e];
            for (int k = 1; k < kRowsWg; ++k) {
                const float2 u = acc_s[k * K * VEC * LPR + e];
                t.x += u.x;
                t.y += u.y;
            }
            part_w[out + col] = t.x;
            if (part_b) part_b[out + col] = t.y;
        }
    }
}

// out[g][c] = sum over k of part[g][k][c]: 16 columns by 64 rows of threads, then the 64
// sums in LDS, in a fixed order
__global__ __launch_bounds__(1024) void norm_sum_kernel(
    const float* __restrict__ part_w, const float* __restrict__ part_b, int parts, int n,
    float* __restrict__ dw, float* __restrict__ db) {
    __shared__ float s[64][17];
    const float* part = blockIdx.z ? part_b : part_w;
    float* out = blockIdx.z ? db : dw;
    const int g = blockIdx.y, c = blockIdx.x * 16 + (threadIdx.x & 15), k0 = threadIdx.x >> 4;
    float t = 0.f;
    if (c < n)
        for (int k = k0; k < parts; k += 64) t += part[((int64_t)g * parts + k) * n + c];
    s[k0][threadIdx.x & 15] = t;
    __syncthreads();
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        if (k0 < o) s[k0][threadIdx.x & 15] += s[k0 + o][threadIdx.x & 15];
        __syncthreads();
    }
    if (k0 == 0 && c < n) out[(int64_t)g * n + c] = s[0][threadIdx.x];
}

struct Shape {
    int lpr, k;
};
// Threads per row and 16-byte pieces per thread: the fewest lanes that hold the row in one
// piece each, then a wave with up to 4 pieces, then workgroups.
Shape norm_shape(int n, int vec) {
    const int pieces = (n + vec - 1) / vec;
    for (int lpr = 8; lpr <= 64; lpr *= 2)
        if (pieces <= lpr) return {lpr, 1};
    for (int k = 2; k <= 4; ++k)
        if (pieces <= 64 * k) return {64, k};
    if (pieces <= 512) return {256, 2};
    if (pieces <= 1024) return {256, 4};
    if (pieces <= 2048) return {1024, 2};
    return {1024, 4};
}

// Workgroups per weight row of a backward pass: enough to fill the chip, each with at
// least 8 rows per row slot where there are that many.
int norm_parts(int rows, int groups, int n) {
    const Shape sh = norm_shape(n, 4);   // (the same count for both types)
    const int per = sh.lpr > 256 ? 1 : 256 / sh.lpr;
    const int most = kMaxBlocksNorm / groups > 0 ? kMaxBlocksNorm / groups : 1;
    const int want = (rows + 8 * per - 1) / (8 * per);
    return want < most ? want : most;
}

template <typename T, bool CENTER, typename F>
void with_shape(int n, F f) {
    const Shape s = norm_shape(n, 16 / (int)sizeof(T));
#define ACP_SHAPE(LPR, K) \
    if (s.lpr == LPR && s.k == K) return f(std::integral_constant<int, LPR>{}, std::integral_constant<int, K>{});
    ACP_SHAPE(8, 1) ACP_SHAPE(16, 1) ACP_SHAPE(32, 1) ACP_SHAPE(64, 1) ACP_SHAPE(64, 2)
    ACP_SHAPE(64, 3) ACP_SHAPE(64, 4) ACP_SHAPE(256, 2) ACP_SHAPE(256, 4) ACP_SHAPE(1024, 2)
    ACP_SHAPE(1024, 4)
#undef ACP_SHAPE
}

NormGeom geom(const NormArgs& a) {
    NormGeom q{};
    q.xs = a.xs; q.dys = a.dys; q.dxs = a.dxs;
    q.H = a.H; q.L = a.L; q.n = a.n;
    q.groups = a.per_head ? a.H : 1;
    q.rows = a.B * a.L * (a.per_head ? 1 : a.H);
    return q;
}

template <typename T, bool CENTER>
void fwd(const NormArgs& a, hipStream_t s) {
    const NormGeom q = geom(a);
    with_shape<T, CENTER>(a.n, [&](auto lpr, auto k) {
        constexpr int LPR = decltype(lpr)::value, K = decltype(k)::value;
        constexpr int kThreads = norm_threads<LPR>(), kRows = kThreads / LPR;
        const int most = (8192 + q.groups - 1) / q.groups;
        const int want = (q.rows + kRows - 1) / kRows;
        hipLaunchKernelGGL((norm_fwd_kernel<T, LPR, K, CENTER>), dim3(want < most ? want : most, q.groups),
                           dim3(kThreads), 0, s, (const T*)a.x, a.weight, a.bias, a.wbf16, q, a.eps,
                           (T*)a.y, a.mean, a.rstd);
    });
}

template <typename T, bool CENTER>
void bwd(const NormArgs& a, hipStream_t s) {
    const NormGeom q = geom(a);
    const int parts = norm_parts(q.rows, q.groups, a.n);
    float* part_b = a.dbias ? a.part + (size_t)q.groups * parts * a.n : nullptr;
    if (parts > 0) with_shape<T, CENTER>(a.n, [&](auto lpr, auto k) {   // (no row: zero sums)
        constexpr int LPR = decltype(lpr)::value, K = decltype(k)::value;
        hipLaunchKernelGGL((norm_bwd_kernel<T, LPR, K, CENTER>), dim3(parts, q.groups),
                           dim3(norm_threads<LPR>()), 0, s, (const T*)a.dy, (const T*)a.x, a.weight,
                           a.wbf16, q, a.mean, a.rstd, (T*)a.y, a.part, part_b);
    });
    hipLaunchKernelGGL(norm_sum_kernel, dim3((a.n + 15) / 16, q.groups, a.dbias ? 2 : 1), dim3(1024), 0,
                       s, a.part, part_b, parts, a.n, a.dweight, a.dbias);
}

}  // namespace

size_t norm_workspace(int B, int H, int L, int n, bool per_head) {
    const int groups = per_head ? H : 1, rows = B * L * (per_head ? 1 : H);
    return (size_t)2 * groups * norm_parts(rows, groups, n) * n * sizeof(float);
}

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t s) {
    trace_begin(ACP_K_COUNT + ACP_OP_NORM, s);
    if (a.bf16) a.center ? fwd<__bf16, true>(a, s) : fwd<__bf16, false>(a, s);
    else a.center ? fwd<float, true>(a, s) : fwd<float, false>(a, s);
    const hipError_t e = hipGetLastError();
    trace_end(ACP_K_COUNT + ACP_OP_NORM, s);
    return e;
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t s) {
    trace_begin(ACP_K_COUNT + ACP_OP_NORM_BWD, s);
    if (a.bf16) a.center ? bwd<__bf16, true>(a, s) : bwd<__bf16, false>(a, s);
    else a.center ? bwd<float, true>(a, s) : bwd<float, false>(a, s);
    const hipError_t e = hipGetLastError();
    trace_end(ACP_K_COUNT + ACP_OP_NORM_BWD, s);
    return e;
}

}  // namespace acp
