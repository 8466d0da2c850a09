// Layer norm and RMS norm of rows, forward and backward.
//
// A row is held in registers by the threads that share it (8 lanes to 1024 threads, each
// with up to 4 pieces of 16 bytes), so that it is read once and the mean is known before
// the squares of the centred row are summed.  Both passes are bound by memory: forward
// reads x and writes y, backward reads x and dy and writes dx.  The weight's gradient
// stays in registers while a workgroup goes through its rows; it leaves one row of
// partial sums per workgroup, and a second launch adds these in a fixed order.
//
// Above 8192 features a thread of the backward pass needs more than the 128 registers that 1024 threads
// leave it: 6 to 45 spill in bfloat16, 33 to 90 in float32.  Gradients of 2048 x 16384 take 50 us (layer
// norm 68), in float32 124 (129), where 4096 x 8192 takes 43 (52) and 80 (85), inputs used again and again.
//
// Layer norm of 32768 x 768 in bfloat16: forward 19 us (5.3 TB/s), backward 31 us (4.9 TB/s),
// sums 4.6 us; the QK-norm of 8 x 12 x 4096 x 64 18, 26 and 4 us.
#include <type_traits>

#include "acp_device.h"
#include "acp_ops_internal.h"

namespace acp {
namespace {

constexpr int kMaxBlocksNorm = 1024;   // workgroups of 256 threads of a backward pass, at most
constexpr int kFwdBlocks = 4096;       // and of a forward pass

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

// 16 bytes of a row, as loaded
template <typename T>
struct Piece {
    static constexpr int VEC = 16 / (int)sizeof(T);
    T v[VEC];
};

// How a row's features are cut into pieces.
//   kWhole    n is a multiple of the piece
//   kShifted  the last piece ends with the row and repeats `skip` features of the one before:
//             both threads form the same values of these, the sums leave them out once
//   kShort    n is less than a piece: the first thread has all of it, feature by feature
enum Cut { kWhole, kShifted, kShort };

// Piece number i of a row of n
template <int CUT, int VEC>
struct Span {
    int c, skip;       // first feature, features of it that another piece has too
    int left;          // features from c to the row's end; 0 or less: no piece
    __device__ __forceinline__ Span(int i, int n) {
        c = i * VEC;
        left = n - c;
        skip = 0;
        if (CUT == kShifted && left > 0 && left < VEC) {
            skip = VEC - left;
            c -= skip;
            left = VEC;
        }
    }
    // whether the sums take element e
    __device__ __forceinline__ bool counts(int e) const {
        return CUT == kShort ? e < left : left > 0 && (CUT == kWhole || e >= skip);
    }
};

// The piece at p + its first feature (aligned to the element only; gfx950 loads it in one
// instruction all the same); zeros past the row's end
template <int CUT, typename T>
__device__ __forceinline__ Piece<T> load_piece(const T* p, const Span<CUT, 16 / sizeof(T)>& at) {
    Piece<T> t;
    if (CUT != kShort && at.left > 0) {
        __builtin_memcpy(&t, p + at.c, 16);
    } else {
#pragma unroll
        for (int i = 0; i < Piece<T>::VEC; ++i)
            t.v[i] = CUT == kShort && i < at.left ? p[at.c + i] : from_f32<T>(0.f);
    }
    return t;
}
template <int CUT, typename T>
__device__ __forceinline__ void store_piece(T* p, const Span<CUT, 16 / sizeof(T)>& at,
                                            const float (&v)[16 / sizeof(T)]) {
    constexpr int VEC = 16 / (int)sizeof(T);
    Piece<T> t;
#pragma unroll
    for (int i = 0; i < VEC; ++i) t.v[i] = from_f32<T>(v[i]);
    if (CUT != kShort && at.left > 0) {
        __builtin_memcpy(p + at.c, &t, 16);
    } else if (CUT == kShort) {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < at.left) p[at.c + i] = t.v[i];
    }
}
// Its weights, from the weight row at `row`
template <int CUT, int VEC>
__device__ __forceinline__ void load_weights(const void* w, bool wbf16, int64_t row, const Span<CUT, VEC>& at,
                                             float (&v)[VEC]) {
    row += at.c;
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = 0.f;
    if (CUT != kShort && at.left > 0) {
        if (wbf16) {
            __bf16 t[VEC];
            __builtin_memcpy(t, (const __bf16*)w + row, sizeof(t));
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = (float)t[i];
        } else {
            __builtin_memcpy(v, (const float*)w + row, sizeof(v));
        }
    } else if (CUT == kShort) {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < at.left) v[i] = wbf16 ? (float)((const __bf16*)w)[row + i] : ((const float*)w)[row + i];
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

template <int LPR> constexpr int norm_threads() { return LPR > 64 ? LPR : 256; }

// LPR threads per row, K pieces each: piece j of a thread starts at (j LPR + lane) VEC.  A
// row's pieces are requested while the row before it is worked on.
template <typename T, int LPR, int K, bool CENTER, int CUT>
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
    const int step = gridDim.x * kRowsWg, sub = (int)threadIdx.x / LPR;

    auto span = [&](int j) __attribute__((always_inline)) { return Span<CUT, VEC>(j * LPR + lane, q.n); };
    Piece<T> next[K];
    RowAt an;
    auto bring = [&](int r) __attribute__((always_inline)) {
        an = row_at(q, g, min(r, q.rows - 1));
        const T* xr = x + at(q.xs, an);
#pragma unroll
        for (int j = 0; j < K; ++j) next[j] = load_piece(xr, span(j));
    };
    int r0 = blockIdx.x * kRowsWg;
    if (r0 < q.rows) bring(r0 + sub);
    float wv[K][VEC], bv[K][VEC];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        load_weights(w, wbf16, (int64_t)g * q.n, span(j), wv[j]);
        if (bias) load_weights(bias, wbf16, (int64_t)g * q.n, span(j), bv[j]);
        else
#pragma unroll
            for (int i = 0; i < VEC; ++i) bv[j][i] = 0.f;
    }
    // every thread of a wave goes through the same number of rows (the sums are over lanes)
    for (; r0 < q.rows; r0 += step) {
        const bool on = r0 + sub < q.rows;
        const RowAt a = an;
        float v[K][VEC];
        float s1 = 0.f;
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[j][i] = to_f32(next[j].v[i]);
        if (r0 + step < q.rows) bring(r0 + step + sub);
        float m = 0.f;
        if constexpr (CENTER) {
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i) s1 += CUT != kShifted || span(j).counts(i) ? v[j][i] : 0.f;
            m = sum(s1, 0.f).x * inv_n;
        }
        float s2 = 0.f;
#pragma unroll
        for (int j = 0; j < K; ++j) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v[j][i] -= m;
                // (features past the row's end are zeros, and -m when centred)
                if ((!CENTER && CUT != kShifted) || span(j).counts(i)) s2 += v[j][i] * v[j][i];
            }
        }
        const float rstd = 1.0f / sqrtf(sum(s2, 0.f).x * inv_n + eps);
        if (on) {
            const int64_t row = (a.b * q.H + a.h) * q.L + a.l;
            T* yr = y + row * q.n;
#pragma unroll
            for (int j = 0; j < K; ++j) {
                float o[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) o[i] = __builtin_fmaf(v[j][i] * rstd, wv[j][i], bv[j][i]);
                store_piece(yr, span(j), o);
            }
            if (lane == 0 && rstd_out) {
                rstd_out[row] = rstd;
                if (CENTER) mean_out[row] = m;
            }
        }
    }
}

template <typename T, int LPR, int K, bool CENTER, int CUT>
__global__ __launch_bounds__(norm_threads<LPR>()) void norm_bwd_kernel(
    const T* dy, const T* __restrict__ x, const void* __restrict__ w, bool wbf16,
    NormGeom q, const float* __restrict__ mean, const float* __restrict__ rstd, T* dx,
    float* __restrict__ part_w, float* __restrict__ part_b) {
    constexpr int VEC = 16 / (int)sizeof(T);
    constexpr int kThreads = norm_threads<LPR>();
    constexpr int kRowsWg = kThreads / LPR;
    __shared__ float2 red[2 * (LPR > 64 ? LPR / 64 : 1)];
    __shared__ float acc_s[LPR > 64 ? 1 : kThreads * K * VEC];
    RowSum<LPR> sum{red};
    const int g = blockIdx.y, lane = threadIdx.x % LPR;
    const float inv_n = 1.0f / (float)q.n;
    const int step = gridDim.x * kRowsWg, sub = (int)threadIdx.x / LPR;

    auto span = [&](int j) __attribute__((always_inline)) { return Span<CUT, VEC>(j * LPR + lane, q.n); };
    Piece<T> xn[K], gn[K];
    float mn = 0.f, rn = 0.f;
    RowAt an;
    auto bring = [&](int r) __attribute__((always_inline)) {
        an = row_at(q, g, min(r, q.rows - 1));
        const T* xr = x + at(q.xs, an);
        const T* dyr = dy + at(q.dys, an);
#pragma unroll
        for (int j = 0; j < K; ++j) {
            xn[j] = load_piece(xr, span(j));
            gn[j] = load_piece(dyr, span(j));
        }
        const int64_t row = (an.b * q.H + an.h) * q.L + an.l;
        if (CENTER) mn = mean[row];
        rn = rstd[row];
    };
    int r0 = blockIdx.x * kRowsWg;
    if (r0 < q.rows) bring(r0 + sub);
    float wv[K][VEC], aw[K][VEC], ab[K][VEC];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        load_weights(w, wbf16, (int64_t)g * q.n, span(j), wv[j]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) aw[j][i] = ab[j][i] = 0.f;
    }
    for (; r0 < q.rows; r0 += step) {
        const bool on = r0 + sub < q.rows;
        const RowAt a = an;
        float xv[K][VEC], gv[K][VEC];
        const float m = mn, rs = rn;
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                xv[j][i] = to_f32(xn[j].v[i]);
                gv[j][i] = on ? to_f32(gn[j].v[i]) : 0.f;   // (a row past the last adds nothing)
            }
        if (r0 + step < q.rows) bring(r0 + step + sub);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < K; ++j) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                // (past the row's end dy and w are zero; xh must be too, m may be not finite)
                const float xh = (CUT == kShort ? i < span(j).left : span(j).left > 0) && on ? (xv[j][i] - m) * rs
                                                                                            : 0.f;
                xv[j][i] = xh;
                aw[j][i] = __builtin_fmaf(gv[j][i], xh, aw[j][i]);
                ab[j][i] += gv[j][i];
                gv[j][i] *= wv[j][i];
                const float gs = CUT != kShifted || span(j).counts(i) ? gv[j][i] : 0.f;
                s1 += gs;
                s2 = __builtin_fmaf(gs, xh, s2);
            }
        }
        const float2 t = sum(CENTER ? s1 : 0.f, s2);
        const float m1 = CENTER ? t.x * inv_n : 0.f, m2 = t.y * inv_n;
        if (on) {
            T* dxr = dx + at(q.dxs, a);
#pragma unroll
            for (int j = 0; j < K; ++j) {
                float o[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    o[i] = rs * (gv[j][i] - m1 - xv[j][i] * m2);
                store_piece(dxr, span(j), o);
            }
        }
    }
    // the workgroup's sums over its rows: [group][workgroup][n]
    const int64_t out = ((int64_t)g * gridDim.x + blockIdx.x) * q.n;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        float* part = b ? part_b : part_w;
        if (part == nullptr) break;
        float (&acc)[K][VEC] = b ? ab : aw;
        if constexpr (LPR > 64) {
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (span(j).counts(i)) part[out + span(j).c + i] = acc[j][i];
        } else {
            if (b) __syncthreads();
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (span(j).counts(i)) acc_s[((sub * K + j) * VEC + i - span(j).skip) * LPR + lane] = acc[j][i];
            __syncthreads();
            // (i fastest, so that the stores are contiguous)
            for (int e = threadIdx.x; e < K * VEC * LPR; e += kThreads) {
                if (e >= q.n) break;
                const int i = e % VEC, ln = e / VEC % LPR, j = e / (VEC * LPR);
                const int o = (j * VEC + i) * LPR + ln;
                float t = acc_s[o];
                for (int k = 1; k < kRowsWg; ++k) t += acc_s[k * K * VEC * LPR + o];
                part[out + e] = t;
            }
        }
    }
}

// out[g][c] = sum over k of part[g][k][c]: 16 columns by 64 rows of threads, then the 64
// sums in LDS, in a fixed order
__global__ __launch_bounds__(1024) void norm_sum_kernel(
    const float* __restrict__ part_w, const float* __restrict__ part_b, int parts, int n,
    float* __restrict__ dw, float* __restrict__ db) {
    constexpr int kAtOnce = 8;
    __shared__ float s[64][17];
    const float* part = blockIdx.z ? part_b : part_w;
    float* out = blockIdx.z ? db : dw;
    const int g = blockIdx.y, c = blockIdx.x * 16 + (threadIdx.x & 15), k0 = threadIdx.x >> 4;
    float t = 0.f;
    if (c < n)
        // (kAtOnce loads in flight)
        for (int k = k0; k < parts; k += 64 * kAtOnce) {
            float v[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
                v[i] = part[((int64_t)g * parts + min(k + 64 * i, parts - 1)) * n + c];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
                if (k + 64 * i < parts) t += v[i];
        }
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
// Threads per row and 16-byte pieces per thread: lanes of a wave while they need up to 2
// pieces (3 where that leaves fewer lanes idle), a workgroup with 2 pieces each beyond (4
// pieces: 130 and more registers in the backward pass; a step of 8192 x 2048 in bfloat16 61
// us instead of 41).
Shape norm_shape(int n, int vec) {
    const int pieces = (n + vec - 1) / vec;
    if (pieces <= 8) return {8, 1};
    if (pieces <= 16) return {16, 1};
    if (pieces <= 32) return {32, 1};
    if (pieces <= 64) return {64, 1};
    if (pieces <= 96) return {32, 3};
    if (pieces <= 128) return {64, 2};
    if (pieces <= 256) return {128, 2};
    if (pieces <= 512) return {256, 2};
    if (pieces <= 1024) return {512, 2};
    if (pieces <= 2048) return {1024, 2};
    return {1024, 4};
}

// Workgroups per weight row of a backward pass: each row slot gets at least 4 rows, and a
// launch at most 1024 workgroups (fewer of larger ones), which fill the chip
int norm_parts(int rows, int groups, int n, int vec) {
    const Shape sh = norm_shape(n, vec);
    const int threads = sh.lpr > 64 ? sh.lpr : 256, per = threads / sh.lpr;
    const int fill = kMaxBlocksNorm * 256 / (threads > 256 ? threads : 256);
    const int most = fill / groups > 0 ? fill / groups : 1;
    const int want = (rows + 4 * per - 1) / (4 * per);
    return want < most ? want : most;
}

template <typename T, int CUT, typename F>
void with_shape(int n, F f) {
    const Shape s = norm_shape(n, 16 / (int)sizeof(T));
#define ACP_SHAPE(LPR, K) \
    if (s.lpr == LPR && s.k == K) return f(std::integral_constant<int, LPR>{}, std::integral_constant<int, K>{});
    ACP_SHAPE(8, 1)
    if constexpr (CUT != kShort) {
        ACP_SHAPE(16, 1) ACP_SHAPE(32, 1) ACP_SHAPE(32, 3) ACP_SHAPE(64, 1) ACP_SHAPE(64, 2)
        ACP_SHAPE(128, 2) ACP_SHAPE(256, 2) ACP_SHAPE(512, 2) ACP_SHAPE(1024, 2)
        if constexpr (sizeof(T) == 4) { ACP_SHAPE(1024, 4) }      // (n up to 16384)
    }
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

template <typename T, bool CENTER, int CUT>
void fwd(const NormArgs& a, hipStream_t s) {
    const NormGeom q = geom(a);
    with_shape<T, CUT>(a.n, [&](auto lpr, auto k) {
        constexpr int LPR = decltype(lpr)::value, K = decltype(k)::value;
        constexpr int kThreads = norm_threads<LPR>(), kRows = kThreads / LPR;
        const int most = (kFwdBlocks * 256 / kThreads + q.groups - 1) / q.groups;
        const int want = (q.rows + kRows - 1) / kRows;
        hipLaunchKernelGGL((norm_fwd_kernel<T, LPR, K, CENTER, CUT>), dim3(want < most ? want : most, q.groups),
                           dim3(kThreads), 0, s, (const T*)a.x, a.weight, a.bias, a.wbf16, q, a.eps,
                           (T*)a.y, a.mean, a.rstd);
    });
}

template <typename T, bool CENTER, int CUT>
void bwd(const NormArgs& a, hipStream_t s) {
    const NormGeom q = geom(a);
    const int parts = norm_parts(q.rows, q.groups, a.n, 16 / (int)sizeof(T));
    float* part_b = a.dbias ? a.part + (size_t)q.groups * parts * a.n : nullptr;
    if (parts > 0) with_shape<T, CUT>(a.n, [&](auto lpr, auto k) {   // (no row: zero sums)
        constexpr int LPR = decltype(lpr)::value, K = decltype(k)::value;
        hipLaunchKernelGGL((norm_bwd_kernel<T, LPR, K, CENTER, CUT>), dim3(parts, q.groups),
                           dim3(norm_threads<LPR>()), 0, s, (const T*)a.dy, (const T*)a.x, a.weight,
                           a.wbf16, q, a.mean, a.rstd, (T*)a.y, a.part, part_b);
    });
    hipLaunchKernelGGL(norm_sum_kernel, dim3((a.n + 15) / 16, q.groups, a.dbias ? 2 : 1), dim3(1024), 0,
                       s, a.part, part_b, parts, a.n, a.dweight, a.dbias);
}

// f(CENTER, CUT) for a call
template <typename T, typename F>
void with_cut(const NormArgs& a, F f) {
    constexpr int VEC = 16 / (int)sizeof(T);
    auto cut = [&](auto center) {
        if (a.n < VEC) f(center, std::integral_constant<int, kShort>{});
        else if (a.n % VEC) f(center, std::integral_constant<int, kShifted>{});
        else f(center, std::integral_constant<int, kWhole>{});
    };
    if (a.center) cut(std::true_type{});
    else cut(std::false_type{});
}
template <typename T>
void fwd(const NormArgs& a, hipStream_t s) {
    with_cut<T>(a, [&](auto center, auto cut) { fwd<T, decltype(center)::value, decltype(cut)::value>(a, s); });
}
template <typename T>
void bwd(const NormArgs& a, hipStream_t s) {
    with_cut<T>(a, [&](auto center, auto cut) { bwd<T, decltype(center)::value, decltype(cut)::value>(a, s); });
}

}  // namespace

// (the larger of the two types' counts: the size does not depend on the type)
size_t norm_workspace(int B, int H, int L, int n, bool per_head) {
    const int groups = per_head ? H : 1, rows = B * L * (per_head ? 1 : H);
    const int p4 = norm_parts(rows, groups, n, 4), p8 = norm_parts(rows, groups, n, 8);
    return (size_t)2 * groups * (p4 > p8 ? p4 : p8) * n * sizeof(float);
}

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t s) {
    trace_begin(ACP_K_COUNT + ACP_OP_NORM, s);
    if (a.bf16) fwd<__bf16>(a, s);
    else fwd<float>(a, s);
    const hipError_t e = hipGetLastError();
    trace_end(ACP_K_COUNT + ACP_OP_NORM, s);
    return e;
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t s) {
    trace_begin(ACP_K_COUNT + ACP_OP_NORM_BWD, s);
    if (a.bf16) bwd<__bf16>(a, s);
    else bwd<float>(a, s);
    const hipError_t e = hipGetLastError();
    trace_end(ACP_K_COUNT + ACP_OP_NORM_BWD, s);
    return e;
}

}  // namespace acp
