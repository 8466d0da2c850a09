// Rotary positions of queries and keys, and their gradient (the negative angle).
//
// Bound by memory: every feature is read and written once.  A thread takes one position
// and one chunk of pairs (16 bytes of each half, or 32 contiguous bytes interleaved),
// forms the chunk's sines and cosines once and turns that chunk of several heads: the
// angles depend on the position alone.  Angles are p f_i in turns, reduced to [-1/2, 1/2]
// in float64 (exact to 2^-53 of the angle), so that sine and cosine are those of the true
// angle at any position below 2^31.
#include "acp_device.h"
#include "acp_ops_internal.h"

namespace acp {
namespace {

struct RotaryKernelArgs {
    RotaryArgs a;
    int chunks;              // of pairs, per position
    int copies;              // chunks of features that are not turned
    int split;               // threads that share the heads of a position's chunk
};

template <typename T, int VEC>
__device__ __forceinline__ void get(const T* p, int left, T (&v)[VEC]) {
    if (left >= VEC) __builtin_memcpy(v, p, sizeof(v));
    else
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < left) v[i] = p[i];
}
template <typename T, int VEC>
__device__ __forceinline__ void put(T* p, int left, const T (&v)[VEC]) {
    if (left >= VEC) __builtin_memcpy(p, v, sizeof(v));
    else
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < left) p[i] = v[i];
}

template <typename T, bool INTER>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryKernelArgs ka, int64_t items) {
    constexpr int C = 16 / (int)sizeof(T);      // pairs per chunk
    const RotaryArgs& a = ka.a;
    const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (item >= items) return;
    const int per = ka.chunks + ka.copies;
    const int64_t bl = item / per;
    const int ch = (int)(item - bl * per);
    const int b = (int)(bl / a.L), l = (int)(bl - (int64_t)b * a.L);
    const int both = a.heads[0] + a.heads[1];
    const int h0 = (int)((int64_t)both * blockIdx.y / ka.split);
    const int h1 = (int)((int64_t)both * (blockIdx.y + 1) / ka.split);

    auto src = [&](int h) {
        const int w = h >= a.heads[0];
        const Strides& s = a.xs[w];
        return (const T*)a.x[w] + b * s.b + (int64_t)(h - (w ? a.heads[0] : 0)) * s.h + l * s.l;
    };
    auto dst = [&](int h) {
        const int w = h >= a.heads[0];
        const Strides& s = a.ys[w];
        return (T*)a.y[w] + b * s.b + (int64_t)(h - (w ? a.heads[0] : 0)) * s.h + l * s.l;
    };

    if (ch >= ka.chunks) {
        const int e = a.rot + (ch - ka.chunks) * 2 * C, left = a.d - e;
        for (int h = h0; h < h1; ++h) {
            T v[2 * C];
            get<T, 2 * C>(src(h) + e, left, v);
            put<T, 2 * C>(dst(h) + e, left, v);
        }
        return;
    }
    int64_t p = a.start + l;
    if (a.pos) {
        const int64_t o = b * a.pos_b + l * a.pos_l;
        p = a.pos_bytes == 4 ? ((const int*)a.pos)[o] : ((const int64_t*)a.pos)[o];
    }
    const int half = a.rot / 2, i0 = ch * C, left = half - i0;
    float cs[C], sn[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const double t = (double)p * a.turns[min(i0 + i, half - 1)];
        float s, c;
        sincospif(2.0f * (float)(t - rint(t)), &s, &c);
        cs[i] = c * a.amplitude;
        sn[i] = (a.inverse ? -s : s) * a.amplitude;
    }
    for (int h = h0; h < h1; ++h) {
        const T* x = src(h);
        T* y = dst(h);
        if constexpr (INTER) {
            T v[2 * C];
            get<T, 2 * C>(x + 2 * i0, 2 * left, v);
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const float u = to_f32(v[2 * i]), w = to_f32(v[2 * i + 1]);
                v[2 * i] = from_f32<T>(u * cs[i] - w * sn[i]);
                v[2 * i + 1] = from_f32<T>(u * sn[i] + w * cs[i]);
            }
            put<T, 2 * C>(y + 2 * i0, 2 * left, v);
        } else {
            T v[C], z[C];
            get<T, C>(x + i0, left, v);
            get<T, C>(x + half + i0, left, z);
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const float u = to_f32(v[i]), w = to_f32(z[i]);
                v[i] = from_f32<T>(u * cs[i] - w * sn[i]);
                z[i] = from_f32<T>(u * sn[i] + w * cs[i]);
            }
            put<T, C>(y + i0, left, v);
            put<T, C>(y + half + i0, left, z);
        }
    }
}

template <typename T>
void rotary(const RotaryArgs& a, hipStream_t s) {
    constexpr int C = 16 / (int)sizeof(T);
    RotaryKernelArgs k{a, 0, 0, 1};
    k.chunks = (a.rot / 2 + C - 1) / C;
    // (a tensor turned in place needs no copy of the rest; both must be)
    bool in_place = true;
    for (int w = 0; w < 2; ++w)
        if (a.x[w] && a.x[w] != a.y[w]) in_place = false;
    k.copies = in_place ? 0 : (a.d - a.rot + 2 * C - 1) / (2 * C);
    const int64_t items = (int64_t)a.B * a.L * (k.chunks + k.copies);
    const int both = a.heads[0] + a.heads[1];
    // heads shared among threads until the chip is full (256 CUs x 2048 threads)
    const int64_t want = ((int64_t)256 * 2048 + items - 1) / items;
    k.split = want < both ? (int)want : both;
    const dim3 grid((unsigned)((items + 255) / 256), k.split);
    if (a.interleaved) hipLaunchKernelGGL((rotary_kernel<T, true>), grid, dim3(256), 0, s, k, items);
    else hipLaunchKernelGGL((rotary_kernel<T, false>), grid, dim3(256), 0, s, k, items);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t s) {
    trace_begin(ACP_K_COUNT + ACP_OP_ROTARY, s);
    if (a.bf16) rotary<__bf16>(a, s);
    else rotary<float>(a, s);
    const hipError_t e = hipGetLastError();
    trace_end(ACP_K_COUNT + ACP_OP_ROTARY, s);
    return e;
}

}  // namespace acp
