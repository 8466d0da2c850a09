// Rotary positions of queries and keys, and their gradient (the negative angle).
//
// Bound by memory: every feature is read and written once.  A thread takes one position
// and one chunk of pairs (16 bytes of each half, or 32 contiguous bytes interleaved),
// forms the chunk's sines and cosines once and turns that chunk of several heads: the
// angles depend on the position alone.  Angles are p f_i in turns, reduced to [-1/2, 1/2]
// in float64 (exact to 2^-53 of the angle), so that none is lost at any position below 2^31.  What is
// left is rounded to float32 for the sine and cosine, off by at most 2^-26 turns, 9.4e-8 of a
// pair's size: nothing beside bfloat16's 2^-9, and half as much again as the rounding of a float32
// output.  q and k of 8 x 12 x 4096 x 64 in bfloat16 take 43 us (4.7
// TB/s), of 30001 positions of 20 heads of 128, 96 of them turned, 60 us (5.1 TB/s).
#include <type_traits>

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

// VEC features from p, aligned to the element only (gfx950 moves them in one instruction all
// the same).  FULL: all are inside the row, else the first `left`.
template <bool FULL, typename T, int VEC>
__device__ __forceinline__ void get(const T* p, int left, T (&v)[VEC]) {
    if (FULL || left >= VEC) __builtin_memcpy(v, p, sizeof(v));
    else
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < left) v[i] = p[i];
}
template <bool FULL, typename T, int VEC>
__device__ __forceinline__ void put(T* p, int left, const T (&v)[VEC]) {
    if (FULL || left >= VEC) __builtin_memcpy(p, v, sizeof(v));
    else
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i < left) p[i] = v[i];
}

template <typename T, bool INTER, bool FULL>
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

    // the thread's position in each tensor; head h of the two together
    const T* xb[2];
    T* yb[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        xb[w] = (const T*)a.x[w] + b * a.xs[w].b + l * a.xs[w].l;
        yb[w] = (T*)a.y[w] + b * a.ys[w].b + l * a.ys[w].l;
    }
    auto src = [&](int h) __attribute__((always_inline)) {
        return h < a.heads[0] ? xb[0] + h * a.xs[0].h : xb[1] + (h - a.heads[0]) * a.xs[1].h;
    };
    auto dst = [&](int h) __attribute__((always_inline)) {
        return h < a.heads[0] ? yb[0] + h * a.ys[0].h : yb[1] + (h - a.heads[0]) * a.ys[1].h;
    };

    int64_t p = a.start + l;
    if (a.pos) {
        const int64_t o = b * a.pos_b + l * a.pos_l;
        p = a.pos_bytes == 4 ? ((const int*)a.pos)[o] : ((const int64_t*)a.pos)[o];
    }
    // The chunk's two vectors of C features: of a chunk of pairs or of one that is copied.
    // FULL: the last chunk of either kind may start earlier and repeat part of the one before
    const int half = a.rot / 2;
    const bool copy = ch >= ka.chunks;
    int i0 = ch * C, e = a.rot + (ch - ka.chunks) * 2 * C;
    if (FULL) {
        i0 = min(i0, half - C);
        e = min(e, a.d - 2 * C);
    }
    const int off = copy ? e : INTER ? 2 * i0 : i0, far = copy || INTER ? C : half;
    const int left_a = copy ? a.d - e : INTER ? a.rot - 2 * i0 : half - i0;
    const int left_b = copy || INTER ? left_a - C : left_a;
    float cs[C], sn[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const double t = (double)p * a.turns[min(max(i0 + i, 0), half - 1)];
        float s, c;
        sincospif(2.0f * (float)(t - rint(t)), &s, &c);
        cs[i] = c * a.amplitude;
        sn[i] = (a.inverse ? -s : s) * a.amplitude;
    }
    // Several heads at a time, all loads before the first store (which could be of the same
    // memory, for all the compiler knows)
    auto group = [&](auto count, int hb) __attribute__((always_inline)) {
        constexpr int N = decltype(count)::value;
        T v[N][C], z[N][C];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const T* x = src(hb + k) + off;
            get<FULL>(x, left_a, v[k]);
            get<FULL>(x + far, left_b, z[k]);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            T o[2 * C];
#pragma unroll
            for (int i = 0; i < C; ++i) {
                // pair i: interleaved, features 2 i and 2 i + 1 of the 2 C in v and z
                const float u = to_f32(!INTER ? v[k][i] : 2 * i < C ? v[k][2 * i % C] : z[k][2 * i % C]);
                const float w = to_f32(!INTER ? z[k][i] : 2 * i < C ? v[k][(2 * i + 1) % C] : z[k][(2 * i + 1) % C]);
                o[INTER ? 2 * i : i] = from_f32<T>(u * cs[i] - w * sn[i]);
                o[INTER ? 2 * i + 1 : C + i] = from_f32<T>(u * sn[i] + w * cs[i]);
            }
            if (!copy) {
                __builtin_memcpy(v[k], o, sizeof(v[k]));
                __builtin_memcpy(z[k], o + C, sizeof(z[k]));
            }
            T* y = dst(hb + k) + off;
            put<FULL>(y, left_a, v[k]);
            put<FULL>(y + far, left_b, z[k]);
        }
    };
    int h = h0;
    for (; h + 4 <= h1; h += 4) group(std::integral_constant<int, 4>{}, h);
    if (h + 2 <= h1) {
        group(std::integral_constant<int, 2>{}, h);
        h += 2;
    }
    if (h < h1) group(std::integral_constant<int, 1>{}, h);
}

template <typename T>
void rotary(const RotaryArgs& a, hipStream_t s) {
    constexpr int C = 16 / (int)sizeof(T);
    RotaryKernelArgs k{a, 0, 0, 1};
    k.chunks = (a.rot / 2 + C - 1) / C;
    // (a tensor turned in place needs no copy of the rest; both must be)
    bool in_place = true, apart = true;
    for (int w = 0; w < 2; ++w) {
        if (a.x[w] && a.x[w] != a.y[w]) in_place = false;
        if (a.x[w] && a.x[w] == a.y[w]) apart = false;
    }
    k.copies = in_place ? 0 : (a.d - a.rot + 2 * C - 1) / (2 * C);
    const int64_t items = (int64_t)a.B * a.L * (k.chunks + k.copies);
    const int both = a.heads[0] + a.heads[1];
    // heads shared among threads until the chip is full (256 CUs x 2048 threads)
    const int64_t want = ((int64_t)256 * 2048 + items - 1) / items;
    k.split = want < both ? (int)want : both;
    const dim3 grid((unsigned)((items + 255) / 256), k.split);
    // Vectors that end with the row's part: where its length is no multiple of them the last
    // one repeats features of the one before, which two threads then turn alike (not in
    // place, where the second would turn them again); shorter parts go feature by feature.
    const auto whole_chunks = [&](int n, int c) { return n % c == 0 || (n >= c && apart); };
    const bool full = whole_chunks(a.rot / 2, C) && (k.copies == 0 || whole_chunks(a.d - a.rot, 2 * C));
    auto run = [&](auto inter, auto whole) {
        hipLaunchKernelGGL((rotary_kernel<T, decltype(inter)::value, decltype(whole)::value>), grid, dim3(256), 0,
                           s, k, items);
    };
    if (a.interleaved) full ? run(std::true_type{}, std::true_type{}) : run(std::true_type{}, std::false_type{});
    else full ? run(std::false_type{}, std::true_type{}) : run(std::false_type{}, std::false_type{});
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
