// Attention of new tokens over a paged cache (fox_attn_paged): the row at position i of head
// h over the positions j <= i of its sequence, logits x_ij = q_i.k_j / sqrt(d) + c_i - c_j,
// pages left out row by row by the block test of ACP.
//
// Two kernels share the arithmetic (RowBlock): S^T = K Q^T on the matrix cores, so that a
// lane holds one query and eight keys of a 32-key half, the running maximum and sum of the
// softmax per query, and O^T += V^T P^T.
//   paged_long_kernel   64 or 128 rows of one head per workgroup, 16 or 32 per wave; the
//                       waves share the pages in LDS.  8000 rows of 16 heads (4 key heads, d =
//                       128, bfloat16) behind 8150 positions take 560 to 610 us, 830 to 910
//                       TFLOP/s of kept products: the matrix cores are busy 41% of the cycles and
//                       overlap the exponentials in part, and 3.3 GB pass the L2s meanwhile (a key
//                       head's 8 MB of pages are read by 63 tiles of 4 heads), 5.4 to 6 TB/s, near
//                       the rate of plain reads.  2 x 4096 rows of 12 heads (d = 64) behind 4096
//                       take 163 us a call in a row of them, 650 TFLOP/s (in a trace, with pauses,
//                       165 and 12 for the merge of 41 MB of sums); matrix cores busy 30%, 12
//                       registers of a lane spilled at three waves per SIMD.
//                       (Not the exponentials alone: the forward without pages has as many per
//                       product at d = 64 and reaches 860 to 890 TFLOP/s.)  float32, 2048 rows
//                       of 4 heads behind 2048, 79 us, 64 TFLOP/s, where a large product reaches
//                       154; matrix cores busy 44%.
//   paged_short_kernel  the rows of all query heads of a key head, where they are at most
//                       16 in a sequence (single tokens above all): the waves take different
//                       pages of the same rows.  Bound by memory: a page is read once for
//                       all query heads that share it.  8 sequences of 4k to 64k positions, 12
//                       heads, bfloat16: 51 us for 311 MB, 6.1 TB/s, what plain reads of such
//                       pages reach.  16 of 3k to 11k, 32 heads on 4 key heads, d = 128: 47 us for
//                       207 MB, 4.4 TB/s (339 registers and 133 KB of LDS: one workgroup per CU).
//                       float32, 8 of 100 to 50k, 12 heads: 81 us for 440 MB, 5.5 TB/s.
// The kept pages of all (rows, head) items, one after the other, are dealt in equal shares to
// as many workgroups as the chip holds at a time, whatever lengths and heads they belong to:
// paged_plan_kernel finds each item's pages, every workgroup adds up where its share lies,
// and paged_join_kernel merges the sums of items that lie in several shares (launches of
// their own order these without a device-wide fence).  Where items are many times the
// workgroups, or have a few pages only, a workgroup takes an item instead.
#include <type_traits>

#include "acp_paged.h"
#include "acp_scan.h"

namespace acp {
namespace {

constexpr int kShortRows = 16;    // rows of a short sequence: new tokens times query heads
constexpr float kSlack = 8.f;     // a weight is at most 2^8 (2^2: chunks 10% slower, for 5% less error)
constexpr double kFixedMax = 52.0;    // largest bound U that serves as reference (paged_long_kernel)

__device__ __forceinline__ f32x4 mfma_f32(float a, float b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

template <typename T> constexpr bool is_bf16() { return sizeof(T) == 2; }

// Key of element j (0..7) of lane group g in a half of 32 keys
template <typename T> __device__ __forceinline__ int key_of(int g, int j) {
    return is_bf16<T>() ? 8 * g + j : 16 * (j >> 2) + 4 * g + (j & 3);
}
// Row of the half that lane r16 of subtile kk reads for the A operand of S^T
template <typename T> __device__ __forceinline__ int key_row(int kk, int r16) {
    return is_bf16<T>() ? 8 * (r16 >> 2) + 4 * kk + (r16 & 3) : 16 * kk + r16;
}

// 16 * NQ queries of a wave.  Lane 16 g + r holds queries r, 16 + r and, of the sums,
// features 16 dt + 4 g + (0..3).
template <typename T, int D, int NQ>
struct RowBlock {
    static constexpr int NK = is_bf16<T>() ? D / 32 : D / 16;   // operand pieces of a row
    static constexpr int ND = D / 16;
    typedef typename std::conditional<is_bf16<T>(), bf16x8, f32x4>::type Frag;
    static constexpr int kFrag = is_bf16<T>() ? 8 : 4;          // features of a piece and lane

    Frag q[NQ][NK];
    f32x4 acc[NQ][ND];
    // Weights are 2^(y - ref).  ref is the largest logit so far up to kSlack: it is moved up
    // only when a logit exceeds it by more (thr: by which a logit may; before the first
    // key every logit moves it), so that the sums are rarely scaled and the lanes of a query
    // need not agree on a maximum for every key.
    float ref[NQ], thr[NQ];
    float l[NQ];                                                // of this lane's keys only

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) {
            ref[qt] = 0.f;
            thr[qt] = -INFINITY;
            l[qt] = 0.f;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) acc[qt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    __device__ __forceinline__ float max_logit(int qt) const { return thr[qt] > 0.f ? ref[qt] : -INFINITY; }
    __device__ __forceinline__ void load_q(int qt, const T* row, int g) {
#pragma unroll
        for (int s = 0; s < NK; ++s)
            q[qt][s] = *reinterpret_cast<const Frag*>(row + 4 * kFrag * s + kFrag * g);
    }
    // s[kk][qt] = start[qt] + K Q^T of subtile kk; k(kk, piece) gives the lane's A operand
    template <typename F>
    __device__ __forceinline__ void scores(f32x4 (&s)[2][NQ], const f32x4 (&start)[NQ], F k) const {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt) s[kk][qt] = start[qt];
#pragma unroll
            for (int p = 0; p < NK; ++p) {
                const Frag a = k(kk, p);
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt) {
                    if constexpr (is_bf16<T>()) {
                        s[kk][qt] = mfma16(a, q[qt][p], s[kk][qt]);
                    } else {
#pragma unroll
                        for (int t = 0; t < 4; ++t) s[kk][qt] = mfma_f32(a[t], q[qt][p][t], s[kk][qt]);
                    }
                }
            }
        }
    }
    // y - ref (log2 units, -inf: left out) -> weights; true if ref[qt] moved.  again(y) forms
    // y - ref anew from the products: formed with a ref far below, y has been rounded in
    // proportion to its distance (2e-5 in the log-sum-exp where the first keys seen are forgotten).
    template <typename F>
    __device__ __forceinline__ bool weights(int qt, float (&y)[8], F again) {
        float mx = fmaxf(y[0], y[1]);
#pragma unroll
        for (int j = 2; j < 8; j += 2) mx = fmaxf(fmaxf(mx, y[j]), y[j + 1]);
        const bool move = __any(mx > thr[qt]);
        if (move) {
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            if (mx > thr[qt]) {
                const float alpha = thr[qt] > 0.f ? fast_exp2(-mx) : 0.f;
                ref[qt] += mx;
                thr[qt] = kSlack;
                l[qt] *= alpha;
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) acc[qt][dt] *= alpha;
            }
            again(y);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            y[j] = fast_exp2(y[j]);
            l[qt] += y[j];
        }
        return move;
    }
    // The same where ref is known to be no less than any logit
    __device__ __forceinline__ void weights_fixed(int qt, float (&y)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            y[j] = fast_exp2(y[j]);
            l[qt] += y[j];
        }
    }
    // acc += V^T P^T, the weights rounded to T for the matrix cores (their sum l is not: the
    // log-sum-exp keeps float32's precision, and O is off by what 2^-9 of a weight makes); v(dt, j): bf16 the lane's eight keys of column 16 dt + r (j unused),
    // float the key of element j
    template <typename F>
    __device__ __forceinline__ void add(const float (&p)[NQ][8], F v) {
        if constexpr (is_bf16<T>()) {
            bf16x8 pb[NQ];
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt)
#pragma unroll
                for (int j = 0; j < 8; ++j) pb[qt][j] = (__bf16)p[qt][j];
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) {
                const bf16x8 a = v(dt, 0);
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt) acc[qt][dt] = mfma16(a, pb[qt], acc[qt][dt]);
            }
        } else {
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float a = v(dt, j);
#pragma unroll
                    for (int qt = 0; qt < NQ; ++qt) acc[qt][dt] = mfma_f32(a, p[qt][j], acc[qt][dt]);
                }
        }
    }
};

// Every lane's sum over the four lanes that hold a query
__device__ __forceinline__ float over_groups(float v) {
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
    return v;
}

// Marks, for the values that are not finite in the keys of `bad` (a bit each) that the query
// at position pos attends to, the feature of the query's row: an infinity of either sign, NaN
// both.  The four lanes of a query share the keys; v0 is the page's first value row.  Rare.
template <typename T, int D>
__device__ __forceinline__ void mark_bad(unsigned long long bad, const T* v0, int first, int pos, int lane,
                                         unsigned (&inf)[2][D / 32]) {
    while (bad) {
        const int key = __builtin_ctzll(bad);
        bad &= bad - 1;
        if ((key & 3) != lane >> 4 || first + key > pos) continue;
#pragma unroll 1
        for (int f = 0; f < D; ++f) {
            const float x = to_f32(v0[key * D + f]);
            if (__builtin_isfinite(x)) continue;
            if (!(x < 0.f)) atomicOr(&inf[0][f >> 5], 1u << (f & 31));
            if (!(x > 0.f)) atomicOr(&inf[1][f >> 5], 1u << (f & 31));
        }
    }
}
// The marks of a query's row into its sums
template <int D>
__device__ __forceinline__ void add_marks(f32x4 (&acc)[D / 16], const unsigned (&inf)[2][D / 32], int g) {
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int f = 16 * dt + 4 * g + t;
            if (inf[0][f >> 5] >> (f & 31) & 1) acc[dt][t] += INFINITY;
            if (inf[1][f >> 5] >> (f & 31) & 1) acc[dt][t] -= INFINITY;
        }
}

// The sequence and the tile of `rows` tokens in it that global tile number `tile` is, among
// the sequences of n tokens, lo < n <= hi; false when there are fewer tiles.
__device__ __forceinline__ bool locate(const PagedArgs& a, int tile, int rows, int lo, int hi, int lane,
                                       int& seq, int& local, Seq& found) {
    int before = 0;
    for (int base = 0; base < a.N; base += 64) {
        const Seq q = seq_of(a, min(base + lane, a.N - 1));
        const int t = base + lane < a.N && q.n > lo && q.n <= hi ? (q.n + rows - 1) / rows : 0;
        int incl = t;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int u = __shfl_up(incl, o);
            if (lane >= o) incl += u;
        }
        const unsigned long long past = __ballot(before + incl > tile);
        if (past) {
            const int f = __builtin_ctzll(past);
            seq = __builtin_amdgcn_readfirstlane(base + f);
            local = __builtin_amdgcn_readfirstlane(tile - before - (__shfl(incl, f) - __shfl(t, f)));
            auto of = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
            found = Seq{of(q.row0), of(q.n), of(q.past)};
            return true;
        }
        before += __shfl(incl, 63);
    }
    return false;
}

// ACP's bound U on a head's logits (without the decay); NaN where no scales are given
__device__ __forceinline__ double head_bound(const PagedArgs& a, int h) {
    if (!(a.log_lmax_over_eps < INFINITY)) return __builtin_nan("");
    return ((double)a.gamma_q[h] * (double)a.gamma_k[h / (a.H / a.Hk)]) * __builtin_sqrt((double)a.d);
}
__device__ __forceinline__ double head_delta(const PagedArgs& a, int h) {
    if (!(a.log_lmax_over_eps < INFINITY)) return -INFINITY;
    return -(2.0 * head_bound(a, h) + a.log_lmax_over_eps);
}

// First page that the row at position pos keeps: the test grows with the page, and 64 pages are
// probed at a time, the first ones while the row's own gate is on its way.  A page that is not in
// the cache counts as left out (it may have been dropped).
__device__ __forceinline__ int first_page(const PagedArgs& a, int s, int h, int pos, int lane) {
    if (a.gamma_q == nullptr || a.W == 0) return 0;
    // (loads without a branch, so that they are asked for together)
    const int* table = a.table + (int64_t)s * a.W;
    auto entry = [&](int n) { return table[min(n, a.W - 1)]; };
    auto page = [&](int e, int n) { return n < a.W && e >= 0 && e < a.P ? e : -1; };
    auto gate = [&](int p, int slot) { return gates_of(a, max(p, 0), h)[slot]; };
    int lo = 0, hi = pos >> 6;              // the answer lies in [lo, hi]; hi is kept
    int step = (hi + 63) / 64, n = lane * step;
    const int own_e = entry(hi), probe = entry(n);
    const int own = page(own_e, hi);
    int p = page(probe, n);
    const double own_c = gate(own, pos & 63);
    double end = gate(p, 63);
    const double delta = head_delta(a, h), ci = own < 0 ? 0.0 : own_c;
    while (lo < hi) {
        const unsigned long long k = __ballot(n >= hi || (p >= 0 && ci - end >= delta));
        const int f = k ? __builtin_ctzll(k) : 64;
        const int top = min(lo + f * step, hi);
        if (f > 0) lo = min(lo + (f - 1) * step + 1, top);
        hi = top;
        step = (hi - lo + 63) / 64;
        n = lo + lane * step;
        p = page(entry(n), n);
        end = gate(p, 63);
    }
    return lo;
}

// First page that any of the rows at positions p0 .. p1 of a tile keeps: the first row's, and where a
// row's own page is not in the cache (c_i counts as 0 there, which keeps more) that row's.  own: all are there.
__device__ __forceinline__ int first_of_tile(const PagedArgs& a, int s, int h, int p0, int p1, int lane, bool& own) {
    // (a tile's rows lie in three pages at most; their entries are asked for before the search)
    const int n = (p0 >> 6) + lane, p = page_of(a, s, min(n, p1 >> 6));
    int lo = first_page(a, s, h, p0, lane);
    unsigned long long bad = __ballot(n <= p1 >> 6 && p < 0);
    own = bad == 0;
    for (; bad; bad &= bad - 1)
        lo = min(lo, first_page(a, s, h, max(p0, ((p0 >> 6) + (int)__builtin_ctzll(bad)) << 6), lane));
    return lo;
}

// ---- items and shares ------------------------------------------------------------------
// An item: rows of a sequence that one head (short: one group of heads) takes over the pages
// lo .. lo + pages - 1.
struct alignas(32) Item {
    int s;             // sequence, -1: no such item
    int t0, n;         // its first packed row, how many new tokens
    int p0;            // position of the first
    int len;           // of the sequence, its new rows included
    int lo, pages;
    int own;           // long: the pages of its rows are there (else c_i, where one is bad, is 0)
};
// What a workgroup found at the start of its share: where the first page of it that another
// share has pages in front of lies, for the merge (item -1: none, or an earlier share says so)
struct alignas(16) Cut {
    int item, skip, chunk, pad;
};
// The items of one kernel.  Item number (key head, tile, head of the group), in this order,
// so that neighbouring shares read the same pages.
struct Work {
    Item* items;
    int* places;       // [n] their lengths in the list (place_of)
    Cut* cuts;         // [wgs]
    float* slots;      // [2 wgs] partial sums of a share's first item and of a later one
    int n, tiles;      // items; tiles of all sequences together, at most
    int wgs, least;    // workgroups; the least pages of a share
    bool shared;       // in shares; else a workgroup per item
    int setup;         // what taking up an item costs, in pages: its place in the list is that
                       // much longer than its pages, in front of them
};

// Pages from lo up to those that the table has, for rows up to position last
__device__ __forceinline__ int page_count(const PagedArgs& a, int lo, int last) {
    return max(min(last >> 6, a.W - 1) - lo + 1, 0);
}
__device__ __forceinline__ double gate_at(const PagedArgs& a, int s, int h, int pos) {
    const int p = page_of(a, s, pos >> 6);
    return p < 0 ? 0.0 : gates_of(a, p, h)[pos & 63];
}
// 0, which the compiler does not know: what is rarely computed from it is not computed ahead
// of a loop and kept
__device__ __forceinline__ int late_zero() {
    int z = 0;
    asm volatile("" : "+s"(z));
    return z;
}
// A kernel's first argument, read anew where it is used, for the same reason
__device__ __forceinline__ const PagedArgs& late_args() {
    typedef const __attribute__((address_space(4))) char* KernargPtr;
    return *(const PagedArgs*)((KernargPtr)__builtin_amdgcn_kernarg_segment_ptr() + late_zero());
}
__device__ __forceinline__ void report(const PagedArgs& a, int s, int h, int lane, int flag = kFlagPage) {
    if (a.flags && lane == 0) atomicOr(a.flags + (int64_t)(s + late_zero()) * a.H + h, flag);
}

// Long item `id`, by a wave
template <int kRows>
__device__ __forceinline__ Item long_item(const PagedArgs& a, int id, int tiles, int short_max, int h, int lane) {
    const int G = a.H / a.Hk, rest = id - id / (tiles * G) * tiles * G;
    Item it{-1, 0, 0, 0, 0, 0, 0, 0};
    int s, tile;
    Seq q;
    // (the last tiles of a sequence have the most pages: they go first)
    if (!locate(a, tiles - 1 - rest / G, kRows, short_max, 0x7fffffff, lane, s, tile, q)) return it;
    it.s = s;
    it.t0 = q.row0 + tile * kRows;
    it.n = min(kRows, q.n - tile * kRows);
    it.p0 = q.past + tile * kRows;
    it.len = q.past + q.n;
    bool own;
    it.lo = first_of_tile(a, s, h, it.p0, it.p0 + it.n - 1, lane, own);
    it.own = own;
    it.pages = page_count(a, it.lo, it.p0 + it.n - 1);
    if (((it.p0 + it.n - 1) >> 6) >= a.W) report(a, s, h, lane);
    return it;
}
__device__ __forceinline__ int long_head(const PagedArgs& a, int id, int tiles) {
    const int G = a.H / a.Hk, hk = id / (tiles * G);
    return hk * G + (id - hk * tiles * G) % G;
}

__device__ __forceinline__ int place_of(const Work& w, int pages) { return pages > 0 ? pages + w.setup : 0; }

// Rows without a page: O = 0, lse = -inf (lane: feature)
template <typename T>
__device__ __forceinline__ void empty_row(const PagedArgs& a, int t, int h, int lane) {
    const int64_t row = (int64_t)t * a.H + h;
    for (int f = lane; f < a.d; f += 64) ((T*)a.O)[row * a.d + f] = from_f32<T>(0.f);
    if (lane == 0) a.lse[row] = -INFINITY;
}

// Rows 64 i .. 64 i + 63 of the call, by a wave: those that no sequence brings, or one of more than
// `limit` rows, become empty
template <typename T>
__device__ __forceinline__ void fill_rows(const PagedArgs& a, int i, int limit, int lane) {
    const int t = 64 * i + lane;
    bool on = true;
    if (t < a.T) {
        const int s = sequence_of(a, t);
        on = s >= 0 && seq_of(a, s).n <= limit;
    }
    for (unsigned long long rows = __ballot(!on); rows; rows &= rows - 1) {
        const int64_t row = (int64_t)(64 * i + (int)__builtin_ctzll(rows)) * a.H;
        uint4* o = reinterpret_cast<uint4*>((T*)a.O + row * a.d);
        for (int e = lane; e < a.H * a.d * (int)sizeof(T) / 16; e += 64) o[e] = make_uint4(0, 0, 0, 0);
        for (int h = lane; h < a.H; h += 64) a.lse[row + h] = -INFINITY;
    }
}

// The items of both kernels, by workgroups of 8 waves: a wave per long item, and per head of
// a short one (8 of them at a time), whose first page is the first that any head of the group
// keeps for any token.  The workgroups from fill_at on look after the rows that no item has.
template <typename T, int kRows>
__global__ __launch_bounds__(512) void paged_plan_kernel(PagedArgs a, Work lw, Work sw, int short_max,
                                                         int long_above, int short_waves, int fill_at, int limit) {
    __shared__ int first[8][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int nl = (lw.n + 7) / 8, G = a.H / a.Hk;
    if ((int)blockIdx.x >= fill_at) {
        fill_rows<T>(a, (blockIdx.x - fill_at) * 8 + wave, limit, lane);
        return;
    }
    if ((int)blockIdx.x < nl) {
        const int id = blockIdx.x * 8 + wave;
        if (id >= lw.n) return;
        const int h = long_head(a, id, lw.tiles);
        const Item it = long_item<kRows>(a, id, lw.tiles, long_above, h, lane);
        if (lane == 0) {
            lw.items[id] = it;
            lw.places[id] = place_of(lw, it.pages);
        }
        if (it.s >= 0 && it.pages == 0)
            for (int r = 0; r < it.n; ++r) empty_row<T>(a, it.t0 + r, h, lane);
        return;
    }
    const int slot = wave / short_waves, w = wave - slot * short_waves;
    const int id = (blockIdx.x - nl) * (8 / short_waves) + slot;
    const int hk = min(id / sw.tiles, a.Hk - 1);
    Item it{-1, 0, 0, 0, 0, 0, 0, 0};
    int s, tile;
    Seq q;
    if (id < sw.n && locate(a, id - hk * sw.tiles, short_max, 0, short_max, lane, s, tile, q)) {
        it = Item{s, q.row0, q.n, q.past, q.past + q.n, 0, 0, 0};
        for (int k = w; k < G; k += short_waves) {
            const int h = hk * G + k;
            bool own;
            const int f = first_of_tile(a, s, h, q.past, it.len - 1, lane, own);
            if (lane == 0) first[slot][k] = f;
            if (((it.len - 1) >> 6) >= a.W) report(a, s, h, lane);
        }
    }
    __syncthreads();
    if (id >= sw.n || w > 0) return;
    if (it.s >= 0) {
        it.lo = first[slot][0];
        for (int k = 1; k < G; ++k) it.lo = min(it.lo, first[slot][k]);
        it.pages = page_count(a, it.lo, it.len - 1);
        if (it.pages == 0)
            for (int r = 0; r < it.n * G; ++r) empty_row<T>(a, it.t0 + r / G, hk * G + r % G, lane);
    }
    if (lane == 0) {
        sw.items[id] = it;
        sw.places[id] = place_of(sw, it.pages);
    }
}


// A workgroup's share: `left` of the list from `skip` in item `item`'s place on
struct Share {
    int item, skip, left;
    bool later;        // past the share's first item
};
struct ShareSmem {
    long long wave[4];
    int item, skip, left;
};
// The share of workgroup wg (256 threads); left = 0: none.  A share fits an int: fewer than 8
// items per workgroup are shared out, to at least kLeastShares, of at most 2^25 pages each.
__device__ __forceinline__ Share find_share(const Work& w, int wg, ShareSmem& sm) {
    if (!w.shared) return Share{wg, 0, 0x7fffffff, false};        // the item, whole
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int per = (w.n + 255) / 256, i0 = min(t * per, w.n), i1 = min(i0 + per, w.n);
    long long sum = 0;
    for (int i = i0; i < i1; ++i) sum += w.places[i];
    long long incl = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long long u = __shfl_up(incl, o);
        if (lane >= o) incl += u;
    }
    if (lane == 63) sm.wave[wave] = incl;
    if (t == 0) sm.left = 0;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (k < wave) incl += sm.wave[k];
        total += sm.wave[k];
    }
    long long before = incl - sum;
    const long long chunk = max((total + w.wgs - 1) / w.wgs, (long long)w.least), at = wg * chunk;
    if (at < total && before <= at && at < incl) {       // (one thread: its items hold pages)
        int i = i0;
        for (; before + w.places[i] <= at; ++i) before += w.places[i];
        const int skip = (int)(at - before);
        sm.item = i;
        sm.skip = skip;
        sm.left = (int)min(chunk, total - at);
        const bool mine = skip > w.setup && skip - chunk <= w.setup;
        w.cuts[wg] = Cut{mine ? i : -1, skip, (int)chunk, 0};
    }
    if (at >= total && t == 0) w.cuts[wg] = Cut{-1, 0, 0, 0};
    __syncthreads();
    return Share{__builtin_amdgcn_readfirstlane(sm.item), __builtin_amdgcn_readfirstlane(sm.skip),
                 __builtin_amdgcn_readfirstlane(sm.left), false};
}
// The share's pages of its present item: first, count (0: the share ends in front of them)
__device__ __forceinline__ int pages_here(const Work& w, const Share& sh, const Item& it, int& first) {
    const int setup = w.shared ? w.setup : 0;
    first = it.lo + max(sh.skip - setup, 0);
    return min(max(sh.left - max(setup - sh.skip, 0), 0), it.lo + it.pages - first);
}
// On to the share's next item that has pages; false at its end
__device__ __forceinline__ bool next_item(const Work& w, Share& sh, const Item& it) {
    sh.left -= place_of(w, it.pages) - sh.skip;
    if (!w.shared || sh.left <= 0) return false;
    sh.skip = 0;
    sh.later = true;
    do ++sh.item;
    while (__builtin_amdgcn_readfirstlane(w.places[sh.item]) == 0);
    return true;
}
__device__ __forceinline__ Item item_at(const Work& w, int i) {
    const Item t = w.items[i];
    auto u = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    return Item{u(t.s), u(t.t0), u(t.n), u(t.p0), u(t.len), u(t.lo), u(t.pages), u(t.own)};
}

// Page numbers of 64 consecutive pages, one per lane
struct PageWindow {
    int base, id;
    __device__ __forceinline__ void fill(const PagedArgs& a, int s, int n, int lane) {
        base = n;
        id = page_of(a, s + late_zero(), n + lane);
    }
    __device__ __forceinline__ int get(const PagedArgs& a, int s, int n, int lane) {
        if (n - base >= 64) fill(a, s, n, lane);
        return __builtin_amdgcn_readlane(id, n - base);
    }
};

// ---- tiles of 64 rows in LDS -----------------------------------------------------------
// bf16: the swizzled panels of acp_device.h.  float: rows of D, 16-byte chunk c of row r at
// position c ^ (r mod 16): conflict-free for 16-byte reads of 16 rows and for 4-byte reads
// of 16 columns from four rows.
template <int D>
__device__ __forceinline__ int f32_off(int row, int col) {
    return row * D * 4 + ((((col >> 2) ^ (row & 15))) << 4) + ((col & 3) << 2);
}

template <typename T, int D>
struct PageDma {
    // (a float tile is as many bytes as a bf16 tile of twice the columns)
    TileDma<(is_bf16<T>() ? D : 2 * D), 4> dma;
    __device__ __forceinline__ void init(int wave, int lane) {
        dma.init(wave, lane);
        if constexpr (!is_bf16<T>()) {
            constexpr int kChunks = D / 4, kRows = 64 / kChunks;   // of an instruction
#pragma unroll
            for (int k = 0; k < dma.kPer; ++k) {
                const int row = (wave + 4 * k) * kRows + lane / kChunks;
                dma.off[k] = (unsigned)(row * D * 4 + (((lane % kChunks) ^ (row & 15)) << 4));
            }
        }
    }
    __device__ __forceinline__ void issue(unsigned char* tile, const T* src, int wave) const {
        dma.issue(tile, reinterpret_cast<const __bf16*>(src), wave);
    }
};

// Values that are not finite are kept out of the products, where 0 times them is not 0, and
// brought into the rows that attend to their key by marks (mark_bad).
//
// The values of a tile of which some row leaves something out: rows from `valid` on (never
// written) become 0, and so does every value that is not finite; bit r of `bad` is set
// where row r held one.  nt threads, thread t.
template <typename T, int D>
__device__ __forceinline__ void clean_values(unsigned char* tile, int valid, unsigned* bad, int t, int nt) {
    constexpr int kPieces = D * (int)sizeof(T) / 16;               // of a row
    for (int i = t; i < 64 * kPieces; i += nt) {
        const int row = i / kPieces, c = i % kPieces;
        uint4* at;
        if constexpr (is_bf16<T>()) at = reinterpret_cast<uint4*>(tile + tile_off(row, 8 * c));
        else at = reinterpret_cast<uint4*>(tile + f32_off<D>(row, 4 * c));
        uint4 v = *at;
        if (row >= valid) {
            *at = make_uint4(0, 0, 0, 0);
            continue;
        }
        unsigned* w = &v.x;
        bool found = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (is_bf16<T>()) {
                if ((w[k] & 0x7f80u) == 0x7f80u) { w[k] &= 0xffff0000u; found = true; }
                if ((w[k] & 0x7f800000u) == 0x7f800000u) { w[k] &= 0xffffu; found = true; }
            } else if ((w[k] & 0x7f800000u) == 0x7f800000u) {
                w[k] = 0;
                found = true;
            }
        }
        if (found) {
            *at = v;
            atomicOr(&bad[row >> 5], 1u << (row & 31));
        }
    }
}

// A row's result: to the output, or to row r of a slot for R rows
template <typename T, int D>
__device__ __forceinline__ void put_row(const PagedArgs& a, int t, int h, const f32x4 (&acc)[D / 16], float m,
                                        float l, int g) {
    const int64_t row = (int64_t)t * a.H + h;
    const float inv = l == 0.f ? 0.f : 1.0f / l;         // (no key: every page was bad)
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
        T o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = from_f32<T>(acc[dt][k] * inv);
        __builtin_memcpy((T*)a.O + row * D + 16 * dt + 4 * g, o, sizeof(o));
    }
    if (g == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + fast_log2(l)) * kLn2;
}
template <int D>
constexpr int slot_floats(int rows) { return rows * (D + 2); }
template <int D, int R>
__device__ __forceinline__ void put_part(float* slot, int r, const f32x4 (&acc)[D / 16], float m, float l, int g) {
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4*>(slot + r * D + 16 * dt + 4 * g) = acc[dt];
    if (g == 0) *reinterpret_cast<float2*>(slot + R * D + 2 * r) = make_float2(m, l);
}

// ---- long ------------------------------------------------------------------------------
template <typename T, int D, int NQ>
struct alignas(1024) LongSmem {
    unsigned char k[2][64 * D * sizeof(T)];
    unsigned char v[2][64 * D * sizeof(T)];
    float kb[2][64];         // (R - c_j) log2(e), less a reference known before
    float2 kd[2][64];        // c_j - R as a sum of two floats
    double end[2];           // c of the page's last position
    double rc[64 * NQ];      // c_i of the rows
    float2 rd[64 * NQ];      // c_i - R likewise
    unsigned bad[2][2];      // keys of the page with values that are not finite
    unsigned inf[64 * NQ][2][D / 32];
    int marked;
    ShareSmem share;
};

template <typename T, int D, int NQ>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 && is_bf16<T>() ? 3 : 2)))
void paged_long_kernel(PagedArgs, Work work, float kscale) {
    constexpr int kRows = 64 * NQ;
    typedef RowBlock<T, D, NQ> Block;
    __shared__ LongSmem<T, D, NQ> sm;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wg = blockIdx.x;
    Share sh = find_share(work, wg, sm.share);
    if (sh.left == 0) return;
    for (;;) {
    // (recomputed for each item: held across the loop, what depends on them costs registers)
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63, g = lane >> 4, r16 = lane & 15;
    const PagedArgs& a = late_args();
    const Item it = item_at(work, sh.item);
    if (it.pages == 0) return;                          // (not in a share)
    const int s = it.s, h = long_head(a, sh.item, work.tiles);
    // this share's pages of the item
    int nb;
    const int taken = pages_here(work, sh, it, nb), ne = nb + taken - 1;
    if (work.shared && taken == 0) return;
    const int hk = h / (a.H / a.Hk);
    const double delta = readfirst_f64(head_delta(a, h));
    const int rows = it.n, p0 = it.p0, p1 = p0 + rows - 1, len = it.len;

    auto gate = [&](int pos) __attribute__((always_inline)) { return gate_at(a, s, h, pos); };
    const double R = readfirst_f64(gate(p0));

    Block blk;
    blk.clear();
    // rows of the wave and of the lane (those past the end repeat the last one)
    // (counted from p0: positions may be as large as an int holds)
    const int o0 = 16 * NQ * wave;
    const bool wave_on = o0 < rows;
    const int w0 = p0 + min(o0, rows - 1), w1 = p0 + min(o0 + 16 * NQ - 1, rows - 1);
    auto pos_of = [&](int qt) __attribute__((always_inline)) { return p0 + min(o0 + 16 * qt + r16, rows - 1); };
    float row[NQ];                                   // (c_i - R) log2(e), less a moved reference
    // The logits of a head lie in [-U, U] by ACP's bound, less a decay that a row's own key has
    // not.  A ref that leaves that key's weight at e^(-64) or more, and every weight at
    // e^(2 kFixedMax - 64) or less, need not be looked for (8000 rows of 16 heads behind 8150,
    // d = 128: 580 us instead of 690).  Not in float32, where products that start at a term as
    // large as U lose bits that count (1.3e-6 instead of 2.6e-7 of O's size).
    const double u = readfirst_f64(head_bound(a, h));
    const bool fixed = is_bf16<T>() && it.own && u >= 0.0 && u <= kFixedMax;
    const float known = fixed ? (float)fmin(u, 64.0 - u) * kLog2e : 0.f;
    if (fixed) {
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) {
            blk.ref[qt] = known;
            blk.thr[qt] = INFINITY;
        }
    }
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
        const int pos = pos_of(qt), i = o0 + 16 * qt + r16;
        const double ci = gate(pos), r = ci - R;
        blk.load_q(qt, (const T*)a.q + (int64_t)(it.t0 + pos - p0) * a.qt + (int64_t)h * a.qh, g);
        // (the wave's own rows: no other reads them)
        const float hi = (float)r;
        sm.rc[i] = ci;
        sm.rd[i] = make_float2(hi, (float)(r - (double)hi));
        row[qt] = hi * kLog2e;
    }
    // Where a row's own page is bad, one row's gate says nothing of another's: for the wave no page
    // is left out (infinity), and for the tile none is whole (NaN; R may be far from the others'
    // gates then, so that it takes both floats of c_i - R and c_j - R)
    const double c_first = it.own ? readfirst_f64(gate(w0)) : INFINITY;
    const double c_tile_last = it.own ? readfirst_f64(gate(p1)) : __builtin_nan("");

    PageDma<T, D> dma;
    dma.init(wave, lane);
    PageWindow win;
    // (all that the loops need of the arguments)
    const T* kp = (const T*)a.kp + (int64_t)hk * 64 * D;
    const T* vp = (const T*)a.vp + (int64_t)hk * 64 * D;
    const double* gates = a.cp + (int64_t)h * 64;
    const int64_t page_stride = (int64_t)a.Hk * 64 * D, gate_stride = (int64_t)a.H * 64;
    double cn = 0.0;                        // the next page's gate, thread t < 64
    int page_next = -1;                     // the page last asked for, -1: not in the cache
    auto issue = [&](int n, int buf) __attribute__((always_inline)) {
        const int p = win.get(a, s, n, lane);
        const int64_t at = max(p, 0) * page_stride;
        page_next = p;
        if (tid < 64) cn = gates[(int64_t)max(p, 0) * gate_stride + tid];
        dma.issue(sm.k[buf], kp + at, wave);
        dma.issue(sm.v[buf], vp + at, wave);
    };
    auto put_gates = [&](int buf) __attribute__((always_inline)) {
        if (tid < 64) {
            const double r = cn - R;
            const float hi = (float)r;
            sm.kb[buf][tid] = __builtin_fmaf(-hi, kLog2e, -known);
            sm.kd[buf][tid] = make_float2(hi, (float)(r - (double)hi));
            if (tid == 63) sm.end[buf] = cn;
            if (tid < 2) sm.bad[buf][tid] = 0;
        }
    };

    // offsets of the lane's operands in a tile
    int koff[Block::NK];
#pragma unroll
    for (int p = 0; p < Block::NK; ++p)
        koff[p] = is_bf16<T>() ? tile_off(key_row<T>(0, r16), 32 * p + 8 * g) : f32_off<D>(r16, 16 * p + 4 * g);

    int voff[is_bf16<T>() ? Block::ND : 1];
    if constexpr (is_bf16<T>())
#pragma unroll
        for (int dt = 0; dt < Block::ND; ++dt) voff[dt] = tile_off(8 * g + (r16 >> 2), 16 * dt + 4 * (r16 & 3));

    auto step = [&](auto mask_tag, auto fixed_tag, const f32x4(&start)[NQ], int n, int buf)
                    __attribute__((always_inline)) {
        constexpr bool kMask = decltype(mask_tag)::value, kFixed = decltype(fixed_tag)::value;
        bool keep[NQ];
        if constexpr (kMask) {
            const double end = sm.end[buf];
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt)
                keep[qt] = n >= (pos_of(qt) >> 6) || sm.rc[o0 + 16 * qt + r16] - end >= delta;
        }
        // LDS operands are asked for together (bf16): all keys of a half before its first
        // product, its values before its weights are formed.  The scheduling barriers keep the
        // reads there: left to itself the compiler reads each operand just before its product
        // and waits.
        constexpr bool kAhead = is_bf16<T>() && !kMask;
        typename Block::Frag kf[2][Block::NK];
        auto load_keys = [&](int ks) __attribute__((always_inline)) {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int p = 0; p < Block::NK; ++p) {
                    // (subtile kk of half ks starts 32 ks + 4 kk (float: 16 kk) rows further: the
                    // swizzle of the lane's rows stays the same)
                    const int o = is_bf16<T>() ? 128 * (32 * ks + 4 * kk) : D * 4 * (32 * ks + 16 * kk);
                    kf[kk][p] = *reinterpret_cast<const typename Block::Frag*>(sm.k[buf] + koff[p] + o);
                }
        };
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            f32x4 x[2][NQ];
            load_keys(ks);
            if constexpr (is_bf16<T>()) __builtin_amdgcn_sched_barrier(0);
            blk.scores(x, start, [&](int kk, int p) __attribute__((always_inline)) { return kf[kk][p]; });
            __builtin_amdgcn_sched_barrier(0);
            bf16x8 vf[is_bf16<T>() ? Block::ND : 1];
            auto load_values = [&]() __attribute__((always_inline)) {
                if constexpr (is_bf16<T>()) {
#pragma unroll
                    for (int dt = 0; dt < Block::ND; ++dt) vf[dt] = tile_col8_at(sm.v[buf] + voff[dt] + 128 * 32 * ks);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            if constexpr (kAhead) load_values();
            float p[NQ][8];
            // weights of query subtile qt; form(qt, p): its y - ref
            auto weigh = [&](int qt, auto form) __attribute__((always_inline)) {
                if constexpr (kFixed) {
                    blk.weights_fixed(qt, p[qt]);
                } else {
                    auto moved = [&]() __attribute__((always_inline)) {
                        row[qt] = __builtin_fmaf(sm.rd[o0 + 16 * qt + r16].x, kLog2e, -blk.ref[qt]);
                    };
                    if (blk.weights(qt, p[qt], [&](float (&y)[8]) __attribute__((always_inline)) {
                            moved();
                            form(qt, y);
                        }))
                        moved();
                }
            };
            if constexpr (kMask) {
                float2 kd[8], rd[NQ];
#pragma unroll
                for (int j = 0; j < 8; ++j) kd[j] = sm.kd[buf][32 * ks + key_of<T>(g, j)];
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt) rd[qt] = sm.rd[o0 + 16 * qt + r16];
                // (held here: read where they are used, each read would stand in a branch of its own)
#pragma unroll
                for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(kd[j].x), "+v"(kd[j].y));
                auto form = [&](int qt, float (&y)[8]) __attribute__((always_inline)) {
                    // keys up to `last` of the half
                    const int last = keep[qt] ? pos_of(qt) - 64 * n - 32 * ks : -1;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float decay = (rd[qt].x - kd[j].x) + (rd[qt].y - kd[j].y);
                        const float v = __builtin_fmaf(x[j >> 2][qt][j & 3], kscale,
                                                       __builtin_fmaf(decay, kLog2e, -blk.ref[qt]));
                        y[j] = key_of<T>(g, j) <= last ? v : -INFINITY;
                    }
                };
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt) form(qt, p[qt]);
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt) weigh(qt, form);
            } else {
                float kb[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) kb[j] = sm.kb[buf][32 * ks + key_of<T>(g, j)];
                auto form = [&](int qt, float (&y)[8]) __attribute__((always_inline)) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        y[j] = __builtin_fmaf(x[j >> 2][qt][j & 3], kscale, kFixed ? kb[j] : kb[j] + row[qt]);
                };
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt) form(qt, p[qt]);
#pragma unroll
                for (int qt = 0; qt < NQ; ++qt) weigh(qt, form);
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (!kAhead) load_values();
            blk.add(p, [&](int dt, int j) __attribute__((always_inline)) {
                if constexpr (is_bf16<T>())
                    return vf[dt];
                else
                    return *reinterpret_cast<const float*>(
                        sm.v[buf] + f32_off<D>(32 * ks + key_of<T>(g, j), 16 * dt + r16));
            });
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    if (tid == 0) sm.marked = 0;
    for (int i = tid; i < 64 * NQ * 2 * (D / 32); i += 256) (&sm.inf[0][0][0])[i] = 0;
    if (nb <= ne) {
        win.fill(a, s, nb, lane);
        issue(nb, 0);
        put_gates(0);
        wait_vmcnt0();
        __syncthreads();
        int buf = 0, n = nb;
        // some row of the tile leaves out something of page n (in buffer buf)
        auto partly = [&]() { return n >= (p0 >> 6) || !(c_tile_last - sm.end[buf] >= delta); };
        auto next = [&](auto mask_tag, auto fixed_tag, const f32x4(&start)[NQ]) __attribute__((always_inline)) {
            constexpr bool kMask = decltype(mask_tag)::value;
            const int page = page_next;
            if (n < ne) issue(n + 1, buf ^ 1);
            unsigned long long bad = 0;
            if (kMask && page >= 0) {
                clean_values<T, D>(sm.v[buf], len - 64 * n, sm.bad[buf], tid, 256);
                lds_barrier();
                bad = (unsigned long long)sm.bad[buf][1] << 32 | sm.bad[buf][0];
            }
            if (page >= 0 && wave_on &&
                (!kMask || (n <= (w1 >> 6) && (n >= (w0 >> 6) || c_first - sm.end[buf] >= delta))))
                step(mask_tag, fixed_tag, start, n, buf);
            if (kMask && bad && wave_on) {
                sm.marked = 1;
#pragma unroll 1
                for (int qt = 0; qt < NQ; ++qt) {
                    const int pos = p0 + min(o0 + 16 * qt + r16, rows - 1);
                    if (o0 + 16 * qt + r16 < rows && (n >= (pos >> 6) || gate(pos) - sm.end[buf] >= delta))
                        mark_bad<T, D>(bad, vp + page * page_stride, 64 * n, pos, lane,
                                       sm.inf[16 * (NQ * wave + qt) + r16]);
                }
            }
            if (page < 0 && wave == 0) report(a, s, h, lane);
            if (n < ne) put_gates(buf ^ 1);
            wait_vmcnt0_lgkmcnt0();
            __syncthreads();
            ++n;
            buf ^= 1;
        };
        // (loops of their own, and a pair for each kind of head: one loop with all forms of the
        // step needs more registers than there are, and so do three that share the masked one)
        const std::true_type yes;
        const std::false_type no;
        const f32x4 zero[NQ] = {};
        if (fixed) {
            // (the products of a row start at its own term, in their units)
            f32x4 start[NQ];
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt) {
                const float x = row[qt] / kscale;
                start[qt] = f32x4{x, x, x, x};
            }
            while (n <= ne) {
                while (n <= ne && !partly()) next(no, yes, start);
                while (n <= ne && partly()) next(yes, yes, zero);
            }
        } else {
            while (n <= ne) {
                while (n <= ne && !partly()) next(no, no, zero);
                while (n <= ne && partly()) next(yes, no, zero);
            }
        }
    }
    if (wave_on) {
        float* slot = work.slots + (int64_t)(2 * wg + sh.later) * slot_floats<D>(kRows);
#pragma unroll
        for (int qt = 0; qt < NQ; ++qt) {
            const float l = over_groups(blk.l[qt]);
            const int r = o0 + 16 * qt + r16;
            if (r >= rows) continue;
            // (with a bound that holds: at least e^(-64) of the row's own key, at most 2^31 keys of
            // e^(2 kFixedMax - 64) = 2^58)
            const int own = (p0 + r) >> 6;
            if (fixed && (!(l <= 0x1p92f) || (l < 0x1p-96f && own >= nb && own <= ne))) report(a, s, h, g, kFlagScales);
            if (nb <= ne && sm.marked) add_marks<D>(blk.acc[qt], sm.inf[r], g);
            if (taken == it.pages) put_row<T, D>(a, it.t0 + r, h, blk.acc[qt], blk.max_logit(qt), l, g);
            else put_part<D, kRows>(slot, r, blk.acc[qt], blk.max_logit(qt), l, g);
        }
    }
    if (!next_item(work, sh, it)) return;
    __syncthreads();                                    // (the marks are read)
    }
}

// ---- short -----------------------------------------------------------------------------
template <typename T, int D>
struct alignas(1024) ShortSmem {
    // value tiles of each wave (float values go straight to registers); at an item's end the
    // wave's sums, [dt][lane]
    unsigned char v[4][2][is_bf16<T>() ? 64 * D * 2 : D * 32];
    unsigned bad[4][2];
    unsigned inf[16][2][D / 32];
    int marked;
    float m[4][16], l[4][16];
    ShareSmem share;
};

// The gates of a page for the heads of a group, in LDS: 16-byte piece i of head k at position
// i ^ k of its 32, so that a read of the same piece of all heads spreads over the banks.
struct GateDma {
    // bytes a wave needs for G heads
    __host__ __device__ static constexpr int bytes(int G) { return (G + 1) / 2 * 1024; }
    // src: the page's gates of the group's first head.  Two heads per instruction (of an odd
    // count the last one twice).  Waited for as TileDma's loads.
    static __device__ __forceinline__ void issue(unsigned char* to, const double* src, int G, int lane) {
        typedef __attribute__((address_space(3))) unsigned char lds_u8;
        const unsigned long long p = reinterpret_cast<unsigned long long>(src);
        const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)p);
        const unsigned hi = __builtin_amdgcn_readfirstlane((unsigned)(p >> 32));
        const unsigned long long base = ((unsigned long long)hi << 32) | lo;
        for (int k = 0; k < G; k += 2) {
            const int head = k + (lane >> 5);
            const unsigned off = min(head, G - 1) * 512 + (((lane & 31) ^ head) << 4);
            const unsigned lds = __builtin_amdgcn_readfirstlane(
                (unsigned)(unsigned long long)(const lds_u8*)(to + 512 * k));
            asm volatile(
                "s_mov_b32 m0, %0\n\t"
                "s_nop 0\n\t"
                "global_load_lds_dwordx4 %1, %2"
                :
                : "s"(lds), "v"(off), "s"(base)
                : "memory", "m0");
        }
    }
    static __device__ __forceinline__ double2 at(const unsigned char* from, int head, int piece) {
        return *reinterpret_cast<const double2*>(from + head * 512 + ((piece ^ head) << 4));
    }
};

// Rows r = token * G + head of the group, r < 16, are the queries of every wave.  A step's
// operands are requested one step ahead; at d = 64 in bfloat16 two workgroups fit a CU.
// gates_lds: the page's gates go through LDS (GateDma::bytes(G) more of it per wave), else each
// lane loads those of its head and keys.
template <typename T, int D>
__global__ __launch_bounds__(256, is_bf16<T>() && D == 64 ? 2 : 1) void paged_short_kernel(PagedArgs, Work work, float kscale,
                                                                           bool gates_lds) {
    typedef RowBlock<T, D, 1> Block;
    constexpr int KH = is_bf16<T>() ? 2 : 1;            // halves of 32 keys per step
    constexpr int ND = D / 16;
    __shared__ ShortSmem<T, D> sm;
    extern __shared__ __align__(16) unsigned char gates_s[];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wg = blockIdx.x;
    Share sh = find_share(work, wg, sm.share);
    if (sh.left == 0) return;
    for (;;) {
    const PagedArgs& a = late_args();
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63, g = lane >> 4, r16 = lane & 15;
    const Item it = item_at(work, sh.item);
    if (it.pages == 0) return;                          // (not in a share)
    const int s = it.s, hk = sh.item / work.tiles;
    int nb;
    const int taken = pages_here(work, sh, it, nb), ne = nb + taken - 1;
    if (work.shared && taken == 0) return;
    const int G = a.H / a.Hk, nrows = it.n * G, len = it.len;
    // the lane's row (those past the end repeat the last one)
    const int r = min(r16, nrows - 1);
    const int h = hk * G + r % G, pi = it.p0 + r / G;
    const int pp = page_of(a, s, pi >> 6);
    const double ci = pp < 0 ? 0.0 : gates_of(a, pp, h)[pi & 63];
    const double delta = head_delta(a, h);
    Block blk;
    blk.clear();
    blk.load_q(0, (const T*)a.q + (int64_t)(it.t0 + r / G) * a.qt + (int64_t)h * a.qh, g);

    if (tid == 0) sm.marked = 0;
    for (int i = tid; i < 16 * 2 * (D / 32); i += 256) (&sm.inf[0][0][0])[i] = 0;
    __syncthreads();

    // (all that the loops need of the arguments)
    const T* kp = (const T*)a.kp + (int64_t)hk * 64 * D;
    const T* vp = (const T*)a.vp + (int64_t)hk * 64 * D;
    const double* gates = a.cp + (int64_t)hk * G * 64;    // of the group's first head
    const int64_t page_stride = (int64_t)a.Hk * 64 * D, gate_stride = (int64_t)a.H * 64;
    const int head = r % G;
    unsigned char* gate_tile = gates_s + (gates_lds ? wave * GateDma::bytes(G) : 0);
    // What a step needs, requested one step ahead
    typename Block::Frag kf[KH][2][Block::NK];
    float vf[is_bf16<T>() ? 1 : ND][8];
    int page = -1;
    TileDma<D, 1> dma;
    if constexpr (is_bf16<T>()) dma.init(0, lane);
    PageWindow win;

    auto load_rest = [&](int n, int hf, int buf) __attribute__((always_inline)) {
        const int p = win.get(a, s, n, lane);
        page = p;
        const int64_t at = max(p, 0) * page_stride;
        if (gates_lds) GateDma::issue(gate_tile, gates + max(p, 0) * gate_stride, G, lane);
        if constexpr (is_bf16<T>()) {
            dma.issue(sm.v[wave][buf], vp + at, 0);
        } else {
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    vf[dt][j] = vp[at + (int64_t)(32 * hf + key_of<T>(g, j)) * D + 16 * dt + r16];
        }
    };
    auto load_keys = [&](int hf) __attribute__((always_inline)) {
        const int64_t at = max(page, 0) * page_stride;
#pragma unroll
        for (int ks = 0; ks < KH; ++ks)
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int i = 0; i < Block::NK; ++i)
                    kf[ks][kk][i] = *reinterpret_cast<const typename Block::Frag*>(
                        kp + at + (int64_t)(32 * (ks + hf) + key_row<T>(kk, r16)) * D +
                        4 * Block::kFrag * i + Block::kFrag * g);
    };

    // wave w takes steps w, w + 4, .. of the part's pages (or half pages)
    const int steps = nb <= ne ? (ne - nb + 1) * (is_bf16<T>() ? 1 : 2) : 0;
    auto page_at = [&](int u) { return nb + (is_bf16<T>() ? u : u >> 1); };
    if (wave < steps) {
        win.fill(a, s, nb, lane);
        load_rest(page_at(wave), is_bf16<T>() ? 0 : wave & 1, 0);
        load_keys(is_bf16<T>() ? 0 : wave & 1);
    }
    int buf = 0;
    for (int u = wave; u < steps; u += 4, buf ^= 1) {
        const int n = page_at(u), hf = is_bf16<T>() ? 0 : u & 1;
        const int pg = page;
        // The step's operands, each followed by the request for the next step's: c_i - c_j and
        // the values in registers first, then the keys (none is held twice)
        float decay[KH][8];
        double end;
        if (gates_lds) {
            wait_vmcnt0();
#pragma unroll
            for (int ks = 0; ks < KH; ++ks)
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const double2 c = GateDma::at(gate_tile, head, (32 * (ks + hf) + key_of<T>(g, j)) >> 1);
                    decay[ks][j] = (float)(ci - c.x);
                    decay[ks][j + 1] = (float)(ci - c.y);
                }
            end = GateDma::at(gate_tile, head, 31).y;
            asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
        } else {
            const double* cp = gates + max(pg, 0) * gate_stride + head * 64;
#pragma unroll
            for (int ks = 0; ks < KH; ++ks)
#pragma unroll
                for (int j = 0; j < 8; ++j) decay[ks][j] = (float)(ci - cp[32 * (ks + hf) + key_of<T>(g, j)]);
            end = cp[63];
            wait_vmcnt0();
        }
        float vc[is_bf16<T>() ? 1 : ND][8];
        if constexpr (!is_bf16<T>()) {
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int j = 0; j < 8; ++j) vc[dt][j] = vf[dt][j];
        }
        const int next_half = is_bf16<T>() ? 0 : u & 1;
        if (u + 4 < steps) load_rest(page_at(u + 4), next_half, buf ^ 1);
        f32x4 x[KH][2][1];
        const f32x4 none[1] = {};
#pragma unroll
        for (int ks = 0; ks < KH; ++ks)
            blk.scores(x[ks], none, [&](int kk, int i) __attribute__((always_inline)) { return kf[ks][kk][i]; });
        if (u + 4 < steps) load_keys(next_half);
        if (pg < 0) {
            if (r16 < nrows) report(a, s, h, lane & 48);
            continue;
        }
        const bool keep = n >= (pi >> 6) || ci - end >= delta;
        const bool partly = __any(!(keep && 64 * n + 63 <= pi));
        unsigned long long bad = 0;
        if (partly) {
            const int valid = len - 64 * n;
            if constexpr (is_bf16<T>()) {
                if (lane < 2) sm.bad[wave][lane] = 0;
                __builtin_amdgcn_wave_barrier();
                clean_values<T, D>(sm.v[wave][buf], valid, sm.bad[wave], lane, 64);
                asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
                bad = (unsigned long long)sm.bad[wave][1] << 32 | sm.bad[wave][0];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int key = 32 * hf + key_of<T>(g, j);
                    bool found = false;
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt) {
                        const bool f = !__builtin_isfinite(vc[dt][j]);
                        if (key >= valid || f) vc[dt][j] = 0.f;
                        found |= f && key < valid;
                    }
                    const unsigned long long b = __ballot(found);
#pragma unroll
                    for (int gg = 0; gg < 4; ++gg)
                        if ((b >> (16 * gg)) & 0xffffull) bad |= 1ull << (32 * hf + key_of<T>(gg, j));
                }
            }
        }
#pragma unroll
        for (int ks = 0; ks < KH; ++ks) {
            float p[1][8];
            auto form = [&](float (&y)[8]) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int key = 32 * (ks + hf) + key_of<T>(g, j);
                    const bool on = keep && 64 * n + key <= pi;
                    const float v = __builtin_fmaf(x[ks][j >> 2][0][j & 3], kscale,
                                                   __builtin_fmaf(decay[ks][j], kLog2e, -blk.ref[0]));
                    y[j] = on ? v : -INFINITY;
                }
            };
            form(p[0]);
            blk.weights(0, p[0], form);
            blk.add(p, [&](int dt, int j) __attribute__((always_inline)) {
                if constexpr (is_bf16<T>()) return tile_col8(sm.v[wave][buf], 32 * ks + 8 * g, 16 * dt, r16);
                else return vc[dt][j];
            });
        }
        if (bad) {
            sm.marked = 1;
            if (keep && r16 < nrows)
                mark_bad<T, D>(bad, vp + pg * page_stride, 64 * n, pi, lane, sm.inf[r16]);
        }
    }

    // the four waves' sums: maxima and sums first, then O through the value tiles' LDS
    const float l = over_groups(blk.l[0]);
    if (g == 0) {
        sm.m[wave][r16] = blk.max_logit(0);
        sm.l[wave][r16] = l;
    }
    __syncthreads();
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, sm.m[w][r16]);
    const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int w = 0; w < 4; ++w) L += sm.l[w][r16] * fast_exp2(sm.m[w][r16] - ref);
    const float scale = fast_exp2(blk.max_logit(0) - ref);
    // (a wave's tiles are no longer read)
    auto o_s = [&](int w) __attribute__((always_inline)) { return reinterpret_cast<f32x4(*)[64]>(&sm.v[w][0][0]); };
    if (wave > 0)
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) o_s(wave)[dt][lane] = blk.acc[0][dt] * scale;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
            f32x4 o = blk.acc[0][dt] * scale;
#pragma unroll
            for (int w = 1; w < 4; ++w) o += o_s(w)[dt][lane];
            blk.acc[0][dt] = o;
        }
        if (sm.marked) add_marks<D>(blk.acc[0], sm.inf[r16], g);
        if (r16 < nrows) {
            if (taken == it.pages) put_row<T, D>(a, it.t0 + r / G, h, blk.acc[0], M, L, g);
            else put_part<D, 16>(work.slots + (int64_t)(2 * wg + sh.later) * slot_floats<D>(16), r16,
                                 blk.acc[0], M, L, g);
        }
    }
    if (!next_item(work, sh, it)) return;
    __syncthreads();                                    // (the sums and marks are read)
    }
}

// ---- merge -----------------------------------------------------------------------------
// The partial sums of an item that lies in several shares, of R rows per slot.  A workgroup
// per share, for the item whose first cut lies at the share's start, and per 16 rows: 16 lanes
// take a row (four rows of a slot in one load of a wave), or, of fewer rows, every so many
// lanes' parts of it.  The first long_wgs workgroups merge long items, the others short ones.
template <typename T, int D, int kLongRows>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedArgs a, Work lw, Work sw, int long_wgs) {
    constexpr int kPer = D / 64;                         // features 64 k + 4 l .. + 3 of lane l
    __shared__ float sm[16][D + 2];
    const bool is_long = (int)blockIdx.x < long_wgs;
    const Work w = is_long ? lw : sw;
    constexpr int kTiles = kLongRows / 16;
    const int R = is_long ? kLongRows : kShortRows;
    const int wg = 1 + (is_long ? (int)blockIdx.x / kTiles : (int)blockIdx.x - long_wgs);
    const Cut cut = w.cuts[wg];
    if (cut.item < 0) return;
    const int id = cut.item;
    const Item it = w.items[id];
    const int G = a.H / a.Hk, r0 = is_long ? 16 * ((int)blockIdx.x % kTiles) : 0;
    const int rows = min(16, (is_long ? it.n : it.n * G) - r0);
    if (rows <= 0) return;
    // the share before has its first pages; its last one lies here or in a later share
    const int w0 = wg - 1, parts = 2 + (w.setup - cut.skip + it.pages - 1) / cut.chunk;
    const int group = threadIdx.x >> 4, l16 = threadIdx.x & 15;
    const int each = rows == 1 ? 16 : rows == 2 ? 8 : rows <= 4 ? 4 : rows <= 8 ? 2 : 1;   // groups per row
    const int r = r0 + group / each, first = group % each;
    const bool on = group / each < rows;
    float M = -INFINITY, L = 0.f;
    f32x4 o[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) o[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    // (a part without a key of the row has zeros and the weight 0)
    auto merge = [&](float m, float l, const f32x4 (&v)[kPer]) __attribute__((always_inline)) {
        const float top = fmaxf(M, m), ref = top == -INFINITY ? 0.f : top;
        const float x = fast_exp2(M - ref), y = fast_exp2(m - ref);
        M = top;
        L = L * x + l * y;
#pragma unroll
        for (int k = 0; k < kPer; ++k) o[k] = o[k] * x + v[k] * y;
    };
    if (on) {
        constexpr int kAtOnce = 4;
        for (int p = first; p < parts; p += kAtOnce * each) {
            float2 ml[kAtOnce];
            f32x4 v[kAtOnce][kPer];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const int q = min(p + i * each, parts - 1);
                const bool later = q == 0 && cut.skip < cut.chunk;
                const float* slot = w.slots + (int64_t)(2 * (w0 + q) + later) * slot_floats<D>(R);
                ml[i] = *reinterpret_cast<const float2*>(slot + R * D + 2 * r);
#pragma unroll
                for (int k = 0; k < kPer; ++k)
                    v[i][k] = *reinterpret_cast<const f32x4*>(slot + r * D + 64 * k + 4 * l16);
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
                if (p + i * each < parts) merge(ml[i].x, ml[i].y, v[i]);
        }
    }
    if (each > 1) {
#pragma unroll
        for (int k = 0; k < kPer; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) sm[group][64 * k + 4 * l16 + e] = o[k][e];
        if (l16 == 0) {
            sm[group][D] = M;
            sm[group][D + 1] = L;
        }
        __syncthreads();
        if (first > 0) return;
        for (int i = 1; i < each; ++i) {
            const float* q = sm[group + i];
            f32x4 v[kPer];
#pragma unroll
            for (int k = 0; k < kPer; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[k][e] = q[64 * k + 4 * l16 + e];
            merge(q[D], q[D + 1], v);
        }
    }
    if (!on) return;
    const int h = is_long ? long_head(a, id, w.tiles) : id / w.tiles * G + r % G;
    const int64_t row = (int64_t)(it.t0 + (is_long ? r : r / G)) * a.H + h;
    const float inv = L == 0.f ? 0.f : 1.0f / L;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        T out[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = from_f32<T>(o[k][e] * inv);
        __builtin_memcpy((T*)a.O + row * D + 64 * k + 4 * l16, out, sizeof(out));
    }
    if (l16 == 0) a.lse[row] = L == 0.f ? -INFINITY : (M + fast_log2(L)) * kLn2;
}

__global__ __launch_bounds__(256) void paged_flags_kernel(PagedArgs a, int limit) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)a.N * a.H) return;
    const int s = (int)(i / a.H), h = (int)(i - (int64_t)s * a.H);
    int f = seq_of(a, s).n > limit ? kFlagMaxNew : 0;
    if (a.gamma_q) {
        const float gq = a.gamma_q[h], gk = a.gamma_k[h / (a.H / a.Hk)];
        if (!(gq >= 0.f && gq < INFINITY) || !(gk >= 0.f && gk < INFINITY)) f |= 8;
    }
    a.flags[i] = f;
}

// How a call is divided.  Sequences of at most short_max new tokens go to the short kernel,
// the others to the long one, tiles of 64 nq rows.
struct Division {
    int short_max, long_above, nq, limit;     // limit: rows of a sequence that its kernels take
    bool short_on, long_on;
    Work lw, sw;       // offsets from the workspace in place of the pointers
    size_t bytes;
};

// (at least so many workgroups, so that a max_len that is too small still spreads the pages)
constexpr int kLeastShares = 96;

// A kernel's items, and their shares: `fit` workgroups (what the chip holds at a time), no
// share under `least` pages.  Items that are many more, or have few pages, are not shared
// out: at 8 items per workgroup the last ones to finish cost an eighth at most (8400 items of
// 10 to 20 pages 355 us, shared out 381; at 3000 items of 16 to 45 pages both take 242).
void share_out(Work& w, int64_t items, int fit, int setup, int least, int64_t pages) {
    w.n = (int)items;
    w.least = least;
    w.setup = setup;
    w.shared = items < 8 * (int64_t)fit && pages > least;
    int64_t wgs = items * pages / least + 1;
    wgs = wgs < kLeastShares ? kLeastShares : wgs > fit ? fit : wgs;
    w.wgs = w.shared ? (int)wgs : w.n;
}

Division divide(const PagedArgs& a) {
    Division v{};
    const int G = a.H / a.Hk, es = a.bf16 ? 2 : 4;
    v.short_max = kShortRows / G;
    const int64_t pages = (a.max_len + 63) / 64;
    v.long_on = a.N > 0 && a.max_new > v.short_max;
    v.limit = v.long_on ? 0x7fffffff : v.short_max;
    v.nq = 1;
    if (a.N == 0) return v;
    // (rows in equal parts that are long: no sequence is short)
    v.short_on = !v.long_on || (int64_t)a.N * a.max_new != a.T;
    v.long_above = v.short_on ? v.short_max : 0;
    // (4 x 64 rows behind 4000, 12 heads of 64: 28 us at one, 32 at two; 2 x 4096 rows behind 4096
    // 179 at two, 241 at one, on a box slower than the one of the head of this file)
    v.nq = a.max_new > 64 ? 2 : 1;
    const int rows = 64 * v.nq;
    auto take = [&](size_t n) {
        const size_t at = v.bytes;
        v.bytes += (n + 255) & ~(size_t)255;
        return at;
    };
    auto place = [&](Work& w, int r) {
        w.items = (Item*)take((size_t)w.n * sizeof(Item));
        w.places = (int*)take((size_t)w.n * sizeof(int));
        if (!w.shared) return;
        w.cuts = (Cut*)take((size_t)w.wgs * sizeof(Cut));
        w.slots = (float*)take((size_t)2 * w.wgs * r * (a.d + 2) * sizeof(float));
    };
    if (v.long_on) {
        // (no more tiles than this, however T rows are dealt to N sequences)
        v.lw.tiles = (int)((a.T + (int64_t)a.N * (rows - 1)) / rows);
        // workgroups at a time: by registers three per CU (d = 64, bfloat16) or by LDS two, one
        const int fit = 256 * (a.d * es == 128 ? 3 : a.d * es == 256 ? 2 : 1);
        // taking up an item costs 9 of the faster pages of bfloat16 (8000 rows behind 8150 591 us,
        // counted as 4 623, as 16 598; chunks beside single tokens 70, 73, 75), 2 of float32's
        share_out(v.lw, (int64_t)v.lw.tiles * a.H, fit, a.bf16 ? 9 : 2, a.bf16 ? 10 : 4, pages);
        place(v.lw, rows);
    }
    if (v.short_on) {
        v.sw.tiles = a.N;
        // two workgroups per CU in bfloat16 (d = 128 holds one at a time: 16 tokens of 32 heads on 4
        // key heads 103 us, with one per CU 105), one in float32 (8 tokens of 12 heads 59 us, with
        // two 67); an item costs 7 pages (256 tokens 242 us, counted as 4 264; the 16 tokens 103,
        // counted as 10 107)
        share_out(v.sw, (int64_t)a.N * a.Hk, a.bf16 ? 512 : 256, 7, 8, pages);
        place(v.sw, kShortRows);
    }
    return v;
}

template <typename T, int D, int NQ>
void attend(const PagedArgs& a, const Division& v, hipStream_t s) {
    const float kscale = kLog2e / sqrtf((float)D);
    Work lw = v.lw, sw = v.sw;
    for (Work* w : {&lw, &sw}) {
        w->items = (Item*)((char*)a.part + (size_t)w->items);
        w->places = (int*)((char*)a.part + (size_t)w->places);
        w->cuts = (Cut*)((char*)a.part + (size_t)w->cuts);
        w->slots = (float*)((char*)a.part + (size_t)w->slots);
    }
    const int G = a.H / a.Hk, waves = G <= 1 ? 1 : G <= 2 ? 2 : G <= 4 ? 4 : 8;   // of a short item
    const int fill_at = (lw.n + 7) / 8 + (sw.n * waves + 7) / 8, fill = a.fill ? (a.T + 511) / 512 : 0;
    hipLaunchKernelGGL((paged_plan_kernel<T, 64 * NQ>), dim3(fill_at + fill), dim3(512), 0, s, a, lw, sw,
                       v.short_max, v.long_above, waves, fill_at, v.limit);
    if (v.long_on)
        hipLaunchKernelGGL((paged_long_kernel<T, D, NQ>), dim3(lw.wgs), dim3(256), 0, s, a, lw, kscale);
    if (v.short_on) {
        // (all of a CU's 160 KB hold the gates of 16 heads beside the values of d = 128, but no more)
        const size_t gates = 4 * GateDma::bytes(G);
        const bool fits = sizeof(ShortSmem<T, D>) + gates <= 160 * 1024;
        hipLaunchKernelGGL((paged_short_kernel<T, D>), dim3(sw.wgs), dim3(256), fits ? gates : 0, s, a, sw, kscale,
                           fits);
    }
    const int long_wgs = lw.shared ? (lw.wgs - 1) * 4 * NQ : 0, short_wgs = sw.shared ? sw.wgs - 1 : 0;
    if (long_wgs + short_wgs > 0)
        hipLaunchKernelGGL((paged_join_kernel<T, D, 64 * NQ>), dim3(long_wgs + short_wgs), dim3(256), 0, s, a, lw,
                           sw, long_wgs);
}
template <typename T, int D>
void attend(const PagedArgs& a, const Division& v, hipStream_t s) {
    v.nq == 2 ? attend<T, D, 2>(a, v, s) : attend<T, D, 1>(a, v, s);
}

}  // namespace

size_t paged_workspace(const PagedArgs& a) { return divide(a).bytes; }

hipError_t launch_paged_attend(const PagedArgs& a, hipStream_t s) {
    trace_begin(ACP_K_COUNT + ACP_OP_ATTEND, s);
    const Division v = divide(a);
    if (a.flags && a.N > 0)
        hipLaunchKernelGGL(paged_flags_kernel, dim3((unsigned)(((int64_t)a.N * a.H + 255) / 256)), dim3(256), 0,
                           s, a, v.limit);
    if (a.T > 0) {
        if (a.bf16 && a.d == 64) attend<__bf16, 64>(a, v, s);
        else if (a.bf16) attend<__bf16, 128>(a, v, s);
        else if (a.d == 64) attend<float, 64>(a, v, s);
        else attend<float, 128>(a, v, s);
    }
    const hipError_t e = hipGetLastError();
    trace_end(ACP_K_COUNT + ACP_OP_ATTEND, s);
    return e;
}

}  // namespace acp
