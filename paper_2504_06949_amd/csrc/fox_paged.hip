// Attention of new tokens over a paged cache (fox_attn_paged): the row at position i of head
// h over the positions j <= i of its sequence, logits x_ij = q_i.k_j / sqrt(d) + c_i - c_j,
// pages left out row by row by the block test of ACP.
//
// Two kernels share the arithmetic (RowBlock): S^T = K Q^T on the matrix cores, so that a
// lane holds one query and eight keys of a 32-key half, the running maximum and sum of the
// softmax per query, and O^T += V^T P^T.
//   paged_long_kernel   64 or 128 rows of one head per workgroup, 16 or 32 per wave; the
//                       waves share the pages in LDS.  Bound by the matrix cores and the
//                       exponentials.
//   paged_short_kernel  the rows of all query heads of a key head, where they are at most
//                       16 in a sequence (single tokens above all): the waves take different
//                       pages of the same rows.  Bound by memory: a page is read once for
//                       all query heads that share it.
// Where rows are few, a sequence's kept pages are divided among several workgroups, whose
// partial sums paged_join_kernel merges (a launch of its own orders them without a
// device-wide fence).
#include <type_traits>

#include "acp_paged.h"
#include "acp_scan.h"

namespace acp {
namespace {

constexpr int kShortRows = 16;    // rows of a short sequence: new tokens times query heads
constexpr int kMaxSplit = 64;     // parts of a row's keys (a lane each in the merge)
constexpr float kSlack = 8.f;     // a weight is at most 2^8

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
    // s[kk][qt] = init[qt] + K Q^T of subtile kk; k(kk, piece) gives the lane's A operand
    template <typename F>
    __device__ __forceinline__ void scores(f32x4 (&s)[2][NQ], const float (&init)[NQ], F k) const {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt) s[kk][qt] = f32x4{init[qt], init[qt], init[qt], init[qt]};
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
    // y - ref (log2 units, -inf: left out) -> weights; true if ref[qt] moved
    __device__ __forceinline__ bool weights(int qt, float (&y)[8]) {
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
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] -= mx;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            y[j] = fast_exp2(y[j]);
            l[qt] += y[j];
        }
        return move;
    }
    // acc += V^T P^T; v(dt, j): bf16 the lane's eight keys of column 16 dt + r (j unused),
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
                                       int& seq, int& local) {
    int before = 0;
    for (int base = 0; base < a.N; base += 64) {
        int t = 0;
        if (base + lane < a.N) {
            const Seq q = seq_of(a, base + lane);
            if (q.n > lo && q.n <= hi) t = (q.n + rows - 1) / rows;
        }
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
            return true;
        }
        before += __shfl(incl, 63);
    }
    return false;
}

__device__ __forceinline__ double head_delta(const PagedArgs& a, int h) {
    if (!(a.log_lmax_over_eps < INFINITY)) return -INFINITY;
    const double u = ((double)a.gamma_q[h] * (double)a.gamma_k[h / (a.H / a.Hk)]) * __builtin_sqrt((double)a.d);
    return -(2.0 * u + a.log_lmax_over_eps);
}

// First page that the row at page nd with cumulative gate ci keeps: the test grows with the
// page, and 64 pages are probed at a time.  A page that is not in the cache counts as left
// out (it may have been dropped).
__device__ __forceinline__ int first_page(const PagedArgs& a, int s, int h, int nd, double ci, double delta,
                                          int lane) {
    if (delta == -INFINITY) return 0;
    int lo = 0, hi = nd;                    // the answer lies in [lo, hi]; hi is kept
    while (lo < hi) {
        const int step = (hi - lo + 63) / 64;
        const int n = lo + lane * step;
        bool keep = true;
        if (n < hi) {
            const int p = page_of(a, s, n);
            keep = p >= 0 && ci - gates_of(a, p, h)[63] >= delta;
        }
        const unsigned long long k = __ballot(keep);
        const int f = k ? __builtin_ctzll(k) : 64;
        const int top = min(lo + f * step, hi);
        if (f > 0) lo = min(lo + (f - 1) * step + 1, top);
        hi = top;
    }
    return lo;
}

// Page numbers of 64 consecutive pages, one per lane
struct PageWindow {
    int base, id;
    __device__ __forceinline__ void fill(const PagedArgs& a, int s, int n, int lane) {
        base = n;
        id = page_of(a, s, n + lane);
    }
    __device__ __forceinline__ int get(const PagedArgs& a, int s, int n, int lane) {
        if (n - base >= 64) fill(a, s, n, lane);
        return __builtin_amdgcn_readlane(id, n - base);
    }
};

__device__ __forceinline__ void report(const PagedArgs& a, int s, int h, int lane) {
    if (a.flags && lane == 0) atomicOr(a.flags + (int64_t)s * a.H + h, kFlagPage);
}

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

// Workgroup -> (head, item).  Workgroups go to the 8 XCDs in turn; each XCD takes every
// eighth item of every head, heads fastest.  Heads keep different numbers of pages, and
// this gives each XCD the same share of each; the workgroups at work on an XCD at one time
// are neighbouring items of all heads, so that those that read the same pages share its L2.
__device__ __forceinline__ void deal(int heads, int& h, int& item) {
    const int x = blockIdx.x & 7, k = blockIdx.x >> 3;
    h = k % heads;
    item = k / heads * 8 + x;
}
__host__ inline unsigned dealt(int64_t items, int heads) { return (unsigned)((items + 7) / 8 * 8 * heads); }

// Row t, head h of the output, or its share of the part `sp` of `splits`
template <typename T, int D>
__device__ __forceinline__ void put_row(const PagedArgs& a, int t, int h, int sp, int splits, int stride,
                                        const f32x4 (&acc)[D / 16], float m, float l, int g) {
    const int64_t row = (int64_t)t * a.H + h;
    if (splits == 1) {
        const float inv = l == 0.f ? 0.f : 1.0f / l;     // (no key: every page was bad)
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) {
            T o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = from_f32<T>(acc[dt][k] * inv);
            __builtin_memcpy((T*)a.O + row * D + 16 * dt + 4 * g, o, sizeof(o));
        }
        if (g == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + fast_log2(l)) * kLn2;
    } else {
        float2* ml = reinterpret_cast<float2*>(a.part) + row * stride;
        float* po = a.part + 2 * (int64_t)a.T * a.H * stride + (row * stride + sp) * D;
        if (g == 0) ml[sp] = make_float2(m, l);
        if (m > -INFINITY || m != m)
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt)
                *reinterpret_cast<f32x4*>(po + 16 * dt + 4 * g) = acc[dt];
    }
}

// ---- long ------------------------------------------------------------------------------
template <typename T, int D, int NQ>
struct alignas(1024) LongSmem {
    unsigned char k[2][64 * D * sizeof(T)];
    unsigned char v[2][64 * D * sizeof(T)];
    float kb[2][64];         // (c_j - R) log2(e), negated
    float2 kd[2][64];        // c_j - R as a sum of two floats
    double end[2];           // c of the page's last position
    unsigned bad[2][2];      // keys of the page with values that are not finite
    unsigned inf[64 * NQ][2][D / 32];
    int marked;
};

template <typename T, int D, int NQ>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 && is_bf16<T>() ? 3 : 2)))
void paged_long_kernel(PagedArgs a, int tiles, int splits, int stride, int short_max, float kscale) {
    constexpr int kRows = 64 * NQ;
    typedef RowBlock<T, D, NQ> Block;
    __shared__ LongSmem<T, D, NQ> sm;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, g = lane >> 4, r16 = lane & 15;
    int h, rest;
    deal(a.H, h, rest);
    const int sp = rest % splits;
    if (rest / splits >= tiles) return;
    int s, tile;
    // (the last tiles of a sequence have the most pages: they go first)
    if (!locate(a, tiles - 1 - rest / splits, kRows, short_max, 0x7fffffff, lane, s, tile)) return;
    const Seq q = seq_of(a, s);
    const int hk = h / (a.H / a.Hk);
    const double delta = readfirst_f64(head_delta(a, h));
    const int row0 = tile * kRows, rows = min(kRows, q.n - row0);    // of the sequence's new rows
    const int p0 = q.past + row0, p1 = p0 + rows - 1;                // positions of the tile
    const int len = q.past + q.n;
    const int nd1 = p1 >> 6;

    auto gate = [&](int pos) __attribute__((always_inline)) {
        const int p = page_of(a, s, pos >> 6);
        return p < 0 ? 0.0 : gates_of(a, p, h)[pos & 63];
    };
    const double R = readfirst_f64(gate(p0));
    const int lo = first_page(a, s, h, p0 >> 6, R, delta, lane);
    // this part's pages, of those the table has (the last one there may be is W - 1)
    const int top = min(nd1, a.W - 1), pages = max(top - lo + 1, 0), per = (pages + splits - 1) / splits;
    const int nb = lo + sp * per, ne = min(nb + per - 1, top);
    if (nd1 >= a.W && wave == 0) report(a, s, h, lane);

    Block blk;
    blk.clear();
    // rows of the wave and of the lane (those past the end repeat the last one)
    // (counted from p0: positions may be as large as an int holds)
    const int o0 = 16 * NQ * wave;
    const bool wave_on = o0 < rows;
    const int w0 = p0 + min(o0, rows - 1), w1 = p0 + min(o0 + 16 * NQ - 1, rows - 1);
    double ci[NQ];
    int pi[NQ];
    float2 rd[NQ];                                                   // c_i - R likewise
    float init[NQ], zero[NQ];                                        // start of the scores
    const float per_y = sqrtf((float)D) * kLn2;                      // q.k per unit of y
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
        pi[qt] = p0 + min(o0 + 16 * qt + r16, rows - 1);
        ci[qt] = gate(pi[qt]);
        blk.load_q(qt, (const T*)a.q + (int64_t)(q.row0 + pi[qt] - q.past) * a.qt + (int64_t)h * a.qh, g);
        const double r = ci[qt] - R;
        rd[qt].x = (float)r;
        rd[qt].y = (float)(r - (double)rd[qt].x);
        init[qt] = rd[qt].x * (kLog2e * per_y);
        zero[qt] = 0.f;
    }
    const double c_first = readfirst_f64(ci[0]);
    const double c_tile_last = readfirst_f64(gate(p1));

    PageDma<T, D> dma;
    dma.init(wave, lane);
    PageWindow win;
    const T* kp = (const T*)a.kp;
    const T* vp = (const T*)a.vp;
    double cn = 0.0;                        // the next page's gate, thread t < 64
    int page_next = -1;                     // the page last asked for, -1: not in the cache
    auto issue = [&](int n, int buf) __attribute__((always_inline)) {
        const int p = win.get(a, s, n, lane);
        const int64_t at = ((int64_t)max(p, 0) * a.Hk + hk) * 64 * D;
        page_next = p;
        if (threadIdx.x < 64) cn = gates_of(a, max(p, 0), h)[threadIdx.x];
        dma.issue(sm.k[buf], kp + at, wave);
        dma.issue(sm.v[buf], vp + at, wave);
    };
    auto put_gates = [&](int buf) __attribute__((always_inline)) {
        if (threadIdx.x < 64) {
            const double r = cn - R;
            const float hi = (float)r;
            sm.kb[buf][threadIdx.x] = -hi * kLog2e;
            sm.kd[buf][threadIdx.x] = make_float2(hi, (float)(r - (double)hi));
            if (threadIdx.x == 63) sm.end[buf] = cn;
            if (threadIdx.x < 2) sm.bad[buf][threadIdx.x] = 0;
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

    auto step = [&](auto mask_tag, int n, int buf) __attribute__((always_inline)) {
        constexpr bool kMask = decltype(mask_tag)::value;
        bool keep[NQ];
        if constexpr (kMask) {
            const double end = sm.end[buf];
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt) keep[qt] = n >= (pi[qt] >> 6) || ci[qt] - end >= delta;
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            f32x4 x[2][NQ];
            __builtin_amdgcn_sched_barrier(0);
            blk.scores(x, kMask ? zero : init, [&](int kk, int p) __attribute__((always_inline)) {
                // (subtile kk of half ks starts 32 ks + 4 kk (float: 16 kk) rows further: the
                // swizzle of the lane's rows stays the same)
                const int o = is_bf16<T>() ? 128 * (32 * ks + 4 * kk) : D * 4 * (32 * ks + 16 * kk);
                return *reinterpret_cast<const typename Block::Frag*>(sm.k[buf] + koff[p] + o);
            });
            __builtin_amdgcn_sched_barrier(0);
            float p[NQ][8];
#pragma unroll
            for (int qt = 0; qt < NQ; ++qt) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int key = 32 * ks + key_of<T>(g, j);
                    float y;
                    if constexpr (kMask) {
                        const float2 kd = sm.kd[buf][key];
                        const float decay = (rd[qt].x - kd.x) + (rd[qt].y - kd.y);
                        y = __builtin_fmaf(x[j >> 2][qt][j & 3], kscale,
                                           __builtin_fmaf(decay, kLog2e, -blk.ref[qt]));
                        if (!keep[qt] || 64 * n + key > pi[qt]) y = -INFINITY;
                    } else {
                        y = __builtin_fmaf(x[j >> 2][qt][j & 3], kscale, sm.kb[buf][key]);
                    }
                    p[qt][j] = y;
                }
                if (blk.weights(qt, p[qt])) init[qt] = __builtin_fmaf(rd[qt].x, kLog2e, -blk.ref[qt]) * per_y;
            }
            __builtin_amdgcn_sched_barrier(0);
            blk.add(p, [&](int dt, int j) __attribute__((always_inline)) {
                if constexpr (is_bf16<T>())
                    return tile_col8_at(sm.v[buf] + voff[dt] + 128 * 32 * ks);
                else
                    return *reinterpret_cast<const float*>(
                        sm.v[buf] + f32_off<D>(32 * ks + key_of<T>(g, j), 16 * dt + r16));
            });
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    if (threadIdx.x == 0) sm.marked = 0;
    for (int i = threadIdx.x; i < 64 * NQ * 2 * (D / 32); i += 256) (&sm.inf[0][0][0])[i] = 0;
    if (nb <= ne) {
        win.fill(a, s, nb, lane);
        issue(nb, 0);
        put_gates(0);
        wait_vmcnt0();
        __syncthreads();
        int buf = 0, n = nb;
        // some row of the tile leaves out something of page n (in buffer buf)
        auto partly = [&]() { return n >= (p0 >> 6) || !(c_tile_last - sm.end[buf] >= delta); };
        auto next = [&](auto mask_tag) __attribute__((always_inline)) {
            constexpr bool kMask = decltype(mask_tag)::value;
            const int page = page_next;
            if (n < ne) issue(n + 1, buf ^ 1);
            unsigned long long bad = 0;
            if (kMask && page >= 0) {
                clean_values<T, D>(sm.v[buf], len - 64 * n, sm.bad[buf], threadIdx.x, 256);
                lds_barrier();
                bad = (unsigned long long)sm.bad[buf][1] << 32 | sm.bad[buf][0];
            }
            if (page >= 0 && wave_on &&
                (!kMask || (n <= (w1 >> 6) && (n >= (w0 >> 6) || c_first - sm.end[buf] >= delta))))
                step(mask_tag, n, buf);
            if (kMask && bad && wave_on) {
                sm.marked = 1;
#pragma unroll 1
                for (int qt = 0; qt < NQ; ++qt) {
                    const int pos = p0 + min(o0 + 16 * qt + r16, rows - 1);
                    if (o0 + 16 * qt + r16 < rows && (n >= (pos >> 6) || gate(pos) - sm.end[buf] >= delta))
                        mark_bad<T, D>(bad, vp + ((int64_t)page * a.Hk + hk) * 64 * D, 64 * n, pos, lane,
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
        // (two loops: one with both forms of the step needs more registers than there are)
        while (n <= ne) {
            while (n <= ne && !partly()) next(std::false_type{});
            while (n <= ne && partly()) next(std::true_type{});
        }
    }
    if (!wave_on) return;
#pragma unroll
    for (int qt = 0; qt < NQ; ++qt) {
        const float l = over_groups(blk.l[qt]);
        if (o0 + 16 * qt + r16 >= rows) continue;
        if (nb <= ne && sm.marked) add_marks<D>(blk.acc[qt], sm.inf[16 * (NQ * wave + qt) + r16], g);
        put_row<T, D>(a, q.row0 + pi[qt] - q.past, h, sp, splits, stride, blk.acc[qt], blk.max_logit(qt), l, g);
    }
}

// ---- short -----------------------------------------------------------------------------
template <typename T, int D>
struct alignas(1024) ShortSmem {
    // value tiles of each wave (bf16; float values go straight to registers)
    unsigned char v[4][2][is_bf16<T>() ? 64 * D * 2 : 1024];
    unsigned bad[4][2];
    unsigned inf[16][2][D / 32];
    int marked;
    float m[4][16], l[4][16];
    int first[16];
};

// Rows r = token * G + head of the group, r < 16, are the queries of every wave.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_short_kernel(PagedArgs a, int splits, int stride, int short_max,
                                                          float kscale) {
    typedef RowBlock<T, D, 1> Block;
    constexpr int KH = is_bf16<T>() ? 2 : 1;            // halves of 32 keys per step
    constexpr int ND = D / 16;
    __shared__ ShortSmem<T, D> sm;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, g = lane >> 4, r16 = lane & 15;
    int hk, rest;
    deal(a.Hk, hk, rest);
    const int sp = rest % splits;
    int s, tile;
    if (!locate(a, rest / splits, short_max, 0, short_max, lane, s, tile)) return;
    const Seq q = seq_of(a, s);
    const int G = a.H / a.Hk, nrows = q.n * G;
    const int len = q.past + q.n, nd1 = (len - 1) >> 6;
    // the lane's row (those past the end repeat the last one)
    const int r = min(r16, nrows - 1);
    const int h = hk * G + r % G, pi = q.past + r / G;
    const int pp = page_of(a, s, pi >> 6);
    const double ci = pp < 0 ? 0.0 : gates_of(a, pp, h)[pi & 63];
    const double delta = head_delta(a, h);
    Block blk;
    blk.clear();
    blk.load_q(0, (const T*)a.q + (int64_t)(q.row0 + r / G) * a.qt + (int64_t)h * a.qh, g);

    // first page that any row keeps: rows 0 .. G - 1 are the first token's
    for (int k = wave; k < G; k += 4) {
        const double ck = readlane_f64(ci, k), dk = readlane_f64(delta, k);
        const int f = first_page(a, s, hk * G + k, q.past >> 6, ck, dk, lane);
        if (lane == 0) sm.first[k] = f;
    }
    if (threadIdx.x == 0) sm.marked = 0;
    for (int i = threadIdx.x; i < 16 * 2 * (D / 32); i += 256) (&sm.inf[0][0][0])[i] = 0;
    __syncthreads();
    int lo = sm.first[0];
    for (int k = 1; k < G; ++k) lo = min(lo, sm.first[k]);
    const int top = min(nd1, a.W - 1), pages = max(top - lo + 1, 0), per = (pages + splits - 1) / splits;
    const int nb = lo + sp * per, ne = min(nb + per - 1, top);
    if (nd1 >= a.W && r16 < nrows) report(a, s, h, lane & 48);

    const T* kp = (const T*)a.kp;
    const T* vp = (const T*)a.vp;
    // What a step needs, requested one step ahead (bf16) or at its start (float)
    typename Block::Frag kf[KH][2][Block::NK];
    double cj[KH][8], cend = 0.0;
    float vf[is_bf16<T>() ? 1 : ND][8];
    int page = -1;
    TileDma<D, 1> dma;
    if constexpr (is_bf16<T>()) dma.init(0, lane);
    PageWindow win;

    auto load = [&](int n, int hf, int buf) __attribute__((always_inline)) {
        const int p = win.get(a, s, n, lane);
        page = p;
        const int64_t at = ((int64_t)max(p, 0) * a.Hk + hk) * 64 * D;
        const double* cp = gates_of(a, max(p, 0), h);
#pragma unroll
        for (int ks = 0; ks < KH; ++ks) {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int i = 0; i < Block::NK; ++i)
                    kf[ks][kk][i] = *reinterpret_cast<const typename Block::Frag*>(
                        kp + at + (int64_t)(32 * (ks + hf) + key_row<T>(kk, r16)) * D +
                        4 * Block::kFrag * i + Block::kFrag * g);
#pragma unroll
            for (int j = 0; j < 8; ++j) cj[ks][j] = cp[32 * (ks + hf) + key_of<T>(g, j)];
        }
        cend = cp[63];
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

    // wave w takes steps w, w + 4, .. of the part's pages (or half pages)
    const int steps = nb <= ne ? (ne - nb + 1) * (is_bf16<T>() ? 1 : 2) : 0;
    auto page_at = [&](int u) { return nb + (is_bf16<T>() ? u : u >> 1); };
    if (wave < steps) {
        win.fill(a, s, nb, lane);
        load(page_at(wave), is_bf16<T>() ? 0 : wave & 1, 0);
    }
    int buf = 0;
    for (int u = wave; u < steps; u += 4, buf ^= 1) {
        const int n = page_at(u), hf = is_bf16<T>() ? 0 : u & 1;
        if constexpr (is_bf16<T>()) wait_vmcnt0();
        // this step's operands; the next step's are requested before they are used
        typename Block::Frag kc[KH][2][Block::NK];
        double cc[KH][8];
        float vc[is_bf16<T>() ? 1 : ND][8];
        const double end = cend;
        const int pg = page;
#pragma unroll
        for (int ks = 0; ks < KH; ++ks) {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int i = 0; i < Block::NK; ++i) kc[ks][kk][i] = kf[ks][kk][i];
#pragma unroll
            for (int j = 0; j < 8; ++j) cc[ks][j] = cj[ks][j];
        }
        if constexpr (!is_bf16<T>()) {
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int j = 0; j < 8; ++j) vc[dt][j] = vf[dt][j];
        }
        if (u + 4 < steps) load(page_at(u + 4), is_bf16<T>() ? 0 : u & 1, buf ^ 1);
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
            f32x4 x[2][1];
            const float zero[1] = {0.f};
            blk.scores(x, zero, [&](int kk, int i) __attribute__((always_inline)) { return kc[ks][kk][i]; });
            float p[1][8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int key = 32 * (ks + hf) + key_of<T>(g, j);
                const bool on = keep && 64 * n + key <= pi;
                const float y = __builtin_fmaf(x[j >> 2][0][j & 3], kscale,
                                               __builtin_fmaf((float)(ci - cc[ks][j]), kLog2e, -blk.ref[0]));
                p[0][j] = on ? y : -INFINITY;
            }
            blk.weights(0, p[0]);
            blk.add(p, [&](int dt, int j) __attribute__((always_inline)) {
                if constexpr (is_bf16<T>()) return tile_col8(sm.v[wave][buf], 32 * ks + 8 * g, 16 * dt, r16);
                else return vc[dt][j];
            });
        }
        if (bad) {
            sm.marked = 1;
            if (keep && r16 < nrows)
                mark_bad<T, D>(bad, vp + ((int64_t)pg * a.Hk + hk) * 64 * D, 64 * n, pi, lane, sm.inf[r16]);
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
    // [wave][dt][lane]; the first three waves' tiles are no longer read
    __shared__ f32x4 o_s[3][ND][64];
    if (wave > 0)
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) o_s[wave - 1][dt][lane] = blk.acc[0][dt] * scale;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) {
        f32x4 o = blk.acc[0][dt] * scale;
#pragma unroll
        for (int w = 0; w < 3; ++w) o += o_s[w][dt][lane];
        blk.acc[0][dt] = o;
    }
    if (sm.marked) add_marks<D>(blk.acc[0], sm.inf[r16], g);
    if (r16 < nrows) put_row<T, D>(a, q.row0 + r / G, h, sp, splits, stride, blk.acc[0], M, L, g);
}

// ---- merge -----------------------------------------------------------------------------
// One wave per row: lane p takes part p's maximum and sum, then features lane, lane + 64.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedArgs a, int split_long, int split_short,
                                                         int stride, int short_max, bool long_on) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (row >= (int64_t)a.T * a.H) return;
    const int t = (int)(row / a.H);
    int lo = 0, hi = a.N;                              // first s with cu[s + 1] > t
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.cu[mid + 1] > t) hi = mid;
        else lo = mid + 1;
    }
    if (lo >= a.N) return;
    const Seq q = seq_of(a, lo);
    if (t < q.row0 || t >= q.row0 + q.n) return;
    const bool is_short = q.n <= short_max;
    if (!is_short && !long_on) return;
    const int splits = is_short ? split_short : split_long;
    if (splits == 1) return;                            // written already
    const float2* ml = reinterpret_cast<const float2*>(a.part) + row * stride;
    const float* po = a.part + 2 * (int64_t)a.T * a.H * stride + row * stride * D;
    float2 v = make_float2(-INFINITY, 0.f);
    if (lane < splits) v = ml[lane];
    float M = v.x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) M = fmaxf(M, __shfl_xor(M, o));
    const float ref = M == -INFINITY ? 0.f : M;
    const float w = fast_exp2(v.x - ref);
    float L = v.y * w;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) L += __shfl_xor(L, o);
    float o0 = 0.f, o1 = 0.f;
    for (int p = 0; p < splits; ++p) {
        const float wp = __shfl(w, p);
        if (__shfl(v.y, p) == 0.f) continue;            // (no key: its sums are not there)
        o0 = __builtin_fmaf(wp, po[(int64_t)p * D + lane], o0);
        if (D == 128) o1 = __builtin_fmaf(wp, po[(int64_t)p * D + 64 + lane], o1);
    }
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    ((T*)a.O)[row * D + lane] = from_f32<T>(o0 * inv);
    if (D == 128) ((T*)a.O)[row * D + 64 + lane] = from_f32<T>(o1 * inv);
    if (lane == 0) a.lse[row] = L == 0.f ? -INFINITY : (M + fast_log2(L)) * kLn2;
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
// the others to the long one.
struct Division {
    int short_max, nq;
    bool short_on, long_on;
    int tiles_short, tiles_long, split_short, split_long, stride;
};

// Parts of the keys: until `wgs` workgroups fill the chip three times, no part under `least`
// pages of the longest sequence
int parts(int64_t wgs, int64_t pages, int least) {
    if (wgs <= 0) return 1;
    int64_t p = (768 + wgs - 1) / wgs;
    const int64_t most = pages / least;
    if (p > most) p = most;
    if (p > kMaxSplit) p = kMaxSplit;
    return p < 1 ? 1 : (int)p;
}

Division divide(const PagedArgs& a) {
    Division v{};
    const int G = a.H / a.Hk;
    v.short_max = kShortRows / G;
    const int64_t pages = (a.max_len + 63) / 64;
    v.long_on = a.max_new > v.short_max;
    // (rows in equal parts that are long: no sequence is short)
    v.short_on = !v.long_on || (int64_t)a.N * a.max_new != a.T;
    v.nq = a.max_new > 64 ? 2 : 1;
    const int rows = 64 * v.nq;
    // (no more tiles than this, however T rows are dealt to N sequences)
    if (v.long_on) v.tiles_long = (int)((a.T + (int64_t)a.N * (rows - 1)) / rows);
    v.tiles_short = v.short_on ? a.N : 0;
    v.split_long = v.long_on ? parts((int64_t)v.tiles_long * a.H, pages, 4) : 1;
    v.split_short = v.short_on ? parts((int64_t)v.tiles_short * a.Hk, pages, 8) : 1;
    v.stride = v.split_long > v.split_short ? v.split_long : v.split_short;
    return v;
}

template <typename T, int D>
void attend(const PagedArgs& a, const Division& v, hipStream_t s) {
    const float kscale = kLog2e / sqrtf((float)D);
    if (v.long_on) {
        const dim3 grid(dealt((int64_t)v.tiles_long * v.split_long, a.H));
        const int sm = v.short_on ? v.short_max : 0;
        if (v.nq == 2)
            hipLaunchKernelGGL((paged_long_kernel<T, D, 2>), grid, dim3(256), 0, s, a, v.tiles_long,
                               v.split_long, v.stride, sm, kscale);
        else
            hipLaunchKernelGGL((paged_long_kernel<T, D, 1>), grid, dim3(256), 0, s, a, v.tiles_long,
                               v.split_long, v.stride, sm, kscale);
    }
    if (v.short_on)
        hipLaunchKernelGGL((paged_short_kernel<T, D>),
                           dim3(dealt((int64_t)v.tiles_short * v.split_short, a.Hk)), dim3(256), 0,
                           s, a, v.split_short, v.stride, v.short_max, kscale);
    if (v.stride > 1)
        hipLaunchKernelGGL((paged_join_kernel<T, D>), dim3((unsigned)(((int64_t)a.T * a.H + 3) / 4)), dim3(256),
                           0, s, a, v.split_long, v.split_short, v.stride, v.short_on ? v.short_max : 0,
                           v.long_on);
}

}  // namespace

size_t paged_workspace(const PagedArgs& a) {
    const Division v = divide(a);
    return v.stride == 1 ? 0 : (size_t)a.T * a.H * v.stride * (a.d + 2) * sizeof(float);
}

hipError_t launch_paged_attend(const PagedArgs& a, hipStream_t s) {
    trace_begin(ACP_K_COUNT + ACP_OP_ATTEND, s);
    const Division v = divide(a);
    if (a.flags)
        hipLaunchKernelGGL(paged_flags_kernel, dim3((unsigned)(((int64_t)a.N * a.H + 255) / 256)), dim3(256), 0,
                           s, a, v.long_on ? 0x7fffffff : v.short_max);
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
