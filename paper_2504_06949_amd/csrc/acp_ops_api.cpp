// Entry points of acp_ops.h: argument checks, layouts and launches.
#include "acp_ops.h"

#include <cmath>

#include "acp_ops_internal.h"

namespace {

using acp::set_error;

acp_status ok() { return set_error(ACP_OK, ""); }

acp_status hip_status(hipError_t e, const char* what) {
    return e == hipSuccess ? ok() : set_error(ACP_EHIP, "%s: %s", what, hipGetErrorString(e));
}

#define ACP_TRY(expr)                      \
    do {                                   \
        const acp_status s_ = (expr);      \
        if (s_ != ACP_OK) return s_;       \
    } while (0)

acp_status check_dt(acp_dtype dt, const char* name) {
    if (dt != ACP_F32 && dt != ACP_BF16) return set_error(ACP_EINVAL, "unknown %s %d", name, (int)dt);
    return ACP_OK;
}

size_t size_of(acp_dtype dt) { return dt == ACP_BF16 ? 2 : 4; }

acp_status check_ptr(const void* p, const char* name, size_t align) {
    if (p == nullptr) return set_error(ACP_EINVAL, "%s is NULL", name);
    if (((uintptr_t)p & (align - 1)) != 0)
        return set_error(ACP_EINVAL, "%s is not %zu-byte aligned", name, align);
    return ACP_OK;
}

// Strides of a [B, H, L, n] tensor, contiguous ones if none are given
acp_status get_strides(const int64_t* s, int H, int L, int n, const char* name, acp::Strides* out) {
    if (s == nullptr) {
        *out = {(int64_t)H * L * n, (int64_t)L * n, (int64_t)n};
        return ACP_OK;
    }
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0) return set_error(ACP_EINVAL, "%s has a negative stride", name);
    *out = {s[0], s[1], s[2]};
    return ACP_OK;
}

acp_status check_rows(int B, int H, int L, int n) {
    if (B < 0 || H < 0 || L < 0 || n <= 0)
        return set_error(ACP_EINVAL, "bad sizes (B=%d H=%d L=%d n=%d)", B, H, L, n);
    if (n > 16384) return set_error(ACP_EUNSUPPORTED, "n=%d exceeds 16384", n);
    const double rows = (double)B * H * L;
    if (rows > 1073741824.0) return set_error(ACP_EUNSUPPORTED, "B*H*L=%.0f exceeds 2^30", rows);
    if (H > 65535) return set_error(ACP_EUNSUPPORTED, "H=%d exceeds 65535", H);
    return ACP_OK;
}

bool overlap_free_in_place(const void* x, const void* y, const acp::Strides& a, const acp::Strides& b) {
    return x != y || (a.b == b.b && a.h == b.h && a.l == b.l);
}

acp_status check_paged(int P, int H, int Hk, int d, acp_dtype dt) {
    ACP_TRY(check_dt(dt, "dtype"));
    if (P <= 0 || H <= 0 || Hk <= 0 || d <= 0)
        return set_error(ACP_EINVAL, "sizes must be positive (P=%d H=%d Hk=%d d=%d)", P, H, Hk, d);
    if (d != 64 && d != 128) return set_error(ACP_EUNSUPPORTED, "head dim %d not in {64, 128}", d);
    if (H > 65535 || H % Hk != 0 || H / Hk > 16)
        return set_error(ACP_EUNSUPPORTED, "H=%d is not 1 to 16 times Hk=%d (H at most 65535)", H, Hk);
    return ACP_OK;
}

acp_paged_layout paged_layout(int P, int H, int Hk, int d, acp_dtype dt) {
    const size_t kv = (size_t)P * Hk * 64 * d * size_of(dt);    // a multiple of 256
    acp_paged_layout y{};
    y.v = kv;
    y.c = 2 * kv;
    y.total = y.c + (size_t)P * H * 64 * 8;
    return y;
}

// (bounds under which no launch of the paged operators has 2^32 threads)
acp_status check_sequences(int T, int N, int H) {
    if (T < 0 || N < 0) return set_error(ACP_EINVAL, "bad sizes (T=%d N=%d)", T, N);
    if (N > 65535) return set_error(ACP_EUNSUPPORTED, "N=%d exceeds 65535", N);
    if ((int64_t)T * H > 1 << 26 || (int64_t)N * H > 1 << 22)
        return set_error(ACP_EUNSUPPORTED, "T*H=%lld exceeds 2^26 or N*H=%lld exceeds 2^22", (long long)T * H,
                         (long long)N * H);
    return ACP_OK;
}

acp_status check_call(int T, int N, int W, int H, const void* cu, const void* past, const void* table) {
    if (W < 0) return set_error(ACP_EINVAL, "bad size W=%d", W);
    ACP_TRY(check_sequences(T, N, H));
    ACP_TRY(check_ptr(cu, "cu", 4));
    if (N > 0) ACP_TRY(check_ptr(past, "past", 4));
    if (N > 0 && W > 0) ACP_TRY(check_ptr(table, "table", 4));
    return ACP_OK;
}

// Strides {token, head} of a packed [T, heads, d] tensor of 16-byte aligned rows
acp_status get_packed(const int64_t* s, int heads, int d, acp_dtype dt, const char* name, int64_t* t, int64_t* h) {
    *t = (int64_t)heads * d;
    *h = d;
    if (s == nullptr) return ACP_OK;
    const int64_t vec = 16 / (int64_t)size_of(dt);
    if (s[0] < 0 || s[1] < 0 || s[0] % vec || s[1] % vec)
        return set_error(ACP_EINVAL, "%s: strides must be multiples of 16 bytes and not negative", name);
    *t = s[0];
    *h = s[1];
    return ACP_OK;
}

acp_status check_cache(const void* cache, size_t bytes, const acp_paged_layout& y) {
    ACP_TRY(check_ptr(cache, "cache", 16));
    if (bytes < y.total) return set_error(ACP_EWORKSPACE, "cache of %zu bytes, %zu needed", bytes, y.total);
    return ACP_OK;
}

acp::PagedArgs paged_args(acp_dtype dt, int T, int N, int W, int P, int H, int Hk, int d, const int32_t* cu,
                          const int32_t* past, const int32_t* table, void* cache, int32_t* flags) {
    acp::PagedArgs a{};
    const acp_paged_layout y = paged_layout(P, H, Hk, d, dt);
    a.bf16 = dt == ACP_BF16;
    a.T = T; a.N = N; a.W = W; a.P = P; a.H = H; a.Hk = Hk; a.d = d;
    a.cu = cu; a.past = past; a.table = table; a.flags = flags;
    a.kp = (char*)cache + y.k;
    a.vp = (char*)cache + y.v;
    a.cp = (double*)((char*)cache + y.c);
    return a;
}

acp_status check_division(int max_new, int64_t max_len) {
    if (max_new < 0 || max_len < 0 || max_len > ((int64_t)1 << 31))
        return set_error(ACP_EINVAL, "max_new=%d or max_len=%lld outside their range", max_new, (long long)max_len);
    return ACP_OK;
}

// fox_attn_paged; fill: and the rows that nothing attends for
acp_status attend_paged(bool fill, const void* q, const int64_t* q_strides, acp_dtype dt, int T, int N, int W, int P,
                        int H, int Hk, int d, const int32_t* cu, const int32_t* past, const int32_t* table,
                        const void* cache, size_t cache_bytes, const float* gamma_q, const float* gamma_k,
                        double eps, int64_t L_max, int max_new, int64_t max_len, void* O, float* lse,
                        int32_t* flags, void* ws, size_t ws_bytes, void* stream) {
    ACP_TRY(check_paged(P, H, Hk, d, dt));
    ACP_TRY(check_call(T, N, W, H, cu, past, table));
    ACP_TRY(check_cache(cache, cache_bytes, paged_layout(P, H, Hk, d, dt)));
    ACP_TRY(check_division(max_new, max_len));
    if (!std::isfinite(eps) || eps < 0.0 || eps >= 1.0) return set_error(ACP_EINVAL, "eps=%g outside [0, 1)", eps);
    if (eps > 0.0) {
        if (L_max < 1 || L_max > (INT64_C(1) << 31))
            return set_error(ACP_EINVAL, "L_max=%lld outside [1, 2^31]", (long long)L_max);
        ACP_TRY(check_ptr(gamma_q, "gamma_q", 4));
        ACP_TRY(check_ptr(gamma_k, "gamma_k", 4));
    }
    if (flags) ACP_TRY(check_ptr(flags, "flags", 4));
    acp::PagedArgs a = paged_args(dt, T, N, W, P, H, Hk, d, cu, past, table, const_cast<void*>(cache), flags);
    ACP_TRY(get_packed(q_strides, H, d, dt, "q", &a.qt, &a.qh));
    a.max_new = max_new; a.max_len = max_len;
    if (T > 0) {
        ACP_TRY(check_ptr(q, "q", 16));
        ACP_TRY(check_ptr(O, "O", 16));
        ACP_TRY(check_ptr(lse, "lse", 4));
        const size_t need = acp::paged_workspace(a);
        if (need > 0) {
            ACP_TRY(check_ptr(ws, "ws", 16));
            if (ws_bytes < need)
                return set_error(ACP_EWORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, need);
        }
    }
    if (N == 0 && !(fill && T > 0)) return ok();
    a.q = q;
    a.gamma_q = eps > 0.0 ? gamma_q : nullptr;
    a.gamma_k = eps > 0.0 ? gamma_k : nullptr;
    a.log_lmax_over_eps = eps == 0.0 ? INFINITY : std::log((double)L_max) - std::log(eps);
    a.fill = fill;
    a.O = O; a.lse = lse;
    a.part = (float*)ws;
    return hip_status(acp::launch_paged_attend(a, (hipStream_t)stream), "fox_attn_paged launch");
}

}  // namespace

extern "C" {

// ---- norms -------------------------------------------------------------------------------
acp_status acp_norm_fwd(const void* x, const int64_t* x_strides, const void* weight, const void* bias,
                        acp_dtype dt, acp_dtype wdt, int B, int H, int L, int n, int per_head, int center,
                        double eps, void* y, float* mean, float* rstd, void* stream) {
    ACP_TRY(check_dt(dt, "dtype"));
    ACP_TRY(check_dt(wdt, "weight dtype"));
    ACP_TRY(check_rows(B, H, L, n));
    if (!(eps >= 0.0) || !std::isfinite(eps)) return set_error(ACP_EINVAL, "eps=%g is negative or not finite", eps);
    acp::NormArgs a{};
    ACP_TRY(get_strides(x_strides, H, L, n, "x", &a.xs));
    if ((int64_t)B * H * L == 0) return ok();
    ACP_TRY(check_ptr(x, "x", size_of(dt)));
    ACP_TRY(check_ptr(weight, "weight", size_of(wdt)));
    if (bias) ACP_TRY(check_ptr(bias, "bias", size_of(wdt)));
    ACP_TRY(check_ptr(y, "y", size_of(dt)));
    if (x == y) return set_error(ACP_EINVAL, "y is x");
    if (rstd == nullptr && mean != nullptr) return set_error(ACP_EINVAL, "mean without rstd");
    if (rstd != nullptr && (mean != nullptr) != (center != 0))
        return set_error(ACP_EINVAL, "mean goes with center");
    a.x = x; a.weight = weight; a.bias = bias;
    a.bf16 = dt == ACP_BF16; a.wbf16 = wdt == ACP_BF16;
    a.B = B; a.H = H; a.L = L; a.n = n;
    a.per_head = per_head != 0; a.center = center != 0;
    a.eps = (float)eps;
    a.y = y; a.mean = mean; a.rstd = rstd;
    return hip_status(acp::launch_norm_fwd(a, (hipStream_t)stream), "acp_norm_fwd launch");
}

acp_status acp_norm_workspace_size(int B, int H, int L, int n, int per_head, size_t* bytes) {
    ACP_TRY(check_rows(B, H, L, n));
    if (bytes == nullptr) return set_error(ACP_EINVAL, "bytes is NULL");
    *bytes = H == 0 ? 0 : acp::norm_workspace(B, H, L, n, per_head != 0);
    return ok();
}

acp_status acp_norm_bwd(const void* dy, const int64_t* dy_strides, const void* x, const int64_t* x_strides,
                        const void* weight, acp_dtype dt, acp_dtype wdt, int B, int H, int L, int n,
                        int per_head, const float* mean, const float* rstd, void* dx,
                        const int64_t* dx_strides, float* dweight, float* dbias, void* ws, size_t ws_bytes,
                        void* stream) {
    ACP_TRY(check_dt(dt, "dtype"));
    ACP_TRY(check_dt(wdt, "weight dtype"));
    ACP_TRY(check_rows(B, H, L, n));
    acp::NormArgs a{};
    ACP_TRY(get_strides(dy_strides, H, L, n, "dy", &a.dys));
    ACP_TRY(get_strides(x_strides, H, L, n, "x", &a.xs));
    ACP_TRY(get_strides(dx_strides, H, L, n, "dx", &a.dxs));
    if (per_head && H == 0) return ok();            // no weight row, no row
    ACP_TRY(check_ptr(dweight, "dweight", 4));
    if (dbias) ACP_TRY(check_ptr(dbias, "dbias", 4));
    const bool rows = (int64_t)B * H * L > 0;
    if (rows) {
        ACP_TRY(check_ptr(dy, "dy", size_of(dt)));
        ACP_TRY(check_ptr(x, "x", size_of(dt)));
        ACP_TRY(check_ptr(weight, "weight", size_of(wdt)));
        ACP_TRY(check_ptr(rstd, "rstd", 4));
        ACP_TRY(check_ptr(dx, "dx", size_of(dt)));
        if (dx == x) return set_error(ACP_EINVAL, "dx is x");
        if (!overlap_free_in_place(dy, dx, a.dys, a.dxs))
            return set_error(ACP_EINVAL, "dx is dy with other strides");
        ACP_TRY(check_ptr(ws, "ws", 16));
        const size_t need = acp::norm_workspace(B, H, L, n, per_head != 0);
        if (ws_bytes < need) return set_error(ACP_EWORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, need);
    }
    a.dy = dy; a.x = x; a.weight = weight;
    a.bf16 = dt == ACP_BF16; a.wbf16 = wdt == ACP_BF16;
    a.B = B; a.H = H; a.L = L; a.n = n;
    a.per_head = per_head != 0; a.center = mean != nullptr;
    a.y = dx;
    a.mean = const_cast<float*>(mean);
    a.rstd = const_cast<float*>(rstd);
    a.dweight = dweight; a.dbias = dbias;
    a.part = (float*)ws;
    return hip_status(acp::launch_norm_bwd(a, (hipStream_t)stream), "acp_norm_bwd launch");
}

// ---- rotary positions ----------------------------------------------------------------------
acp_status acp_rotary_table(int rot, double base, int scaling, double factor, double train_len, double slow,
                            double fast, double* turns) {
    if (rot < 2 || rot % 2 != 0) return set_error(ACP_EINVAL, "rot=%d is not a positive even number", rot);
    if (!(base > 1.0) || !std::isfinite(base)) return set_error(ACP_EINVAL, "base=%g is not above 1", base);
    if (scaling < ACP_SCALE_NONE || scaling > ACP_SCALE_RAMP)
        return set_error(ACP_EINVAL, "unknown scaling %d", scaling);
    if (scaling != ACP_SCALE_NONE && (!(factor >= 1.0) || !std::isfinite(factor)))
        return set_error(ACP_EINVAL, "factor=%g is below 1 or not finite", factor);
    if (scaling == ACP_SCALE_BASE && rot < 4) return set_error(ACP_EINVAL, "a scaled base needs rot >= 4");
    if (scaling == ACP_SCALE_RAMP &&
        (!(train_len > 0.0) || !(slow >= 0.0) || !(fast > slow) || !std::isfinite(fast) || !std::isfinite(train_len)))
        return set_error(ACP_EINVAL, "the ramp needs train_len > 0 and fast > slow >= 0");
    if (turns == nullptr) return set_error(ACP_EINVAL, "turns is NULL");
    const double two_pi = 6.283185307179586476925286766559;
    if (scaling == ACP_SCALE_BASE) base *= std::pow(factor, (double)rot / (rot - 2));
    for (int i = 0; i < rot / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rot) / two_pi;
        if (scaling == ACP_SCALE_LINEAR) f /= factor;
        if (scaling == ACP_SCALE_RAMP) {
            const double r = train_len * f;
            double keep = (r - slow) / (fast - slow);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f = f * keep + f / factor * (1.0 - keep);
        }
        turns[i] = f;
    }
    return ok();
}

acp_status acp_rotary(const void* q, const int64_t* q_strides, const void* k, const int64_t* k_strides,
                      acp_dtype dt, int B, int H, int Hk, int L, int d, int rot, int layout, int inverse,
                      double amplitude, const double* turns, const void* positions, int pos_bytes,
                      const int64_t* pos_strides, int64_t start, void* q_out, const int64_t* q_out_strides,
                      void* k_out, const int64_t* k_out_strides, void* stream) {
    ACP_TRY(check_dt(dt, "dtype"));
    if (B < 0 || H < 0 || Hk < 0 || L < 0 || d <= 0)
        return set_error(ACP_EINVAL, "bad sizes (B=%d H=%d Hk=%d L=%d d=%d)", B, H, Hk, L, d);
    if (d % 2 != 0 || d > 1024) return set_error(ACP_EUNSUPPORTED, "d=%d is not even, up to 1024", d);
    if (rot < 2 || rot % 2 != 0 || rot > d) return set_error(ACP_EINVAL, "rot=%d is not even in [2, d=%d]", rot, d);
    if (layout != ACP_ROTARY_HALF && layout != ACP_ROTARY_INTERLEAVED)
        return set_error(ACP_EINVAL, "unknown layout %d", layout);
    if (!std::isfinite((float)amplitude)) return set_error(ACP_EINVAL, "amplitude is not finite");
    // (threads of a launch: fewer than d / 8 + 2 chunks per position)
    if ((double)B * L * (d / 8 + 2) >= 4294967296.0 || H + (int64_t)Hk > 65535)
        return set_error(ACP_EUNSUPPORTED, "B*L*(d/8 + 2) reaches 2^32 or H + Hk exceeds 65535");
    if ((int64_t)B * L == 0 || H + Hk == 0) return ok();
    if (q == nullptr && k == nullptr) return set_error(ACP_EINVAL, "q and k are NULL");
    acp::RotaryArgs a{};
    const void* in[2] = {q, k};
    void* out[2] = {q_out, k_out};
    const int64_t* is[2] = {q_strides, k_strides};
    const int64_t* os[2] = {q_out_strides, k_out_strides};
    const char* names[2][2] = {{"q", "q_out"}, {"k", "k_out"}};
    int heads = 0;
    for (int w = 0; w < 2; ++w) {
        if (in[w] == nullptr) continue;
        const int n = w ? Hk : H;
        ACP_TRY(get_strides(is[w], n, L, d, names[w][0], &a.xs[w]));
        ACP_TRY(get_strides(os[w], n, L, d, names[w][1], &a.ys[w]));
        ACP_TRY(check_ptr(in[w], names[w][0], size_of(dt)));
        ACP_TRY(check_ptr(out[w], names[w][1], size_of(dt)));
        if (!overlap_free_in_place(in[w], out[w], a.xs[w], a.ys[w]))
            return set_error(ACP_EINVAL, "%s is its input with other strides", names[w][1]);
        a.x[w] = in[w]; a.y[w] = out[w]; a.heads[w] = n;
        heads += n;
    }
    if (q && k && q_out == k_out && H > 0 && Hk > 0) return set_error(ACP_EINVAL, "k_out is q_out");
    ACP_TRY(check_ptr(turns, "turns", 8));
    if (positions) {
        if (pos_bytes != 4 && pos_bytes != 8) return set_error(ACP_EINVAL, "pos_bytes=%d is not 4 or 8", pos_bytes);
        ACP_TRY(check_ptr(positions, "positions", (size_t)pos_bytes));
        if (pos_strides == nullptr) return set_error(ACP_EINVAL, "pos_strides is NULL");
        if (pos_strides[0] < 0 || pos_strides[1] < 0) return set_error(ACP_EINVAL, "positions has a negative stride");
        a.pos_b = pos_strides[0]; a.pos_l = pos_strides[1];
    } else if (start <= -(INT64_C(1) << 31) || start > (INT64_C(1) << 31) - L) {
        return set_error(ACP_EINVAL, "start=%lld outside (-2^31, 2^31 - L]", (long long)start);
    }
    if (heads == 0) return ok();
    a.bf16 = dt == ACP_BF16;
    a.B = B; a.L = L; a.d = d; a.rot = rot;
    a.interleaved = layout == ACP_ROTARY_INTERLEAVED; a.inverse = inverse != 0;
    a.amplitude = (float)amplitude;
    a.turns = turns;
    a.pos = positions; a.pos_bytes = pos_bytes; a.start = start;
    return hip_status(acp::launch_rotary(a, (hipStream_t)stream), "acp_rotary launch");
}

// ---- paged cache -----------------------------------------------------------------------------
acp_status acp_paged_cache_size(int P, int H, int Hk, int d, acp_dtype dt, size_t* bytes) {
    ACP_TRY(check_paged(P, H, Hk, d, dt));
    if (bytes == nullptr) return set_error(ACP_EINVAL, "bytes is NULL");
    *bytes = paged_layout(P, H, Hk, d, dt).total;
    return ok();
}

acp_status acp_paged_offsets(int P, int H, int Hk, int d, acp_dtype dt, acp_paged_layout* out) {
    ACP_TRY(check_paged(P, H, Hk, d, dt));
    if (out == nullptr) return set_error(ACP_EINVAL, "out is NULL");
    *out = paged_layout(P, H, Hk, d, dt);
    return ok();
}

acp_status acp_paged_append(const void* k, const int64_t* k_strides, const void* v, const int64_t* v_strides,
                            const float* log_f, const int64_t* f_strides, acp_dtype dt, int T, int N, int W,
                            int P, int H, int Hk, int d, const int32_t* cu, const int32_t* past,
                            const int32_t* table, void* cache, size_t cache_bytes, int32_t* flags,
                            void* stream) {
    ACP_TRY(check_paged(P, H, Hk, d, dt));
    ACP_TRY(check_call(T, N, W, H, cu, past, table));
    ACP_TRY(check_cache(cache, cache_bytes, paged_layout(P, H, Hk, d, dt)));
    if (flags) ACP_TRY(check_ptr(flags, "flags", 4));
    acp::PagedArgs a = paged_args(dt, T, N, W, P, H, Hk, d, cu, past, table, cache, flags);
    ACP_TRY(get_packed(k_strides, Hk, d, dt, "k", &a.kt, &a.kh));
    ACP_TRY(get_packed(v_strides, Hk, d, dt, "v", &a.vt, &a.vh));
    a.ft = H;
    a.fh = 1;
    if (f_strides) {
        if (f_strides[0] < 0 || f_strides[1] < 0) return set_error(ACP_EINVAL, "log_f has a negative stride");
        a.ft = f_strides[0];
        a.fh = f_strides[1];
    }
    if (T > 0) {
        ACP_TRY(check_ptr(k, "k", 16));
        ACP_TRY(check_ptr(v, "v", 16));
        ACP_TRY(check_ptr(log_f, "log_f", 4));
    }
    if (N == 0) return ok();
    a.k = k; a.v = v; a.log_f = log_f;
    return hip_status(acp::launch_paged_append(a, (hipStream_t)stream), "acp_paged_append launch");
}

acp_status acp_paged_workspace_size(int T, int N, int H, int Hk, int d, acp_dtype dt, int max_new,
                                    int64_t max_len, size_t* bytes) {
    ACP_TRY(check_paged(1, H, Hk, d, dt));
    ACP_TRY(check_sequences(T, N, H));
    ACP_TRY(check_division(max_new, max_len));
    if (bytes == nullptr) return set_error(ACP_EINVAL, "bytes is NULL");
    acp::PagedArgs a{};
    a.bf16 = dt == ACP_BF16;
    a.T = T; a.N = N; a.H = H; a.Hk = Hk; a.d = d;
    a.max_new = max_new; a.max_len = max_len;
    *bytes = acp::paged_workspace(a);
    return ok();
}

acp_status fox_attn_paged(const void* q, const int64_t* q_strides, acp_dtype dt, int T, int N, int W, int P,
                          int H, int Hk, int d, const int32_t* cu, const int32_t* past, const int32_t* table,
                          const void* cache, size_t cache_bytes, const float* gamma_q, const float* gamma_k,
                          double eps, int64_t L_max, int max_new, int64_t max_len, void* O, float* lse,
                          int32_t* flags, void* ws, size_t ws_bytes, void* stream) {
    return attend_paged(false, q, q_strides, dt, T, N, W, P, H, Hk, d, cu, past, table, cache, cache_bytes, gamma_q,
                        gamma_k, eps, L_max, max_new, max_len, O, lse, flags, ws, ws_bytes, stream);
}

acp_status fox_attn_paged_filled(const void* q, const int64_t* q_strides, acp_dtype dt, int T, int N, int W,
                                 int P, int H, int Hk, int d, const int32_t* cu, const int32_t* past,
                                 const int32_t* table, const void* cache, size_t cache_bytes,
                                 const float* gamma_q, const float* gamma_k, double eps, int64_t L_max,
                                 int max_new, int64_t max_len, void* O, float* lse, int32_t* flags, void* ws,
                                 size_t ws_bytes, void* stream) {
    return attend_paged(true, q, q_strides, dt, T, N, W, P, H, Hk, d, cu, past, table, cache, cache_bytes, gamma_q,
                        gamma_k, eps, L_max, max_new, max_len, O, lse, flags, ws, ws_bytes, stream);
}

}  // extern "C"
