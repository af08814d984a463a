// The C boundary of include/tagore_embed.h and include/tagore_learn.h: argument checks and workspaces.  Host code only; the device's steps are the launchers of
// tg_embed.h.
#include "../../include/tagore_embed.h"
#include "../../include/tagore_learn.h"
#include "tg_embed.h"
#include "tg_error.h"

#include <algorithm>
#include <new>

#define TG_MAX_COUNT (1ll << 30)
#define TG_MAX_LOOKUP_D 65536
#define TG_MAX_D 8192
#define TG_MAX_TOKENS (1ll << 28)  // of a softmax: its gradient runs along them, in bytes of 32 bits
#define TG_MAX_K 65536
#define TG_MAX_BEST 32                // rows of a token
#define TG_MAX_TENSORS (1 << 20)
#define TG_MAX_VALUES (1ll << 40)
#define TG_MAX_PITCH (1 << 20)       // bytes between rows that are read where they are

static hipStream_t stream_of(void* s) { return reinterpret_cast<hipStream_t>(s); }
static int launched(const char* what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TG_OK : tg_fail(TG_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

static int check_dtype(int32_t dtype)
{
    return dtype >= TG_DTYPE_F32 && dtype <= TG_DTYPE_F16 ? TG_OK : tg_fail(TG_ERR_INVALID_ARG, "unknown dtype %d", dtype);
}
// a count of rows, none among them where `least` is 0
static int check_count(const char* name, int64_t n, int64_t least)
{
    if (n < least || n >= TG_MAX_COUNT) return tg_fail(TG_ERR_INVALID_ARG, "%s = %lld outside %lld..2^30-1", name, (long long)n, (long long)least);
    return TG_OK;
}
static int check_length(const char* name, int32_t d, int32_t most)
{
    return d >= 1 && d <= most ? TG_OK : tg_fail(TG_ERR_INVALID_ARG, "%s = %d outside 1..%d", name, d, most);
}
static int check_ld(const char* name, int64_t ld, int32_t d)
{
    if (ld < d || ld >= (1ll << 40)) return tg_fail(TG_ERR_INVALID_ARG, "%s = %lld below the row length %d", name, (long long)ld, d);
    return TG_OK;
}
static int check_flag(const char* name, int32_t f)
{
    return f == 0 || f == 1 ? TG_OK : tg_fail(TG_ERR_INVALID_ARG, "%s = %d must be 0 or 1", name, f);
}
static int check_space(const void* ws, size_t have, size_t need)
{
    if (need == 0) return TG_OK;
    if (!ws) return tg_fail(TG_ERR_INVALID_ARG, "workspace is NULL");
    if ((uintptr_t)ws & 255) return tg_fail(TG_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (have < need) return tg_fail(TG_ERR_INVALID_ARG, "workspace too small: %zu bytes given, %zu needed", have, need);
    return TG_OK;
}
static int null_argument() { return tg_fail(TG_ERR_INVALID_ARG, "NULL argument"); }
#define CHECK(expr)                      \
    do {                                 \
        const int rc_ = (expr);          \
        if (rc_ != TG_OK) return rc_;    \
    } while (0)

extern "C" int tg_embed_lookup(const void* table, int64_t ld, int32_t dtype, int64_t n_rows, int32_t d, const void* ids, int32_t ids64,
                               int64_t n, float scale, void* out, void* stream)
{
    CHECK(check_dtype(dtype));
    CHECK(check_count("n", n, 0));
    CHECK(check_count("n_rows", n_rows, 1));
    CHECK(check_length("d", d, TG_MAX_LOOKUP_D));
    CHECK(check_ld("ld", ld, d));
    CHECK(check_flag("ids64", ids64));
    if (n == 0) return TG_OK;
    if (!table || !ids || !out) return null_argument();
    tg_launch_lookup(table, ld, dtype, n_rows, d, ids, ids64, n, scale, out, stream_of(stream));
    return launched("lookup");
}

extern "C" size_t tg_embed_lookup_grad_workspace(int64_t n, int64_t n_rows, int32_t d)
{
    if (check_count("n", n, 0) != TG_OK || check_count("n_rows", n_rows, 1) != TG_OK || check_length("d", d, TG_MAX_LOOKUP_D) != TG_OK) return 0;
    return tg_lookup_grad_space(n, n_rows, d);
}
extern "C" int tg_embed_lookup_grad(const void* grad, int64_t ld, int32_t dtype, const void* ids, int32_t ids64, int64_t n, int64_t n_rows,
                                    int32_t d, float scale, int32_t accumulate, void* out, int32_t out_dtype, void* workspace,
                                    size_t workspace_bytes, void* stream)
{
    CHECK(check_dtype(dtype));
    CHECK(check_count("n", n, 0));
    CHECK(check_count("n_rows", n_rows, 1));
    CHECK(check_length("d", d, TG_MAX_LOOKUP_D));
    CHECK(check_ld("ld", ld, d));
    CHECK(check_flag("ids64", ids64));
    CHECK(check_flag("accumulate", accumulate));
    if (out_dtype != TG_DTYPE_F32 && out_dtype != dtype) return tg_fail(TG_ERR_INVALID_ARG, "out_dtype = %d must be fp32 or the gradient's", out_dtype);
    if (!out || (n > 0 && (!grad || !ids))) return null_argument();
    CHECK(check_space(workspace, workspace_bytes, tg_lookup_grad_space(n, n_rows, d)));
    tg_launch_lookup_grad(grad, ld, dtype, ids, ids64, n, n_rows, d, scale, accumulate, out, out_dtype, workspace, stream_of(stream));
    return launched("gradient of the lookup");
}

static int check_norm(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, int32_t dtype, int64_t n, int32_t d)
{
    CHECK(check_dtype(dtype));
    CHECK(check_count("n", n, 0));
    CHECK(check_length("d", d, TG_MAX_D));
    CHECK(check_ld("ld_x", ld_x, d));
    if (residual) CHECK(check_ld("ld_residual", ld_residual, d));
    return n > 0 && !x ? null_argument() : TG_OK;
}
// out_r in place of x or the residual: its rows are d apart, so theirs have to be
static int check_in_place(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, const void* out_r, int64_t n, int32_t d)
{
    if (!residual || n < 2 || !((out_r == x && ld_x != d) || (out_r == residual && ld_residual != d))) return TG_OK;
    return tg_fail(TG_ERR_INVALID_ARG, "out_r is an input whose rows are not back to back");
}
static int check_eps(float eps)
{
    return eps >= 0.0f && eps <= 3.4028234e38f ? TG_OK : tg_fail(TG_ERR_INVALID_ARG, "eps must be finite and not below 0");
}

extern "C" int tg_add_rms_norm(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, const void* weight, int32_t dtype,
                               int64_t n, int32_t d, float eps, void* out_y, void* out_r, float* out_rstd, void* stream)
{
    CHECK(check_norm(x, ld_x, residual, ld_residual, dtype, n, d));
    CHECK(check_eps(eps));
    if (n == 0) return TG_OK;
    if (!weight || !out_y || (residual && !out_r)) return null_argument();
    CHECK(check_in_place(x, ld_x, residual, ld_residual, out_r, n, d));
    tg_launch_norm(x, ld_x, residual, ld_residual, weight, dtype, n, d, eps, out_y, out_r, out_rstd, stream_of(stream));
    return launched("norm");
}

extern "C" size_t tg_add_rms_norm_grad_workspace(int64_t n, int32_t d)
{
    if (check_count("n", n, 0) != TG_OK || check_length("d", d, TG_MAX_D) != TG_OK) return 0;
    return tg_norm_grad_space(n, d);
}
extern "C" int tg_add_rms_norm_grad(const void* dy, int64_t ld_dy, const void* dr, int64_t ld_dr, const void* r, int64_t ld_r,
                                    const void* weight, const float* rstd, int32_t dtype, int64_t n, int32_t d, void* out_dx,
                                    void* out_dweight, void* workspace, size_t workspace_bytes, void* stream)
{
    CHECK(check_norm(dy, ld_dy, dr, ld_dr, dtype, n, d));
    CHECK(check_ld("ld_r", ld_r, d));
    if (!weight || !out_dweight || (n > 0 && (!r || !rstd || !out_dx))) return null_argument();
    CHECK(check_space(workspace, workspace_bytes, tg_norm_grad_space(n, d)));
    tg_launch_norm_grad(dy, ld_dy, dr, ld_dr, r, ld_r, weight, rstd, dtype, n, d, out_dx, out_dweight, workspace, stream_of(stream));
    return launched("gradient of the norm");
}

extern "C" int tg_add_rms_norm_q8(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, const void* weight, int32_t dtype,
                                  int64_t n, int32_t d, float eps, int8_t* out_q, float* out_scale, void* out_r, void* stream)
{
    CHECK(check_norm(x, ld_x, residual, ld_residual, dtype, n, d));
    CHECK(check_eps(eps));
    if (n == 0) return TG_OK;
    if (!weight || !out_q || !out_scale || (residual && !out_r)) return null_argument();
    CHECK(check_in_place(x, ld_x, residual, ld_residual, out_r, n, d));
    tg_launch_norm_q8(x, ld_x, residual, ld_residual, weight, dtype, n, d, eps, out_q, out_scale, out_r, stream_of(stream));
    return launched("norm to 8 bits");
}
extern "C" int tg_quantize_rows(const void* x, int64_t ld_x, int32_t dtype, int64_t n, int32_t d, int8_t* out_q, float* out_scale, void* stream)
{
    CHECK(check_norm(x, ld_x, nullptr, 0, dtype, n, d));
    if (n == 0) return TG_OK;
    if (!out_q || !out_scale) return null_argument();
    tg_launch_norm_q8(x, ld_x, nullptr, 0, nullptr, dtype, n, d, 0.0f, out_q, out_scale, nullptr, stream_of(stream));
    return launched("rows to 8 bits");
}
extern "C" int tg_dequantize_rows(const int8_t* q, const float* scale, int64_t n, int32_t d, int32_t dtype, void* out, void* stream)
{
    CHECK(check_dtype(dtype));
    CHECK(check_count("n", n, 0));
    CHECK(check_length("d", d, TG_MAX_D));
    if (n == 0) return TG_OK;
    if (!q || !scale || !out) return null_argument();
    tg_launch_dequantize(q, scale, n, d, dtype, out, stream_of(stream));
    return launched("rows from 8 bits");
}

static int check_product(int64_t m, int64_t n, int32_t k)
{
    CHECK(check_count("m", m, 0));
    CHECK(check_count("n", n, 1));
    return check_length("k", k, TG_MAX_K);
}
extern "C" size_t tg_matmul_q8_workspace(int64_t m, int64_t n, int32_t k, int32_t aligned)
{
    return check_product(m, n, k) != TG_OK || check_flag("aligned", aligned) != TG_OK ? 0 : tg_product_space(m, n, k, aligned != 0);
}
extern "C" int tg_matmul_q8(const int8_t* a, const float* a_scale, const int8_t* b, const float* b_scale, const float* bias, int64_t m,
                            int64_t n, int32_t k, void* out, int32_t dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    CHECK(check_dtype(dtype));
    CHECK(check_product(m, n, k));
    if (m == 0) return TG_OK;
    if (!a || !a_scale || !b || !b_scale || !out) return null_argument();
    CHECK(check_space(workspace, workspace_bytes, tg_product_space(m, n, k, (((uintptr_t)a | (uintptr_t)b) & 15) == 0)));
    tg_launch_product(a, a_scale, b, b_scale, bias, m, n, k, out, dtype, workspace, stream_of(stream));
    return launched("8-bit product");
}

static int check_xent(int64_t n, int64_t n_rows, int32_t d, int32_t dtype)
{
    CHECK(check_dtype(dtype));
    CHECK(check_count("n", n, 0));
    CHECK(check_count("n_rows", n_rows, 1));
    if (n >= TG_MAX_TOKENS) return tg_fail(TG_ERR_INVALID_ARG, "n = %lld must be below 2^28", (long long)n);
    return check_length("d", d, TG_MAX_D);
}
static int check_aligned(int32_t aligned)
{
    return aligned >= 0 && aligned <= 3 ? TG_OK : tg_fail(TG_ERR_INVALID_ARG, "aligned = %d outside 0..3", aligned);
}
// which operand's rows begin at multiples of 16 bytes, as `aligned` says it (that their length is one is looked at where it is known, with the sizes)
static int rows_ready(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int32_t dtype)
{
    const int64_t e = (int64_t)tg_type_bytes(dtype);
    const auto ready = [&](const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && (ld * e & 15) == 0 && ld * e <= TG_MAX_PITCH; };
    return ready(w, ld_w) ? (ready(h, ld_h) ? 1 : 2) : ready(h, ld_h) ? 3 : 0;
}
extern "C" size_t tg_softmax_xent_workspace(int64_t n, int64_t n_rows, int32_t d, int32_t dtype, int32_t aligned)
{
    return check_xent(n, n_rows, d, dtype) != TG_OK || check_aligned(aligned) != TG_OK ? 0 : tg_xent_space(n, n_rows, d, dtype, aligned);
}
extern "C" int tg_softmax_xent(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int32_t dtype, int64_t n, int64_t n_rows, int32_t d,
                               const void* targets, int32_t targets64, float scale, float* out_loss, float* out_lse, void* workspace,
                               size_t workspace_bytes, void* stream)
{
    CHECK(check_xent(n, n_rows, d, dtype));
    CHECK(check_ld("ld_h", ld_h, d));
    CHECK(check_ld("ld_w", ld_w, d));
    CHECK(check_flag("targets64", targets64));
    if (n == 0) return TG_OK;
    if (!h || !w || !targets || !out_loss || !out_lse) return null_argument();
    CHECK(check_space(workspace, workspace_bytes, tg_xent_space(n, n_rows, d, dtype, rows_ready(h, ld_h, w, ld_w, dtype))));
    tg_launch_xent(h, ld_h, w, ld_w, dtype, n, n_rows, d, targets, targets64, scale, out_loss, out_lse, workspace, stream_of(stream));
    return launched("softmax cross entropy");
}
extern "C" size_t tg_softmax_xent_grad_workspace(int64_t n, int64_t n_rows, int32_t d, int32_t dtype, int32_t aligned)
{
    return check_xent(n, n_rows, d, dtype) != TG_OK || check_aligned(aligned) != TG_OK ? 0 : tg_xent_grad_space(n, n_rows, d, dtype, aligned, false, true);
}
extern "C" int tg_softmax_xent_grad(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int32_t dtype, int64_t n, int64_t n_rows, int32_t d,
                                    const void* targets, int32_t targets64, const float* lse, const float* dloss, float scale, void* out_dh,
                                    void* out_dw, void* workspace, size_t workspace_bytes, void* stream)
{
    CHECK(check_xent(n, n_rows, d, dtype));
    CHECK(check_ld("ld_h", ld_h, d));
    CHECK(check_ld("ld_w", ld_w, d));
    CHECK(check_flag("targets64", targets64));
    if (!out_dw || (n > 0 && (!h || !w || !targets || !lse || !dloss || !out_dh))) return null_argument();
    CHECK(check_space(workspace, workspace_bytes, tg_xent_grad_space(n, n_rows, d, dtype, rows_ready(h, ld_h, w, ld_w, dtype), true, true)));
    const XentTokens t{targets, targets64, lse, dloss, 1.0f, nullptr, nullptr};
    tg_launch_xent_grad(h, ld_h, w, ld_w, dtype, n, n_rows, d, t, scale, out_dh, out_dw, workspace, workspace_bytes, stream_of(stream));
    return launched("gradient of the softmax cross entropy");
}

static int check_best(int32_t top)
{
    return top >= 0 && top <= TG_MAX_BEST ? TG_OK : tg_fail(TG_ERR_INVALID_ARG, "top = %d outside 0..%d", top, TG_MAX_BEST);
}
extern "C" size_t tg_log_probs_workspace(int64_t n, int64_t n_rows, int32_t d, int32_t dtype, int32_t top, int32_t aligned)
{
    return check_xent(n, n_rows, d, dtype) != TG_OK || check_best(top) != TG_OK || check_aligned(aligned) != TG_OK ? 0
                                                                                                                  : tg_log_probs_space(n, n_rows, d, dtype, top, aligned);
}
extern "C" int tg_log_probs(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int32_t dtype, int64_t n, int64_t n_rows, int32_t d,
                            const void* targets, int32_t targets64, float scale, int32_t top, float* out_logp, float* out_entropy, float* out_lse,
                            int32_t* out_rows, float* out_row_logp, void* workspace, size_t workspace_bytes, void* stream)
{
    CHECK(check_xent(n, n_rows, d, dtype));
    CHECK(check_best(top));
    CHECK(check_ld("ld_h", ld_h, d));
    CHECK(check_ld("ld_w", ld_w, d));
    CHECK(check_flag("targets64", targets64));
    if (n == 0) return TG_OK;
    if (!h || !w || (targets && !out_logp) || !out_entropy || !out_lse || (top && (!out_rows || !out_row_logp))) return null_argument();
    CHECK(check_space(workspace, workspace_bytes, tg_log_probs_space(n, n_rows, d, dtype, top, rows_ready(h, ld_h, w, ld_w, dtype))));
    tg_launch_log_probs(h, ld_h, w, ld_w, dtype, n, n_rows, d, targets, targets64, scale, top, out_logp, out_entropy, out_lse, out_rows, out_row_logp,
                        workspace, stream_of(stream));
    return launched("log probabilities");
}
extern "C" size_t tg_log_probs_grad_workspace(int64_t n, int64_t n_rows, int32_t d, int32_t dtype, int32_t table, int32_t aligned)
{
    return check_xent(n, n_rows, d, dtype) != TG_OK || check_flag("table", table) != TG_OK || check_aligned(aligned) != TG_OK
               ? 0
               : tg_xent_grad_space(n, n_rows, d, dtype, aligned, false, table != 0);
}
extern "C" int tg_log_probs_grad(const void* h, int64_t ld_h, const void* w, int64_t ld_w, int32_t dtype, int64_t n, int64_t n_rows, int32_t d,
                                 const void* targets, int32_t targets64, const float* lse, const float* dlogp, const float* entropy,
                                 const float* dentropy, float scale, void* out_dh, void* out_dw, void* workspace, size_t workspace_bytes, void* stream)
{
    CHECK(check_xent(n, n_rows, d, dtype));
    CHECK(check_ld("ld_h", ld_h, d));
    CHECK(check_ld("ld_w", ld_w, d));
    CHECK(check_flag("targets64", targets64));
    if (n > 0 && (!h || !w || !targets || !lse || !dlogp || !out_dh || (dentropy && !entropy))) return null_argument();
    if (n == 0 && !out_dw) return TG_OK;
    CHECK(check_space(workspace, workspace_bytes, tg_xent_grad_space(n, n_rows, d, dtype, rows_ready(h, ld_h, w, ld_w, dtype), true, out_dw != nullptr)));
    const XentTokens t{targets, targets64, lse, dlogp, -1.0f, entropy, dentropy};
    tg_launch_xent_grad(h, ld_h, w, ld_w, dtype, n, n_rows, d, t, scale, out_dh, out_dw, workspace, workspace_bytes, stream_of(stream));
    return launched("gradient of the log probabilities");
}

static int check_counts(const int64_t* counts, int32_t tensors)
{
    if (tensors < 0 || tensors > TG_MAX_TENSORS) return tg_fail(TG_ERR_INVALID_ARG, "tensors = %d outside 0..2^20", tensors);
    if (tensors && !counts) return null_argument();
    for (int32_t i = 0; i < tensors; ++i)
        if (counts[i] < 0 || counts[i] >= TG_MAX_VALUES) return tg_fail(TG_ERR_INVALID_ARG, "counts[%d] = %lld outside 0..2^40-1", i, (long long)counts[i]);
    return TG_OK;
}
static int check_grads(const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t tensors, float scale)
{
    CHECK(check_counts(counts, tensors));
    if (tensors && (!grads || !dtypes)) return null_argument();
    if (!(scale >= -3.4028234e38f && scale <= 3.4028234e38f)) return tg_fail(TG_ERR_INVALID_ARG, "scale must be finite");
    for (int32_t i = 0; i < tensors; ++i) {
        CHECK(check_dtype(dtypes[i]));
        if (counts[i] > 0 && !grads[i]) return null_argument();
        if ((uintptr_t)grads[i] % tg_type_bytes(dtypes[i])) return tg_fail(TG_ERR_INVALID_ARG, "grads[%d] is not aligned to its type", i);
    }
    return TG_OK;
}
extern "C" size_t tg_grad_norm_workspace(const int64_t* counts, int32_t tensors)
{
    return check_counts(counts, tensors) != TG_OK ? 0 : tg_grad_norm_space(counts, tensors);
}
extern "C" int tg_grad_norm(const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t tensors, float scale, float* out_norm,
                            void* workspace, size_t workspace_bytes, void* stream)
{
    CHECK(check_grads(grads, counts, dtypes, tensors, scale));
    if (!out_norm) return null_argument();
    CHECK(check_space(workspace, workspace_bytes, tg_grad_norm_space(counts, tensors)));
    tg_launch_clip(grads, nullptr, counts, dtypes, tensors, scale, 0.0f, out_norm, workspace, stream_of(stream));
    return launched("norm of the gradients");
}

// No tensor is written where another is read or written.
struct ClipRange {
    uintptr_t from, to;
    bool written;
};
static int check_ranges(const void* const* grads, void* const* out, const int64_t* counts, const int32_t* dtypes, int32_t tensors)
{
    ClipRange* const r = new (std::nothrow) ClipRange[2 * (size_t)tensors + 1];
    if (!r) return tg_fail(TG_ERR_INVALID_ARG, "no memory for the ranges of %d tensors", tensors);
    size_t n = 0;
    for (int32_t i = 0; i < tensors; ++i) {
        const uintptr_t bytes = (uintptr_t)counts[i] * tg_type_bytes(dtypes[i]), o = (uintptr_t)out[i], g = (uintptr_t)grads[i];
        if (!bytes) continue;
        r[n++] = ClipRange{o, o + bytes, true};
        if (o != g) r[n++] = ClipRange{g, g + bytes, false};
    }
    const auto before = [](const ClipRange& x, const ClipRange& y) { return x.from < y.from; };
    if (!std::is_sorted(r, r + n, before)) std::sort(r, r + n, before);
    uintptr_t read = 0, written = 0;             // the ends of what is before
    bool apart = true;
    for (size_t i = 0; i < n; ++i) {
        apart = apart && r[i].from >= written && !(r[i].written && r[i].from < read);
        uintptr_t& end = r[i].written ? written : read;
        if (r[i].to > end) end = r[i].to;
    }
    delete[] r;
    return apart ? TG_OK : tg_fail(TG_ERR_INVALID_ARG, "a tensor would be written where another one of the call is");
}
extern "C" int tg_clip_grads(const void* const* grads, void* const* out, const int64_t* counts, const int32_t* dtypes, int32_t tensors, float max_norm,
                             float scale, float* out_norm, void* workspace, size_t workspace_bytes, void* stream)
{
    CHECK(check_grads(grads, counts, dtypes, tensors, scale));
    if (!(max_norm >= 0.0f)) return tg_fail(TG_ERR_INVALID_ARG, "max_norm must not be below 0");
    if (!out_norm || (tensors && !out)) return null_argument();
    for (int32_t i = 0; i < tensors; ++i) {
        if (counts[i] > 0 && !out[i]) return null_argument();
        if ((uintptr_t)out[i] % tg_type_bytes(dtypes[i])) return tg_fail(TG_ERR_INVALID_ARG, "out[%d] is not aligned to its type", i);
    }
    CHECK(check_ranges(grads, out, counts, dtypes, tensors));
    CHECK(check_space(workspace, workspace_bytes, tg_grad_norm_space(counts, tensors)));
    tg_launch_clip(grads, out, counts, dtypes, tensors, scale, max_norm, out_norm, workspace, stream_of(stream));
    return launched("clipping of the gradients");
}
