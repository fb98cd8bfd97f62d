// C ABI of the operators around the melded layer: argument validation on the host, then kernel launches on the caller's stream.
// Nothing here allocates, synchronises or keeps state.
#include <cmath>

#include "logprob.h"
#include "mx.h"
#include "norm.h"
#include "swiglu.h"

namespace falqon {
namespace {

constexpr int64_t kMaxRows = int64_t(1) << 24, kMaxWidth = int64_t(1) << 20, kMaxElements = int64_t(1) << 40;

template <typename... P>
bool any_misaligned(P... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) & 15u) != 0; }     // NULL is aligned
template <typename... P>
bool any_odd(unsigned by, P... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) & (by - 1)) != 0; }
bool bad_type(falqon_dtype t) { return t != FALQON_BF16 && t != FALQON_F32; }
bool bad_matrix(int64_t rows, int64_t cols, int64_t by) { return rows < 1 || rows > kMaxRows || cols < by || cols > kMaxWidth || cols % by; }
bool bad_stride(int64_t ld, int64_t cols) { return ld < cols || ld % 16 || ld > (int64_t(1) << 32); }
// What a launch takes along a dimension: fewer than 2^32 threads.
bool too_many(int64_t blocks, int64_t threads) { return blocks > ((int64_t(1) << 32) - 1) / threads; }
// the passes of one 16-byte piece a lane (mx_common.h), in which a row's last block of 32 columns counts whole
bool too_many_pieces(int64_t rows, int64_t cols, falqon_dtype t) { return too_many((rows * ((cols + 31) / 32 * (t == FALQON_F32 ? 8 : 4)) + 255) / 256, 256); }
falqon_status status_of(hipError_t e) { return e == hipSuccess ? FALQON_OK : FALQON_ERR_HIP; }
hipStream_t on(void* stream) { return static_cast<hipStream_t>(stream); }

}  // namespace
}  // namespace falqon

using namespace falqon;

extern "C" {

int64_t falqon_mx4_exp_pitch(int64_t cols) { return cols < 32 || cols % 32 ? 0 : (cols + 511) / 512 * 16; }

static bool bad_mx(int64_t rows, int64_t cols, int64_t ld, falqon_mx_fmt fmt, falqon_dtype t)
{
    return rows < 0 || rows > kMaxRows || cols < 16 || cols > kMaxWidth || cols % (fmt == FALQON_MX_E2M1 ? 32 : 16) || rows * cols > kMaxElements ||
           too_many_pieces(rows, cols, t) || bad_stride(ld, cols);
}

falqon_status falqon_mx_quantize(const void* x, falqon_dtype xt, int64_t rows, int64_t cols, int64_t ld_x, falqon_mx_fmt fmt,
                                 uint8_t* q, uint8_t* exps, void* stream)
{
    if (bad_type(xt) || (fmt != FALQON_MX_E4M3 && fmt != FALQON_MX_E2M1)) return FALQON_ERR_ENUM;
    if (bad_mx(rows, cols, ld_x, fmt, xt)) return FALQON_ERR_SHAPE;
    if (rows == 0) return FALQON_OK;
    if (!x || !q || !exps) return FALQON_ERR_NULL;
    if (any_misaligned(x, q, exps)) return FALQON_ERR_ALIGN;
    return status_of(launch_mx_quantize(x, xt == FALQON_F32, rows, cols, ld_x, fmt == FALQON_MX_E2M1, q, exps, on(stream)));
}

falqon_status falqon_mx_dequantize(const uint8_t* q, const uint8_t* exps, falqon_mx_fmt fmt, int64_t rows, int64_t cols,
                                   void* x, falqon_dtype xt, int64_t ld_x, void* stream)
{
    if (bad_type(xt) || (fmt != FALQON_MX_E4M3 && fmt != FALQON_MX_E2M1)) return FALQON_ERR_ENUM;
    if (bad_mx(rows, cols, ld_x, fmt, xt)) return FALQON_ERR_SHAPE;
    if (rows == 0) return FALQON_OK;
    if (!x || !q || !exps) return FALQON_ERR_NULL;
    if (any_misaligned(x, q, exps)) return FALQON_ERR_ALIGN;
    return status_of(launch_mx_values(q, exps, rows, cols, fmt == FALQON_MX_E2M1, x, xt == FALQON_F32, ld_x, on(stream)));
}

falqon_status falqon_mx4_linear(const void* x, const uint8_t* wq, const uint8_t* w_exp, int64_t T, int64_t n, int64_t m,
                                uint8_t* xq, uint8_t* x_exp, void* y, falqon_dtype yt, void* stream)
{
    if (bad_type(yt)) return FALQON_ERR_ENUM;
    if (bad_matrix(T, n, 32) || bad_matrix(T, m, 16) || T * n > kMaxElements || T * m > kMaxElements ||
        too_many(((T + 255) / 256 * ((m + 255) / 256) + 7) / 8 * 8, 256) || (x && too_many_pieces(T, n, FALQON_BF16)))
        return FALQON_ERR_SHAPE;
    if (!wq || !w_exp || !xq || !x_exp || !y) return FALQON_ERR_NULL;
    if (any_misaligned(x, wq, w_exp, xq, x_exp, y)) return FALQON_ERR_ALIGN;
    const Mx4Gemm product{xq, x_exp, wq, w_exp, T, m, n, y, yt == FALQON_F32};
    const bool thin = mx4_thin_supported(T, m), inside = x && thin && mx4_thin_quantizes(T, n);
    if (x && !inside) {
        const hipError_t e = launch_mx_quantize(x, false, T, n, n, true, xq, x_exp, on(stream));
        if (e != hipSuccess) return FALQON_ERR_HIP;
    }
    return status_of(thin ? launch_mx4_thin(product, inside ? x : nullptr, xq, x_exp, on(stream)) : launch_mx4_gemm(product, on(stream)));
}

falqon_status falqon_norm_fwd(const falqon_norm_fwd_args* a, void* stream)
{
    if (!a) return FALQON_ERR_NULL;
    if (bad_type(a->xt)) return FALQON_ERR_ENUM;
    if (bad_matrix(a->T, a->d, 16) || a->d > kNormMaxWidth || bad_stride(a->ld_x, a->d) || (a->b && bad_stride(a->ld_b, a->d)) ||
        !std::isfinite(static_cast<float>(a->scale)) || !(a->eps >= 0.0) || norm_fwd_threads(a->T, a->d, a->xt == FALQON_F32) >= int64_t(1) << 32)
        return FALQON_ERR_SHAPE;
    if (!a->x || !a->w || !a->h || !a->rstd || (!a->b && (a->w_post || a->gate || a->bq)) || (a->b && !a->s) || (a->w_post && !a->rstd_b) ||
        !a->sq != !a->s_exp || !a->bq != !a->b_exp)
        return FALQON_ERR_NULL;
    if (any_misaligned(a->x, a->b, a->w, a->w_post, a->gate, a->s, a->h, a->sq, a->bq) || any_odd(4, a->rstd, a->rstd_b)) return FALQON_ERR_ALIGN;
    const NormFwd n{a->x, a->b, a->w, a->w_post, a->gate, static_cast<float>(a->scale), static_cast<float>(a->eps), a->T, a->d, a->ld_x, a->ld_b,
                    a->s, a->h, a->rstd, a->rstd_b, a->sq, a->s_exp, a->bq, a->b_exp};
    return status_of(launch_norm_fwd(n, a->xt == FALQON_F32, on(stream)));
}

size_t falqon_norm_workspace_bytes(int64_t T, int64_t d)
{
    if (bad_matrix(T, d, 16) || d > kNormMaxWidth) return 0;
    return static_cast<size_t>(T < kNormGroups ? T : kNormGroups) * static_cast<size_t>(d) * 2 * sizeof(float);
}

falqon_status falqon_norm_bwd(const falqon_norm_bwd_args* a, void* stream)
{
    if (!a) return FALQON_ERR_NULL;
    if (bad_type(a->xt)) return FALQON_ERR_ENUM;
    const bool codes = a->s_exp != nullptr, reads_b = a->w_post || a->dgate;
    if (bad_matrix(a->T, a->d, 16) || a->d > kNormMaxWidth || bad_stride(a->ld_dh, a->d) || (a->ds && bad_stride(a->ld_ds, a->d)) ||
        (!codes && (bad_stride(a->ld_s, a->d) || (reads_b && bad_stride(a->ld_b, a->d)))) || !std::isfinite(static_cast<float>(a->scale)))
        return FALQON_ERR_SHAPE;
    if (!a->dh || !a->s || !a->w || !a->rstd || !a->dx || (reads_b && (!a->b || (codes && !a->b_exp))) || (a->w_post && !a->rstd_b) ||
        (a->dw_post && !a->w_post))
        return FALQON_ERR_NULL;
    if (any_misaligned(a->dh, a->ds, a->s, a->b, a->w, a->w_post, a->gate, a->dx, a->db, a->ws) || any_odd(4, a->rstd, a->rstd_b, a->dw, a->dw_post, a->dgate))
        return FALQON_ERR_ALIGN;
    if ((a->dw || a->dw_post || a->dgate) && (!a->ws || a->ws_bytes < falqon_norm_workspace_bytes(a->T, a->d))) return FALQON_ERR_WORKSPACE;
    const NormBwd n{a->dh, a->ds, a->ld_dh, a->ld_ds, a->s, a->ld_s, a->s_exp, a->rstd, a->b, a->ld_b, a->b_exp, a->rstd_b, a->w, a->w_post, a->gate,
                    static_cast<float>(a->scale), a->T, a->d, a->dx, a->db, a->dw, a->dw_post, a->dgate};
    return status_of(launch_norm_bwd(n, a->xt == FALQON_F32, static_cast<float*>(a->ws), on(stream)));
}

falqon_status falqon_swiglu_fwd(const void* g, const void* u, falqon_dtype xt, int64_t T, int64_t m, int64_t ld_g, int64_t ld_u,
                                void* h, uint8_t* gq, uint8_t* g_exp, uint8_t* uq, uint8_t* u_exp, void* stream)
{
    if (bad_type(xt)) return FALQON_ERR_ENUM;
    if (bad_matrix(T, m, 16) || T * m > kMaxElements || too_many_pieces(T, m, xt) || bad_stride(ld_g, m) || bad_stride(ld_u, m)) return FALQON_ERR_SHAPE;
    if (!g || !u || !h || !gq != !g_exp || !gq != !uq || !gq != !u_exp) return FALQON_ERR_NULL;
    if (any_misaligned(g, u, h, gq, uq)) return FALQON_ERR_ALIGN;
    return status_of(launch_swiglu_fwd(SwigluFwd{g, u, ld_g, ld_u, T, m, h, gq, g_exp, uq, u_exp}, xt == FALQON_F32, on(stream)));
}

falqon_status falqon_swiglu_bwd(const void* dh, int64_t ld_dh, const void* g, const void* u, const uint8_t* g_exp, const uint8_t* u_exp,
                                int64_t ld_g, int64_t ld_u, falqon_dtype xt, int64_t T, int64_t m, void* dg, void* du, void* stream)
{
    if (bad_type(xt)) return FALQON_ERR_ENUM;
    if (bad_matrix(T, m, 16) || T * m > kMaxElements || too_many_pieces(T, m, xt) || bad_stride(ld_dh, m) ||
        (!g_exp && (bad_stride(ld_g, m) || bad_stride(ld_u, m))))
        return FALQON_ERR_SHAPE;
    if (!dh || !g || !u || !dg || !du || !g_exp != !u_exp) return FALQON_ERR_NULL;
    if (any_misaligned(dh, g, u, dg, du)) return FALQON_ERR_ALIGN;
    return status_of(launch_swiglu_bwd(SwigluBwd{dh, ld_dh, g, u, ld_g, ld_u, g_exp, u_exp, T, m, dg, du}, xt == FALQON_F32, on(stream)));
}

static bool bad_logits(int64_t T, int64_t V) { return T < 1 || T > kMaxRows || V < 1 || V > kMaxWidth; }
static bool bad_pairs(int64_t P) { return P < 1 || P > 65536; }

size_t falqon_logprob_workspace_bytes(int64_t T, int64_t V, int64_t P)
{
    if (bad_logits(T, V) || bad_pairs(P)) return 0;
    const int splits = token_splits(T, V);
    const size_t parts = splits > 1 ? static_cast<size_t>(T) * static_cast<size_t>(splits) * sizeof(float2) : 0, pairs = static_cast<size_t>(P) * sizeof(float);
    return ((parts > pairs ? parts : pairs) + 15) / 16 * 16;
}

falqon_status falqon_token_logprob(const void* logits, falqon_dtype lt, int64_t T, int64_t V, int64_t ld, const int64_t* labels,
                                   float* logp, float* lse, void* ws, size_t ws_bytes, void* stream)
{
    return falqon_token_logprob_low(logits, lt, T, V, ld, labels, logp, lse, nullptr, ws, ws_bytes, stream);
}

falqon_status falqon_token_logprob_low(const void* logits, falqon_dtype lt, int64_t T, int64_t V, int64_t ld, const int64_t* labels,
                                       float* logp, float* lse, float* lse_low, void* ws, size_t ws_bytes, void* stream)
{
    if (bad_type(lt)) return FALQON_ERR_ENUM;
    if (bad_logits(T, V) || ld < V || too_many(T, 256)) return FALQON_ERR_SHAPE;
    if (!logits || !labels || !logp || !lse) return FALQON_ERR_NULL;
    if (any_odd(lt == FALQON_F32 ? 4 : 2, logits) || any_odd(8, labels) || any_odd(4, logp, lse, lse_low) || any_misaligned(ws)) return FALQON_ERR_ALIGN;
    if (!ws || ws_bytes < falqon_logprob_workspace_bytes(T, V, 1)) return FALQON_ERR_WORKSPACE;
    return status_of(launch_token_logprob(TokenLogprob{logits, ld, labels, T, V, logp, lse, lse_low, static_cast<float2*>(ws)}, lt == FALQON_F32, on(stream)));
}

falqon_status falqon_token_logprob_bwd(const float* d_logp, const void* logits, falqon_dtype lt, int64_t T, int64_t V, int64_t ld,
                                       const int64_t* labels, const float* lse, void* dlogits, int64_t ld_d, void* stream)
{
    return falqon_token_logprob_bwd_low(d_logp, logits, lt, T, V, ld, labels, lse, nullptr, dlogits, ld_d, stream);
}

falqon_status falqon_token_logprob_bwd_low(const float* d_logp, const void* logits, falqon_dtype lt, int64_t T, int64_t V, int64_t ld,
                                           const int64_t* labels, const float* lse, const float* lse_low, void* dlogits, int64_t ld_d, void* stream)
{
    if (bad_type(lt)) return FALQON_ERR_ENUM;
    if (bad_logits(T, V) || too_many(T, 256) || ld < V || ld_d < V || (logits == dlogits && ld != ld_d)) return FALQON_ERR_SHAPE;
    if (!d_logp || !logits || !labels || !lse || !dlogits) return FALQON_ERR_NULL;
    if (any_odd(lt == FALQON_F32 ? 4 : 2, logits, dlogits) || any_odd(8, labels) || any_odd(4, d_logp, lse, lse_low)) return FALQON_ERR_ALIGN;
    return status_of(launch_token_logprob_bwd(TokenLogprobBwd{d_logp, logits, ld, labels, lse, lse_low, T, V, dlogits, ld_d}, lt == FALQON_F32, on(stream)));
}

falqon_status falqon_preference_loss(const float* logp, const float* ref_logp, const int64_t* offsets, int64_t T, int64_t P, double beta,
                                     double smoothing, float* loss, float* rewards, float* d_logp, void* ws, size_t ws_bytes, void* stream)
{
    if (T < 1 || T > kMaxRows || bad_pairs(P) || !std::isfinite(static_cast<float>(beta)) || !(smoothing >= 0.0 && smoothing < 0.5)) return FALQON_ERR_SHAPE;
    if (!logp || !ref_logp || !offsets || !loss || !rewards || !d_logp) return FALQON_ERR_NULL;
    if (any_odd(8, offsets) || any_odd(4, logp, ref_logp, loss, rewards, d_logp) || any_misaligned(ws)) return FALQON_ERR_ALIGN;
    if (!ws || ws_bytes < falqon_logprob_workspace_bytes(T, 1, P)) return FALQON_ERR_WORKSPACE;
    return status_of(launch_preference_loss(logp, ref_logp, offsets, T, P, static_cast<float>(beta), static_cast<float>(smoothing), static_cast<float*>(ws), loss,
                                            rewards, d_logp, on(stream)));
}

}  // extern "C"
