// extern "C" entry points of the output head: validation on the host, then sbn_head.hip and sbn_mxfp4.hip.
#include <cmath>

#include "sbn_internal.hpp"

namespace sbn {

namespace {

sbn_status check_sizes(int64_t tokens, int64_t d_in, int64_t vocab, int64_t top_k)
{
    if (tokens <= 0 || d_in <= 0 || vocab <= 0 || top_k < 0) return SBN_EINVAL;
    if (d_in % 8 != 0 || d_in > HEAD_MAX_D || tokens > HEAD_MAX_TOKENS || vocab > HEAD_MAX_VOCAB) return SBN_EUNSUPPORTED;
    // a launch has fewer than 2^32 threads
    if (tokens * vocab > (int64_t)1 << 38 || tokens * d_in > (int64_t)1 << 34 || vocab * d_in > (int64_t)1 << 34) return SBN_EUNSUPPORTED;
    if (top_k > HEAD_MAX_TOP || (top_k && vocab > HEAD_MAX_TEACHER_VOCAB)) return SBN_EUNSUPPORTED;
    return SBN_OK;
}

// what all calls have in common; the caller has looked at its own pointers for null
sbn_status check_call(const HeadCall &h, const void *workspace, size_t ws_bytes, bool backward)
{
    if (!h.H || !h.W || !workspace) return SBN_EINVAL;
    const sbn_status st = check_sizes(h.tokens, h.d_in, h.vocab, h.top_k);
    if (st != SBN_OK) return st;
    if (h.top_idx && !(h.tau > 0.0f && std::isfinite(h.tau))) return SBN_EINVAL;
    if (h.top_idx && h.top_dtype != SBN_F32 && h.top_dtype != SBN_BF16) return SBN_EINVAL;
    if (!aligned(h.H, 16) || !aligned(h.W, 16) || !aligned(h.dH, 16) || !aligned(h.dW, 16) || !aligned(workspace, 256)) return SBN_EALIGN;
    if (!aligned(h.targets, 8) || !aligned(h.top_idx, 8) || !aligned(h.top_logits, h.top_dtype == SBN_BF16 ? 2 : 4) || !aligned(h.ce, 4) ||
        !aligned(h.kd, 4) || !aligned(h.lse1, 4) || !aligned(h.d_ce, 4) || !aligned(h.d_kd, 4))
        return SBN_EALIGN;
    return ws_bytes >= head_workspace_bytes(h.tokens, h.d_in, h.vocab, h.top_k, backward) ? SBN_OK : SBN_ESIZE;
}

HeadCall head_call(const void *H, const void *W, const int64_t *targets, int64_t tokens, int64_t d_in, int64_t vocab)
{
    HeadCall h{};
    h.H = H;
    h.W = W;
    h.targets = targets;
    h.tokens = tokens;
    h.d_in = d_in;
    h.vocab = vocab;
    return h;
}

void set_teacher(HeadCall &h, const int64_t *top_idx, const void *top_logits, sbn_dtype top_dtype, int64_t top_k, float tau)
{
    h.top_idx = top_idx;
    h.top_logits = top_logits;
    h.top_dtype = top_dtype;
    h.top_k = top_k;
    h.tau = tau;
}

// a matrix in microscaled form: a launch has fewer than 2^32 threads
sbn_status check_mxfp4(int64_t rows, int64_t cols)
{
    if (rows <= 0 || cols <= 0) return SBN_EINVAL;
    return cols % 8 != 0 || cols > MXFP4_MAX_COLS || rows > ((int64_t)1 << 34) / (ceil_div(cols, 128) * 128) ? SBN_EUNSUPPORTED : SBN_OK;
}

sbn_status check_mxfp4_product(int64_t tokens, int64_t d_in, int64_t d_out)
{
    sbn_status st = check_mxfp4(tokens, d_in);
    if (st == SBN_OK) st = check_mxfp4(d_out, d_in);
    return st != SBN_OK ? st : tokens * d_out >= (int64_t)1 << 38 ? SBN_EUNSUPPORTED : SBN_OK;
}

}  // namespace

}  // namespace sbn

using namespace sbn;

extern "C" {

void sbn_test_set_head_tiles(int logits, int gradients, int mxfp4)
{
    set_head_tiles(logits, gradients);
    set_mxfp4_tiles(mxfp4);
}

sbn_status sbn_test_chosen_mxfp4_tile(int64_t tokens, int64_t d_in, int64_t d_out, int *size, int64_t *threads)
{
    if (!size || !threads) return SBN_EINVAL;
    const sbn_status st = check_mxfp4_product(tokens, d_in, d_out);
    if (st == SBN_OK) *threads = mxfp4_tile_threads(tokens, d_in, d_out, size);
    return st;
}

sbn_status sbn_head_workspace_bytes(int64_t tokens, int64_t d_in, int64_t vocab, int64_t top_k, int backward, size_t *bytes)
{
    if (!bytes) return SBN_EINVAL;
    const sbn_status st = check_sizes(tokens, d_in, vocab, top_k);
    if (st == SBN_OK) *bytes = head_workspace_bytes(tokens, d_in, vocab, top_k, backward != 0);
    return st;
}

sbn_status sbn_head_cross_entropy(const void *H, const void *W, const int64_t *targets, int64_t tokens, int64_t d_in, int64_t vocab, float *ce, float *lse,
                                  void *workspace, size_t ws_bytes, void *stream)
{
    if (!targets || !ce || !lse) return SBN_EINVAL;
    HeadCall h = head_call(H, W, targets, tokens, d_in, vocab);
    h.ce = ce;
    h.lse1 = lse;
    const sbn_status st = check_call(h, workspace, ws_bytes, false);
    return st != SBN_OK ? st : launch_head_forward(h, workspace, static_cast<hipStream_t>(stream));
}

sbn_status sbn_head_cross_entropy_backward(const void *H, const void *W, const int64_t *targets, const float *lse, const float *d_ce, int64_t tokens,
                                           int64_t d_in, int64_t vocab, void *dH, void *dW, void *workspace, size_t ws_bytes, void *stream)
{
    if (!targets || !lse || !d_ce || (!dH && !dW)) return SBN_EINVAL;
    HeadCall h = head_call(H, W, targets, tokens, d_in, vocab);
    h.lse1 = const_cast<float *>(lse);   // read only
    h.d_ce = d_ce;
    h.dH = dH;
    h.dW = dW;
    const sbn_status st = check_call(h, workspace, ws_bytes, true);
    return st != SBN_OK ? st : launch_head_backward(h, workspace, static_cast<hipStream_t>(stream));
}

sbn_status sbn_head_distill(const void *H, const void *W, const int64_t *top_idx, const void *top_logits, sbn_dtype top_dtype, int64_t top_k, float tau,
                            const int64_t *targets, int64_t tokens, int64_t d_in, int64_t vocab, float *kd, float *ce, float *lse, void *workspace,
                            size_t ws_bytes, void *stream)
{
    if (!top_idx || !top_logits || top_k <= 0 || !kd || !lse || !targets != !ce) return SBN_EINVAL;
    HeadCall h = head_call(H, W, targets, tokens, d_in, vocab);
    set_teacher(h, top_idx, top_logits, top_dtype, top_k, tau);
    h.kd = kd;
    h.ce = ce;
    h.lse1 = lse;
    h.lse2 = lse + tokens;
    const sbn_status st = check_call(h, workspace, ws_bytes, false);
    return st != SBN_OK ? st : launch_head_forward(h, workspace, static_cast<hipStream_t>(stream));
}

sbn_status sbn_head_distill_backward(const void *H, const void *W, const int64_t *top_idx, const void *top_logits, sbn_dtype top_dtype, int64_t top_k,
                                     float tau, const int64_t *targets, const float *lse, const float *d_kd, const float *d_ce, int64_t tokens,
                                     int64_t d_in, int64_t vocab, void *dH, void *dW, void *workspace, size_t ws_bytes, void *stream)
{
    if (!top_idx || !top_logits || top_k <= 0 || !lse || !d_kd || !targets != !d_ce || (!dH && !dW)) return SBN_EINVAL;
    HeadCall h = head_call(H, W, targets, tokens, d_in, vocab);
    set_teacher(h, top_idx, top_logits, top_dtype, top_k, tau);
    h.lse1 = const_cast<float *>(lse);   // read only
    h.lse2 = h.lse1 + tokens;
    h.d_kd = d_kd;
    h.d_ce = d_ce;
    h.dH = dH;
    h.dW = dW;
    const sbn_status st = check_call(h, workspace, ws_bytes, true);
    return st != SBN_OK ? st : launch_head_backward(h, workspace, static_cast<hipStream_t>(stream));
}

sbn_status sbn_mxfp4_bytes(int64_t rows, int64_t cols, size_t *code_bytes, size_t *scale_bytes)
{
    if (!code_bytes || !scale_bytes) return SBN_EINVAL;
    const sbn_status st = check_mxfp4(rows, cols);
    if (st == SBN_OK) mxfp4_bytes(rows, cols, *code_bytes, *scale_bytes);
    return st;
}

sbn_status sbn_mxfp4_quantize(const void *X, sbn_dtype dtype, int64_t rows, int64_t cols, void *codes, void *scales, void *stream)
{
    if (!X || !codes || !scales || (dtype != SBN_F32 && dtype != SBN_BF16)) return SBN_EINVAL;
    const sbn_status st = check_mxfp4(rows, cols);
    if (st != SBN_OK) return st;
    if (!aligned(X, 16) || !aligned(codes, 16) || !aligned(scales, 4)) return SBN_EALIGN;
    return launch_mxfp4_quantize(X, dtype, rows, cols, static_cast<uint8_t *>(codes), static_cast<uint8_t *>(scales), static_cast<hipStream_t>(stream));
}

sbn_status sbn_mxfp4_dequantize(const void *codes, const void *scales, int64_t rows, int64_t cols, void *Y, sbn_dtype dtype, void *stream)
{
    if (!codes || !scales || !Y || (dtype != SBN_F32 && dtype != SBN_BF16)) return SBN_EINVAL;
    const sbn_status st = check_mxfp4(rows, cols);
    if (st != SBN_OK) return st;
    if (!aligned(Y, 16) || !aligned(codes, 16) || !aligned(scales, 4)) return SBN_EALIGN;
    return launch_mxfp4_dequantize(static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), rows, cols, Y, dtype,
                                   static_cast<hipStream_t>(stream));
}

sbn_status sbn_mxfp4_workspace_bytes(int64_t tokens, int64_t d_in, size_t *bytes)
{
    if (!bytes) return SBN_EINVAL;
    const sbn_status st = check_mxfp4(tokens, d_in);
    if (st == SBN_OK) *bytes = mxfp4_workspace_bytes(tokens, d_in);
    return st;
}

sbn_status sbn_mxfp4_linear(const void *X, int64_t tokens, int64_t d_in, int64_t d_out, const void *codes, const void *scales, const float *bias, float *Y,
                            void *workspace, size_t ws_bytes, void *stream)
{
    if (!X || !codes || !scales || !Y || !workspace) return SBN_EINVAL;
    const sbn_status st = check_mxfp4_product(tokens, d_in, d_out);
    if (st != SBN_OK) return st;
    if (!aligned(X, 16) || !aligned(codes, 16) || !aligned(scales, 4) || !aligned(bias, 4) || !aligned(Y, 16) || !aligned(workspace, 256)) return SBN_EALIGN;
    if (ws_bytes < mxfp4_workspace_bytes(tokens, d_in)) return SBN_ESIZE;
    return launch_mxfp4_linear(X, tokens, d_in, d_out, static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), bias, Y, workspace,
                               static_cast<hipStream_t>(stream));
}

}  // extern "C"
