// extern "C" entry points of the parts of a training step around the layers and the head: validation on the host, then sbn_norm.hip,
// sbn_embed.hip and sbn_optim.hip.
#include <algorithm>
#include <cmath>
#include <new>

#include "sbn_internal.hpp"

namespace sbn {

namespace {

bool known(sbn_dtype t) { return t == SBN_F32 || t == SBN_BF16; }
size_t size_of(sbn_dtype t) { return t == SBN_F32 ? 4 : 2; }

sbn_status check_norm_sizes(int64_t tokens, int64_t d)
{
    if (tokens <= 0 || d <= 0) return SBN_EINVAL;
    return tokens > ROWS_MAX || d > NORM_MAX_D ? SBN_EUNSUPPORTED : SBN_OK;
}

sbn_status check_embedding_sizes(int64_t tokens, int64_t d, int64_t vocab)
{
    if (tokens <= 0 || d <= 0 || vocab <= 0) return SBN_EINVAL;
    if (tokens > ROWS_MAX || vocab > ROWS_MAX || d > HEAD_MAX_D) return SBN_EUNSUPPORTED;
    return tokens * d > (int64_t)1 << 34 || vocab * d > (int64_t)1 << 34 ? SBN_EUNSUPPORTED : SBN_OK;
}

constexpr int64_t OPTIM_MAX_VALUES = (int64_t)1 << 31;   // of a tensor: its values are numbered in 32 bits for the rounding

sbn_status check_tensors(int count, const int64_t *sizes)
{
    if (count <= 0 || !sizes) return SBN_EINVAL;
    if (count > OPTIM_MAX_TENSORS) return SBN_EUNSUPPORTED;
    for (int i = 0; i < count; ++i)
        if (sizes[i] <= 0) return SBN_EINVAL;
    for (int i = 0; i < count; ++i)
        if (sizes[i] > OPTIM_MAX_VALUES) return SBN_EUNSUPPORTED;
    return SBN_OK;
}

sbn_status check_pointers(int count, const void *const *p, size_t align)
{
    for (int i = 0; i < count; ++i)
        if (!p[i]) return SBN_EINVAL;
    for (int i = 0; i < count; ++i)
        if (!aligned(p[i], align)) return SBN_EALIGN;
    return SBN_OK;
}

// whether no two of the buffers share a byte; lists in the order of their addresses are looked through once
bool apart(int count, const void *const *p, const int64_t *sizes, int64_t bytes_of(int64_t, size_t), size_t size)
{
    struct Range {
        uintptr_t begin, end;
    };
    const auto range = [&](int i) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p[i]);
        return Range{at, at + (uintptr_t)bytes_of(sizes[i], size)};
    };
    bool in_order = true;
    for (int i = 1; i < count && in_order; ++i) in_order = range(i).begin >= range(i - 1).end;
    if (in_order) return true;
    Range *r = new (std::nothrow) Range[count];
    if (!r) return false;
    for (int i = 0; i < count; ++i) r[i] = range(i);
    std::sort(r, r + count, [](const Range &a, const Range &b) { return a.begin < b.begin; });
    bool good = true;
    for (int i = 1; i < count; ++i) good = good && r[i].begin >= r[i - 1].end;
    delete[] r;
    return good;
}
int64_t plain_bytes(int64_t n, size_t size) { return n * (int64_t)size; }
int64_t code_bytes(int64_t n, size_t) { return ceil_div(n, 32) * 32; }
int64_t scale_bytes(int64_t n, size_t) { return ceil_div(n, 32); }

}  // namespace

}  // namespace sbn

using namespace sbn;

extern "C" {

sbn_status sbn_norm(const void *X, const void *residual, sbn_dtype dtype, int64_t tokens, int64_t d_in, const float *gain, const float *bias, float eps, int layer,
                    void *Y, void *sum_out, void *stream)
{
    if (!X || !Y || !residual != !sum_out || !known(dtype) || !(eps >= 0.0f) || !std::isfinite(eps)) return SBN_EINVAL;
    const sbn_status st = check_norm_sizes(tokens, d_in);
    if (st != SBN_OK) return st;
    const size_t a = size_of(dtype);
    if (!aligned(X, a) || !aligned(residual, a) || !aligned(Y, a) || !aligned(sum_out, a) || !aligned(gain, 4) || !aligned(bias, 4)) return SBN_EALIGN;
    if (Y == sum_out) return SBN_EINVAL;
    return launch_norm(X, residual, dtype, tokens, d_in, gain, bias, eps, layer != 0, Y, sum_out, static_cast<hipStream_t>(stream));
}

sbn_status sbn_norm_workspace_bytes(int64_t tokens, int64_t d_in, size_t *bytes)
{
    if (!bytes) return SBN_EINVAL;
    const sbn_status st = check_norm_sizes(tokens, d_in);
    if (st == SBN_OK) *bytes = norm_workspace_bytes(tokens, d_in);
    return st;
}

sbn_status sbn_norm_backward(const void *X, const void *dY, const void *d_residual, sbn_dtype dtype, int64_t tokens, int64_t d_in, const float *gain, float eps,
                             int layer, void *dX, float *dgain, float *dbias, void *workspace, size_t ws_bytes, void *stream)
{
    if (!X || !dY || (!dX && !dgain && !dbias) || (d_residual && !dX) || !workspace || !known(dtype) || !(eps >= 0.0f) || !std::isfinite(eps)) return SBN_EINVAL;
    const sbn_status st = check_norm_sizes(tokens, d_in);
    if (st != SBN_OK) return st;
    const size_t a = size_of(dtype);
    if (!aligned(X, a) || !aligned(dY, a) || !aligned(d_residual, a) || !aligned(dX, a) || !aligned(gain, 4) || !aligned(dgain, 4) || !aligned(dbias, 4) ||
        !aligned(workspace, 256))
        return SBN_EALIGN;
    if (ws_bytes < norm_workspace_bytes(tokens, d_in)) return SBN_ESIZE;
    return launch_norm_backward(X, dY, d_residual, dtype, tokens, d_in, gain, eps, layer != 0, dX, dgain, dbias, workspace, static_cast<hipStream_t>(stream));
}

sbn_status sbn_embedding(const void *E, sbn_dtype table_dtype, int64_t vocab, int64_t d_in, const int64_t *ids, int64_t tokens, float scale, void *Y, sbn_dtype y_dtype,
                         void *stream)
{
    if (!E || !ids || !Y || !known(table_dtype) || !known(y_dtype) || !std::isfinite(scale)) return SBN_EINVAL;
    const sbn_status st = check_embedding_sizes(tokens, d_in, vocab);
    if (st != SBN_OK) return st;
    if (!aligned(E, size_of(table_dtype)) || !aligned(Y, size_of(y_dtype)) || !aligned(ids, 8)) return SBN_EALIGN;
    return launch_embedding(E, table_dtype, vocab, d_in, ids, tokens, scale, Y, y_dtype, static_cast<hipStream_t>(stream));
}

sbn_status sbn_embedding_workspace_bytes(int64_t tokens, int64_t d_in, int64_t vocab, size_t *bytes)
{
    if (!bytes) return SBN_EINVAL;
    const sbn_status st = check_embedding_sizes(tokens, d_in, vocab);
    if (st == SBN_OK) *bytes = embedding_workspace_bytes(tokens, d_in, vocab);
    return st;
}

sbn_status sbn_embedding_backward(const void *dY, sbn_dtype y_dtype, const int64_t *ids, int64_t tokens, int64_t vocab, int64_t d_in, float scale, int accumulate,
                                  void *dE, sbn_dtype table_dtype, void *workspace, size_t ws_bytes, void *stream)
{
    if (!dY || !ids || !dE || !workspace || !known(table_dtype) || !known(y_dtype) || !std::isfinite(scale)) return SBN_EINVAL;
    const sbn_status st = check_embedding_sizes(tokens, d_in, vocab);
    if (st != SBN_OK) return st;
    if (!aligned(dY, size_of(y_dtype)) || !aligned(dE, size_of(table_dtype)) || !aligned(ids, 8) || !aligned(workspace, 256)) return SBN_EALIGN;
    if (ws_bytes < embedding_workspace_bytes(tokens, d_in, vocab)) return SBN_ESIZE;
    return launch_embedding_backward(dY, y_dtype, ids, tokens, vocab, d_in, scale, accumulate != 0, dE, table_dtype, workspace, static_cast<hipStream_t>(stream));
}

sbn_status sbn_grad_norm_workspace_bytes(int count, const int64_t *sizes, size_t *bytes)
{
    if (!bytes) return SBN_EINVAL;
    const sbn_status st = check_tensors(count, sizes);
    if (st == SBN_OK) *bytes = grad_norm_workspace_bytes(count, sizes);
    return st;
}

sbn_status sbn_grad_norm(int count, const void *const *grads, sbn_dtype dtype, const int64_t *sizes, float max_norm, float *out, void *workspace, size_t ws_bytes,
                         void *stream)
{
    if (!grads || !out || !workspace || !known(dtype) || !(max_norm > 0.0f)) return SBN_EINVAL;
    sbn_status st = check_tensors(count, sizes);
    if (st == SBN_OK) st = check_pointers(count, grads, size_of(dtype));
    if (st != SBN_OK) return st;
    if (!aligned(out, 4) || !aligned(workspace, 256)) return SBN_EALIGN;
    if (ws_bytes < grad_norm_workspace_bytes(count, sizes)) return SBN_ESIZE;
    return launch_grad_norm(count, grads, dtype, sizes, max_norm, out, workspace, static_cast<hipStream_t>(stream));
}

sbn_status sbn_adamw_state_bytes(int64_t n, size_t *codes, size_t *scales)
{
    if (!codes || !scales) return SBN_EINVAL;
    const sbn_status st = check_tensors(1, &n);
    if (st != SBN_OK) return st;
    *codes = (size_t)code_bytes(n, 0);
    *scales = (size_t)scale_bytes(n, 0);
    return SBN_OK;
}

sbn_status sbn_adamw_state_values(const void *codes, const uint8_t *scales, int64_t n, int second, void *out, sbn_dtype dtype, void *stream)
{
    if (!codes || !scales || !out || !known(dtype)) return SBN_EINVAL;
    const sbn_status st = check_tensors(1, &n);
    if (st != SBN_OK) return st;
    if (!aligned(codes, 8) || !aligned(out, size_of(dtype))) return SBN_EALIGN;
    return launch_adamw_state_values(codes, scales, n, second != 0, out, dtype, static_cast<hipStream_t>(stream));
}

sbn_status sbn_adamw_step(int count, void *const *params, sbn_dtype param_dtype, const void *const *grads, sbn_dtype grad_dtype, void *const *m, void *const *v,
                          uint8_t *const *m_scales, uint8_t *const *v_scales, const int64_t *sizes, const float *weight_decay, const float *lr, const int64_t *step,
                          double beta1, double beta2, double eps, const float *clip, const uint64_t *seed, void *stream)
{
    if (!params || !grads || !m || !v || !m_scales != !v_scales || !lr || !step || !known(param_dtype) || !known(grad_dtype)) return SBN_EINVAL;
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !std::isfinite((float)eps)) return SBN_EINVAL;
    sbn_status st = check_tensors(count, sizes);
    if (st != SBN_OK) return st;
    const bool bits8 = m_scales != nullptr;
    const auto check = [&](const void *const *p, size_t a) {
        if (st == SBN_OK) st = check_pointers(count, p, a);
    };
    check(params, size_of(param_dtype));
    check(grads, size_of(grad_dtype));
    check(m, bits8 ? 8 : 4);
    check(v, bits8 ? 8 : 4);
    if (bits8) {
        check(reinterpret_cast<const void *const *>(m_scales), 1);
        check(reinterpret_cast<const void *const *>(v_scales), 1);
    }
    if (st != SBN_OK) return st;
    if (!aligned(lr, 4) || !aligned(clip, 4) || !aligned(step, 8)) return SBN_EALIGN;
    for (int i = 0; weight_decay && i < count; ++i)
        if (!std::isfinite(weight_decay[i])) return SBN_EINVAL;
    // a tensor that is listed twice would be written by two blocks at once
    bool good = apart(count, params, sizes, plain_bytes, size_of(param_dtype));
    good = good && apart(count, m, sizes, bits8 ? code_bytes : plain_bytes, 4) && apart(count, v, sizes, bits8 ? code_bytes : plain_bytes, 4);
    if (good && bits8)
        good = apart(count, reinterpret_cast<const void *const *>(m_scales), sizes, scale_bytes, 1) &&
               apart(count, reinterpret_cast<const void *const *>(v_scales), sizes, scale_bytes, 1);
    if (!good) return SBN_EINVAL;
    AdamWCall c{};
    c.count = count;
    c.params = params;
    c.param_dtype = param_dtype;
    c.grads = grads;
    c.grad_dtype = grad_dtype;
    c.m = m;
    c.v = v;
    c.m_scales = m_scales;
    c.v_scales = v_scales;
    c.sizes = sizes;
    c.weight_decay = weight_decay;
    c.lr = lr;
    c.step = step;
    c.beta1 = beta1;
    c.beta2 = beta2;
    c.eps = eps;
    c.clip = clip;
    c.seed = seed;
    return launch_adamw(c, static_cast<hipStream_t>(stream));
}

}  // extern "C"
