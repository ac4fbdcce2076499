// RMS and layer norm of rows, forward and backward.
//
// With x a row, mu its mean (RMS form: 0), r = 1 / sqrt(mean (x - mu)^2 + eps) and h = (x - mu) r:
//   y  = h gain (+ bias)
//   dx = r (a - mean a (layer form) - h mean(a h)) (+ d_residual),   a = dy gain
//   dgain = sum over rows of dy h,   dbias = sum over rows of dy
// A row is read once and held in registers: its statistics are sums over what a thread holds, so the backward pass makes them again
// rather than keeping them.  Bound by memory.
//
// The mean of a row is made in two steps, a first sum and the sum of what that leaves over (the differences to a nearby value are exact or
// nearly so), so that rows far off zero keep their digits; the second sum shares its reduction with the squares.
#include <algorithm>

#include "sbn_internal.hpp"
#include "sbn_rows.hpp"

namespace sbn {

namespace {

struct NormArgs {
    const void *X, *R, *dY;   // R: residual (forward), d_residual (backward), or null
    const float *gain, *bias;
    void *Y, *S, *dX;
    float *partials;          // [2][blocks][d]: shares of dgain and dbias
    int64_t tokens, d;
    float eps;
    int want_gain, want_bias;
};

// sums over the TPT threads of a row, K at a time
template <int TPT, int K, class F> __device__ __forceinline__ void row_sums(F (&s)[K], F *scratch)
{
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = wave_sum(s[k]);
    if constexpr (TPT > 64) {
        __syncthreads();   // the scratch may still be read
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) scratch[(threadIdx.x >> 6) * K + k] = s[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) s[k] = 0;
        for (int w = 0; w < TPT / 64; ++w) {
#pragma unroll
            for (int k = 0; k < K; ++k) s[k] += scratch[w * K + k];
        }
    }
}

// TPT threads share a row: a wavefront (four rows to a block) or a block.  VMAX vectors of the row in each.
template <sbn_dtype DT, bool LAYER, int TPT, int VMAX> __global__ void __launch_bounds__(TPT < 256 ? 256 : TPT) norm_kernel(const NormArgs n)
{
    constexpr int E = Row<DT>::E;
    constexpr int ROWS = TPT < 256 ? 256 / TPT : 1;
    __shared__ double scratch[32];
    const int sub = threadIdx.x % TPT;
    const int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPT;
    if (t >= n.tokens) return;   // whole wavefronts; a block that shares a row has one
    const int64_t first = t * n.d;
    const auto row = [&](const void *p) { return static_cast<const void *>(static_cast<const typename Row<DT>::value *>(p) + first); };
    const auto out = [&](void *p) { return static_cast<void *>(static_cast<typename Row<DT>::value *>(p) + first); };
    u32x4 x[VMAX];
#pragma unroll
    for (int i = 0; i < VMAX; ++i) x[i] = load_vec<DT>(row(n.X), sub + i * TPT, n.d);
    if (n.R) {
        u32x4 r[VMAX];
#pragma unroll
        for (int i = 0; i < VMAX; ++i) r[i] = load_vec<DT>(row(n.R), sub + i * TPT, n.d);
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            float a[E], b[E];
            Row<DT>::unpack(x[i], a);
            Row<DT>::unpack(r[i], b);
#pragma unroll
            for (int k = 0; k < E; ++k) a[k] += b[k];
            x[i] = Row<DT>::pack(a);
            store_vec<DT>(out(n.S), sub + i * TPT, n.d, x[i]);
        }
    }
    float mu = 0.0f, rest = 0.0f, r;
    if constexpr (LAYER) {
        float s[1] = {0.0f}, q[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            float f[E];
            Row<DT>::unpack(x[i], f);
#pragma unroll
            for (int k = 0; k < E; ++k) s[0] += f[k];
        }
        row_sums<TPT>(s, reinterpret_cast<float *>(scratch));
        mu = s[0] / (float)n.d;
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            float f[E];
            Row<DT>::unpack(x[i], f);
#pragma unroll
            for (int k = 0; k < E; ++k)
                if ((sub + i * TPT) * E + k < n.d) {
                    const float c = f[k] - mu;
                    q[0] += c;
                    q[1] += c * c;
                }
        }
        row_sums<TPT>(q, reinterpret_cast<float *>(scratch));
        rest = q[0] / (float)n.d;
        r = 1.0f / sqrtf(fmaxf(q[1] / (float)n.d - rest * rest, 0.0f) + n.eps);
    } else {
        // in double, rounded once: the row's factor is then the one of the fused norm and quantizer, bit for bit
        double s[1] = {0.0};
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            float f[E];
            Row<DT>::unpack(x[i], f);
#pragma unroll
            for (int k = 0; k < E; ++k) s[0] += (double)f[k] * (double)f[k];
        }
        row_sums<TPT>(s, scratch);
        r = (float)(1.0 / sqrt(s[0] / (double)n.d + (double)n.eps));
    }
#pragma unroll
    for (int i = 0; i < VMAX; ++i) {
        float f[E], g[E];
        Row<DT>::unpack(x[i], f);
        const int64_t c = (int64_t)(sub + i * TPT) * E;
        if (c >= n.d) break;
#pragma unroll
        for (int k = 0; k < E; ++k) f[k] = LAYER ? ((f[k] - mu) - rest) * r : f[k] * r;
        if (n.gain) {
            load_floats<E>(n.gain, c, n.d, 0.0f, g);
#pragma unroll
            for (int k = 0; k < E; ++k) f[k] *= g[k];
        }
        if (n.bias) {
            load_floats<E>(n.bias, c, n.d, 0.0f, g);
#pragma unroll
            for (int k = 0; k < E; ++k) f[k] += g[k];
        }
        store_vec<DT>(out(n.Y), sub + i * TPT, n.d, Row<DT>::pack(f));
    }
}

// Rows are dealt to the row groups of the grid in turn; a thread meets the same columns in each and adds up their dgain and dbias.  At the end
// a block adds its groups' sums in LDS and leaves one share of both vectors, which the next kernel adds in the order of the blocks: no
// atomics, the same bits every time.
template <sbn_dtype DT, bool LAYER, int TPT, int VMAX> __global__ void __launch_bounds__(TPT < 256 ? 256 : TPT) norm_backward_kernel(const NormArgs n)
{
    constexpr int E = Row<DT>::E;
    constexpr int BLOCK = TPT < 256 ? 256 : TPT;
    constexpr int ROWS = BLOCK / TPT;
    __shared__ float scratch[64];
    __shared__ float shares[ROWS > 1 ? ROWS * TPT * E : 1];
    const int sub = threadIdx.x % TPT, group = threadIdx.x / TPT;
    const float inverse_d = 1.0f / (float)n.d;
    float dgain[VMAX][E], dbias[VMAX][E];
#pragma unroll
    for (int i = 0; i < VMAX; ++i)
#pragma unroll
        for (int k = 0; k < E; ++k) dgain[i][k] = dbias[i][k] = 0.0f;
    for (int64_t t = (int64_t)blockIdx.x * ROWS + group; t < n.tokens; t += (int64_t)gridDim.x * ROWS) {
        const int64_t first = t * n.d;
        const auto row = [&](const void *p) { return static_cast<const void *>(static_cast<const typename Row<DT>::value *>(p) + first); };
        u32x4 x[VMAX], y[VMAX];
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            x[i] = load_vec<DT>(row(n.X), sub + i * TPT, n.d);
            y[i] = load_vec<DT>(row(n.dY), sub + i * TPT, n.d);
        }
        float mu = 0.0f;
        if constexpr (LAYER) {
            float s[1] = {0.0f};
#pragma unroll
            for (int i = 0; i < VMAX; ++i) {
                float f[E];
                Row<DT>::unpack(x[i], f);
#pragma unroll
                for (int k = 0; k < E; ++k) s[0] += f[k];
            }
            row_sums<TPT>(s, scratch);
            mu = s[0] * inverse_d;
        }
        // sums of c, c^2, a and a c, with c = x - mu
        float q[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            float f[E], a[E], g[E];
            const int64_t c = (int64_t)(sub + i * TPT) * E;
            Row<DT>::unpack(x[i], f);
            Row<DT>::unpack(y[i], a);
            if (n.gain && c < n.d) {
                load_floats<E>(n.gain, c, n.d, 0.0f, g);
#pragma unroll
                for (int k = 0; k < E; ++k) a[k] *= g[k];
            }
#pragma unroll
            for (int k = 0; k < E; ++k) {
                if (LAYER) f[k] = c + k < n.d ? f[k] - mu : 0.0f;
                if (LAYER) q[0] += f[k];
                q[1] += f[k] * f[k];
                if (LAYER) q[2] += a[k];
                q[3] += a[k] * f[k];
            }
        }
        float rest = 0.0f, r, of_h, of_a = 0.0f;   // dx = r (a - of_a - h of_h)
        if constexpr (LAYER) {
            row_sums<TPT>(q, scratch);
            rest = q[0] * inverse_d;
            r = 1.0f / sqrtf(fmaxf(q[1] * inverse_d - rest * rest, 0.0f) + n.eps);
            of_a = q[2] * inverse_d;
            of_h = (q[3] - rest * q[2]) * r * inverse_d;
        } else {
            float p[2] = {q[1], q[3]};
            row_sums<TPT>(p, scratch);
            r = 1.0f / sqrtf(p[0] * inverse_d + n.eps);
            of_h = p[1] * r * inverse_d;
        }
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            float f[E], a[E], g[E];
            const int64_t c = (int64_t)(sub + i * TPT) * E;
            if (c >= n.d) break;
            Row<DT>::unpack(x[i], f);
            Row<DT>::unpack(y[i], a);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                f[k] = LAYER ? ((f[k] - mu) - rest) * r : f[k] * r;
                dgain[i][k] += a[k] * f[k];
                dbias[i][k] += a[k];
            }
            if (!n.dX) continue;
            if (n.gain) {
                load_floats<E>(n.gain, c, n.d, 0.0f, g);
#pragma unroll
                for (int k = 0; k < E; ++k) a[k] *= g[k];
            }
#pragma unroll
            for (int k = 0; k < E; ++k) a[k] = r * ((LAYER ? a[k] - of_a : a[k]) - f[k] * of_h);
            if (n.R) {
                Row<DT>::unpack(load_vec<DT>(row(n.R), sub + i * TPT, n.d), g);
#pragma unroll
                for (int k = 0; k < E; ++k) a[k] += g[k];
            }
            store_vec<DT>(static_cast<typename Row<DT>::value *>(n.dX) + first, sub + i * TPT, n.d, Row<DT>::pack(a));
        }
    }
    const auto leave = [&](const float (&sum)[VMAX][E], float *share) {
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            if constexpr (ROWS == 1) {
#pragma unroll
                for (int k = 0; k < E; ++k) {
                    const int64_t c = (int64_t)(sub + i * TPT) * E + k;
                    if (c < n.d) share[c] = sum[i][k];
                }
            } else {
                __syncthreads();
#pragma unroll
                for (int k = 0; k < E; ++k) shares[(group * TPT + sub) * E + k] = sum[i][k];
                __syncthreads();
                for (int j = threadIdx.x; j < TPT * E; j += BLOCK) {
                    const int64_t c = (int64_t)i * TPT * E + j;
                    float s = 0.0f;
#pragma unroll
                    for (int w = 0; w < ROWS; ++w) s += shares[w * TPT * E + j];
                    if (c < n.d) share[c] = s;
                }
            }
        }
    };
    if (n.want_gain) leave(dgain, n.partials + (int64_t)blockIdx.x * n.d);
    if (n.want_bias) leave(dbias, n.partials + (int64_t)(gridDim.x + blockIdx.x) * n.d);
}

// adds the shares of the blocks: 64 columns, sixteen runs of blocks
__global__ void __launch_bounds__(1024) norm_shares_kernel(const float *partials, int blocks, int64_t d, float *dgain, float *dbias)
{
    __shared__ float runs[16][64];
    float *out = blockIdx.y ? dbias : dgain;
    if (!out) return;
    const float *in = partials + (blockIdx.y ? (int64_t)blocks * d : 0);
    const int64_t c = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const int run = threadIdx.x >> 6;
    float s = 0.0f;
    if (c < d) {
#pragma unroll 8
        for (int b = run; b < blocks; b += 16) s += in[b * d + c];
    }
    runs[run][threadIdx.x & 63] = s;
    __syncthreads();
    if (run == 0 && c < d) {
        s = 0.0f;
        for (int k = 0; k < 16; ++k) s += runs[k][threadIdx.x];
        out[c] = s;
    }
}

constexpr int NORM_BACKWARD_BLOCKS = 512;

template <sbn_dtype DT, bool LAYER, int TPT, int VMAX> sbn_status launch_forward(const NormArgs &n, hipStream_t stream)
{
    const int rows = TPT < 256 ? 256 / TPT : 1;
    hipLaunchKernelGGL((norm_kernel<DT, LAYER, TPT, VMAX>), dim3((unsigned)ceil_div(n.tokens, rows)), dim3(TPT < 256 ? 256 : TPT), 0, stream, n);
    return check_launch("norm_kernel");
}

template <sbn_dtype DT, bool LAYER, int TPT, int VMAX> sbn_status launch_backward_rows(const NormArgs &n, float *dgain, float *dbias, hipStream_t stream)
{
    const int rows = TPT < 256 ? 256 / TPT : 1;
    const int blocks = (int)std::min<int64_t>(NORM_BACKWARD_BLOCKS, ceil_div(n.tokens, rows));
    hipLaunchKernelGGL((norm_backward_kernel<DT, LAYER, TPT, VMAX>), dim3(blocks), dim3(TPT < 256 ? 256 : TPT), 0, stream, n);
    if (n.want_gain || n.want_bias)
        hipLaunchKernelGGL(norm_shares_kernel, dim3((unsigned)ceil_div(n.d, 64), 2), dim3(1024), 0, stream, n.partials, blocks, n.d, dgain, dbias);
    return check_launch("norm_backward_kernel");
}

template <sbn_dtype DT, bool LAYER> sbn_status forward_as(const NormArgs &n, hipStream_t stream)
{
    const int64_t vecs = ceil_div(n.d, Row<DT>::E);
    if (vecs <= 64 * 2) return launch_forward<DT, LAYER, 64, 2>(n, stream);
    if (vecs <= 64 * 5) return launch_forward<DT, LAYER, 64, 5>(n, stream);
    if (vecs <= 256 * 4) return launch_forward<DT, LAYER, 256, 4>(n, stream);
    return launch_forward<DT, LAYER, 1024, 16 / Row<DT>::E>(n, stream);   // up to NORM_MAX_D values
}

template <sbn_dtype DT, bool LAYER> sbn_status backward_as(const NormArgs &n, float *dgain, float *dbias, hipStream_t stream)
{
    const int64_t vecs = ceil_div(n.d, Row<DT>::E);
    if (vecs <= 64 * 2) return launch_backward_rows<DT, LAYER, 64, 2>(n, dgain, dbias, stream);
    if (vecs <= 64 * 5) return launch_backward_rows<DT, LAYER, 64, 5>(n, dgain, dbias, stream);
    if (vecs <= 256 * 4) return launch_backward_rows<DT, LAYER, 256, 4>(n, dgain, dbias, stream);
    return launch_backward_rows<DT, LAYER, 1024, 16 / Row<DT>::E>(n, dgain, dbias, stream);
}

}  // namespace

size_t norm_workspace_bytes(int64_t, int64_t d) { return (size_t)2 * NORM_BACKWARD_BLOCKS * d * sizeof(float); }

sbn_status launch_norm(const void *X, const void *residual, sbn_dtype dtype, int64_t tokens, int64_t d, const float *gain, const float *bias, float eps, bool layer,
                       void *Y, void *sum_out, hipStream_t stream)
{
    NormArgs n{};
    n.X = X;
    n.R = residual;
    n.gain = gain;
    n.bias = bias;
    n.Y = Y;
    n.S = sum_out;
    n.tokens = tokens;
    n.d = d;
    n.eps = eps;
    if (dtype == SBN_BF16) return layer ? forward_as<SBN_BF16, true>(n, stream) : forward_as<SBN_BF16, false>(n, stream);
    return layer ? forward_as<SBN_F32, true>(n, stream) : forward_as<SBN_F32, false>(n, stream);
}

sbn_status launch_norm_backward(const void *X, const void *dY, const void *d_residual, sbn_dtype dtype, int64_t tokens, int64_t d, const float *gain, float eps,
                                bool layer, void *dX, float *dgain, float *dbias, void *workspace, hipStream_t stream)
{
    NormArgs n{};
    n.X = X;
    n.R = d_residual;
    n.dY = dY;
    n.gain = gain;
    n.dX = dX;
    n.partials = static_cast<float *>(workspace);
    n.tokens = tokens;
    n.d = d;
    n.eps = eps;
    n.want_gain = dgain != nullptr;
    n.want_bias = dbias != nullptr;
    if (dtype == SBN_BF16) return layer ? backward_as<SBN_BF16, true>(n, dgain, dbias, stream) : backward_as<SBN_BF16, false>(n, dgain, dbias, stream);
    return layer ? backward_as<SBN_F32, true>(n, dgain, dbias, stream) : backward_as<SBN_F32, false>(n, dgain, dbias, stream);
}

}  // namespace sbn
