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
#include <type_traits>

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
    float eps, inverse_d;
    int want_gain, want_bias;
};

constexpr int MOST_SUMS = 4;   // of a team at once

// How a launch deals rows to threads.  A team shares a row, one vector of it to a thread (VMAX vectors where a row is too long for that): 8, 16 or 32
// lanes of a wavefront, a wavefront, or the wavefronts of a block.
struct Deal {
    int team_threads, teams;   // threads of a team; teams of a block (one where a team is more than a wavefront)
};

// Sums over a team, N of them at once.  A wavefront adds by DPP (the last lane has the sum), the wavefronts of a team by LDS: two pieces of scratch
// in turn, so that one barrier is enough (whoever writes a piece again has passed the barrier of the other, which its readers reach after reading).
template <int L> __device__ __forceinline__ float team_sum_in_wave(float x)
{
    if constexpr (L == 64) {
        const auto step = [](float v, auto ctrl, auto rows) {
            return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
        };
        using std::integral_constant;
        x = step(x, integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});   // row_shr: 1, 2, 4, 8
        x = step(x, integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
        x = step(x, integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
        x = step(x, integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
        x = step(x, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});   // row_bcast: 15, 31
        x = step(x, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
        return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), 63));
    } else {
#pragma unroll
        for (int off = L / 2; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
        return x;
    }
}
template <int L> __device__ __forceinline__ double team_sum_in_wave(double x)
{
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
    return x;
}

template <int L, int N, class F> __device__ __forceinline__ void team_sums(F (&s)[N], const Deal &deal, F *scratch, int &turn)
{
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = team_sum_in_wave<L>(s[k]);
    if (L < 64 || deal.team_threads == 64) return;
    F *piece = scratch + (turn ^= 1) * (16 * MOST_SUMS);
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) piece[(threadIdx.x >> 6) * N + k] = s[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = piece[k];
    for (int w = 1; w < deal.team_threads / 64; ++w) {
#pragma unroll
        for (int k = 0; k < N; ++k) s[k] += piece[w * N + k];
    }
}

// vectors of a row; they are read once
template <sbn_dtype DT, int VMAX> __device__ __forceinline__ void load_row(u32x4 (&x)[VMAX], const void *rows, int64_t t, const NormArgs &n, const Deal &deal, int sub)
{
#pragma unroll
    for (int i = 0; i < VMAX; ++i) x[i] = load_vec<DT, true>(static_cast<const typename Row<DT>::value *>(rows) + t * n.d, sub + i * deal.team_threads, n.d);
}
template <sbn_dtype DT> __device__ __forceinline__ void store_row(void *rows, int64_t t, const NormArgs &n, const Deal &deal, int sub, int i, u32x4 v)
{
    store_vec<DT>(static_cast<typename Row<DT>::value *>(rows) + t * n.d, sub + i * deal.team_threads, n.d, v);
}

// column factors (or terms) of a thread's vectors
template <int E, int VMAX> __device__ __forceinline__ void load_columns(float (&g)[VMAX][E], const float *p, float none, const NormArgs &n, const Deal &deal, int sub)
{
#pragma unroll
    for (int i = 0; i < VMAX; ++i) {
#pragma unroll
        for (int k = 0; k < E; ++k) g[i][k] = none;
        const int64_t c = (int64_t)(sub + i * deal.team_threads) * E;
        if (p && c < n.d) load_floats<E>(p, c, n.d, none, g[i]);
    }
}

// the mean of a row by its first sum
template <sbn_dtype DT, int L, int VMAX> __device__ __forceinline__ float first_mean(const u32x4 (&x)[VMAX], const NormArgs &n, const Deal &deal, float *scratch, int &turn)
{
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < VMAX; ++i) {
        float f[Row<DT>::E];
        Row<DT>::unpack(x[i], f);
#pragma unroll
        for (int k = 0; k < Row<DT>::E; ++k) s[0] += f[k];
    }
    team_sums<L>(s, deal, scratch, turn);
    return s[0] * n.inverse_d;
}

// threads of a block at most
constexpr int most_threads(int L) { return L < 64 ? 256 : 1024; }

// Bound by memory: 16384 layer-form rows of 2560 bf16 values with a residual move 336 MB in 57 us, 5.9 TB/s, where a copy that moves as much takes 62.
// Blocks that stay and go from row to row read gain and bias once; some 25 wavefronts to a processor were fastest (five blocks of five: 57 us; four
// 60, six 69, a block for each row 71), with nontemporal loads of what is read once (69 without, three blocks).  Two or four rows at a time with shared
// barriers were slower or no faster.
template <sbn_dtype DT, bool LAYER, int L, int VMAX> __global__ void __launch_bounds__(most_threads(L)) norm_kernel(const NormArgs n, const Deal deal)
{
    constexpr int E = Row<DT>::E;
    __shared__ double scratch[2 * 16 * MOST_SUMS];
    float *const fscratch = reinterpret_cast<float *>(scratch);
    const int team = threadIdx.x / deal.team_threads, sub = threadIdx.x - team * deal.team_threads;
    int turn = 0;
    float gain[VMAX][E], bias[VMAX][E];
    if (VMAX == 1) {
        load_columns<E, VMAX>(gain, n.gain, 1.0f, n, deal, sub);
        load_columns<E, VMAX>(bias, n.bias, 0.0f, n, deal, sub);
    }
    for (int64_t t = (int64_t)blockIdx.x * deal.teams + team; t < n.tokens; t += (int64_t)gridDim.x * deal.teams) {
        u32x4 x[VMAX];
        load_row<DT>(x, n.X, t, n, deal, sub);
        if (n.R) {
            u32x4 r[VMAX];
            load_row<DT>(r, n.R, t, n, deal, sub);
#pragma unroll
            for (int i = 0; i < VMAX; ++i) {
                float a[E], b[E];
                Row<DT>::unpack(x[i], a);
                Row<DT>::unpack(r[i], b);
#pragma unroll
                for (int k = 0; k < E; ++k) a[k] += b[k];
                x[i] = Row<DT>::pack(a);
                store_row<DT>(n.S, t, n, deal, sub, i, x[i]);
            }
        }
        float mu = 0.0f, rest = 0.0f, r;
        if constexpr (LAYER) {
            mu = first_mean<DT, L>(x, n, deal, fscratch, turn);
            float q[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < VMAX; ++i) {
                float f[E];
                Row<DT>::unpack(x[i], f);
#pragma unroll
                for (int k = 0; k < E; ++k) {
                    const float c = (sub + i * deal.team_threads) * E + k < n.d ? f[k] - mu : 0.0f;
                    q[0] += c;
                    q[1] += c * c;
                }
            }
            team_sums<L>(q, deal, fscratch, turn);
            rest = q[0] * n.inverse_d;
            r = 1.0f / sqrtf(fmaxf(q[1] * n.inverse_d - rest * rest, 0.0f) + n.eps);
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
            team_sums<L>(s, deal, scratch, turn);
            r = (float)(1.0 / sqrt(s[0] / (double)n.d + (double)n.eps));
        }
        if (VMAX > 1) {
            load_columns<E, VMAX>(gain, n.gain, 1.0f, n, deal, sub);
            load_columns<E, VMAX>(bias, n.bias, 0.0f, n, deal, sub);
        }
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            float f[E];
            Row<DT>::unpack(x[i], f);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                f[k] = LAYER ? ((f[k] - mu) - rest) * r : f[k] * r;
                f[k] *= gain[i][k];
                if (n.bias) f[k] += bias[i][k];
            }
            store_row<DT>(n.Y, t, n, deal, sub, i, Row<DT>::pack(f));
        }
    }
}

// A thread meets the same columns in every row of its team and adds up their dgain and dbias.  At the end a block adds its teams' sums in LDS and
// leaves one share of both vectors, which the next kernel adds in the order of the blocks: no atomics, the same bits every time.
// Bound by memory: 16384 RMS rows of 2560 bf16 values with d_residual move 336 MB in 61 us, 5.5 TB/s.  Three blocks of five wavefronts to each of the 256
// processors: as many on all of them (819 blocks: 88 us), and no more (four: 72) nor fewer (two: 69).
template <sbn_dtype DT, bool LAYER, int L, int VMAX> __global__ void __launch_bounds__(most_threads(L)) norm_backward_kernel(const NormArgs n, const Deal deal)
{
    constexpr int E = Row<DT>::E;
    __shared__ float scratch[2 * 16 * MOST_SUMS];
    __shared__ float shares[256 * E];   // of the threads of several teams
    const int team = threadIdx.x / deal.team_threads, sub = threadIdx.x - team * deal.team_threads;
    int turn = 0;
    float dgain[VMAX][E], dbias[VMAX][E], gain[VMAX][E];
#pragma unroll
    for (int i = 0; i < VMAX; ++i)
#pragma unroll
        for (int k = 0; k < E; ++k) dgain[i][k] = dbias[i][k] = 0.0f;
    if (VMAX == 1) load_columns<E, VMAX>(gain, n.gain, 1.0f, n, deal, sub);
    for (int64_t t = (int64_t)blockIdx.x * deal.teams + team; t < n.tokens; t += (int64_t)gridDim.x * deal.teams) {
        u32x4 x[VMAX], y[VMAX], res[VMAX];
        load_row<DT>(x, n.X, t, n, deal, sub);
        load_row<DT>(y, n.dY, t, n, deal, sub);
        if (VMAX == 1 && n.R) load_row<DT>(res, n.R, t, n, deal, sub);   // (with more vectors there are no registers for it)
        if (VMAX > 1) load_columns<E, VMAX>(gain, n.gain, 1.0f, n, deal, sub);
        const float mu = LAYER ? first_mean<DT, L>(x, n, deal, scratch, turn) : 0.0f;
        // sums of c^2 and a c (layer form: of c and a too), with c = x - mu
        float q[LAYER ? 4 : 2] = {};
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            float f[E], a[E];
            Row<DT>::unpack(x[i], f);
            Row<DT>::unpack(y[i], a);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                if (LAYER) f[k] = (sub + i * deal.team_threads) * E + k < n.d ? f[k] - mu : 0.0f;
                a[k] *= gain[i][k];
                q[0] += f[k] * f[k];
                q[1] += a[k] * f[k];
                if constexpr (LAYER) {
                    q[2] += f[k];
                    q[3] += a[k];
                }
            }
        }
        team_sums<L>(q, deal, scratch, turn);
        float rest = 0.0f, of_a = 0.0f;   // dx = r (a - of_a - h of_h)
        if constexpr (LAYER) {
            rest = q[2] * n.inverse_d;
            of_a = q[3] * n.inverse_d;
            q[1] -= rest * q[3];
        }
        const float r = 1.0f / sqrtf(fmaxf(q[0] * n.inverse_d - rest * rest, 0.0f) + n.eps);
        const float of_h = q[1] * r * n.inverse_d;
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            float f[E], a[E];
            Row<DT>::unpack(x[i], f);
            Row<DT>::unpack(y[i], a);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                f[k] = LAYER ? ((f[k] - mu) - rest) * r : f[k] * r;
                dgain[i][k] += a[k] * f[k];
                dbias[i][k] += a[k];
                a[k] *= gain[i][k];
                a[k] = r * ((LAYER ? a[k] - of_a : a[k]) - f[k] * of_h);
            }
            if (!n.dX) continue;
            if (n.R) {
                Row<DT>::unpack(VMAX == 1 ? res[i] : load_vec<DT>(static_cast<const typename Row<DT>::value *>(n.R) + t * n.d, sub + i * deal.team_threads, n.d), f);
#pragma unroll
                for (int k = 0; k < E; ++k) a[k] += f[k];
            }
            store_row<DT>(n.dX, t, n, deal, sub, i, Row<DT>::pack(a));
        }
    }
    const auto leave = [&](const float (&sum)[VMAX][E], float *share) {
        if (deal.teams == 1) {
#pragma unroll
            for (int i = 0; i < VMAX; ++i) store_unit<SBN_F32, E>(share, sub + i * deal.team_threads, n.d, sum[i]);
            return;
        }
        // several teams: one vector to a thread, 256 threads
        __syncthreads();
#pragma unroll
        for (int k = 0; k < E; ++k) shares[threadIdx.x * E + k] = sum[0][k];
        __syncthreads();
        const int wide = deal.team_threads * E;
        for (int c = threadIdx.x; c < min((int64_t)wide, n.d); c += 256) {
            float s = 0.0f;
            for (int w = 0; w < deal.teams; ++w) s += shares[w * wide + c];
            share[c] = s;
        }
    };
    if (n.want_gain) leave(dgain, n.partials + (int64_t)blockIdx.x * n.d);
    if (n.want_bias) leave(dbias, n.partials + (int64_t)(gridDim.x + blockIdx.x) * n.d);
}

// adds the shares of the blocks: 32 columns, 32 runs of blocks
__global__ void __launch_bounds__(1024) norm_shares_kernel(const float *partials, int blocks, int64_t d, float *dgain, float *dbias)
{
    __shared__ float runs[32][33];
    float *out = blockIdx.y ? dbias : dgain;
    if (!out) return;
    const float *in = partials + (blockIdx.y ? (int64_t)blocks * d : 0);
    const int64_t c = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
    const int run = threadIdx.x >> 5;
    float s = 0.0f;
    if (c < d) {
#pragma unroll 8
        for (int b = run; b < blocks; b += 32) s += in[b * d + c];
    }
    runs[run][threadIdx.x & 31] = s;
    __syncthreads();
    if (run == 0 && c < d) {
        s = 0.0f;
#pragma unroll
        for (int k = 0; k < 32; ++k) s += runs[k][threadIdx.x];
        out[c] = s;
    }
}

constexpr int FORWARD_WAVES = 25, BACKWARD_WAVES = 15;   // of a processor, by the kernels' measurements
constexpr int PROCESSORS = 256;

// blocks of `waves` wavefronts each that stay until all rows are done, the same number for every processor
int64_t staying_blocks(int waves, int most) { return PROCESSORS * std::max(1, most / waves); }

// wavefronts of a block: four with a team or several each, or those of one team
int block_waves(int64_t d, int values)
{
    const int64_t vecs = ceil_div(d, values);
    return vecs <= 64 ? 4 : (int)std::min<int64_t>(16, ceil_div(vecs, 64));
}

// blocks of the backward at most, in either type: each leaves its shares
int64_t most_shares(int64_t d)
{
    return std::max(staying_blocks(block_waves(d, Row<SBN_BF16>::E), BACKWARD_WAVES), staying_blocks(block_waves(d, Row<SBN_F32>::E), BACKWARD_WAVES));
}

// calls f with the lanes of a team that is part of a wavefront (64: whole wavefronts), the vectors of a thread, the deal, the wavefronts of a block and
// the blocks that give every row a team of its own
template <sbn_dtype DT, class F> sbn_status dealt(int64_t tokens, int64_t d, F &&f)
{
    using std::integral_constant;
    const auto with = [&](auto L, auto VMAX, int team_threads) {
        const int waves = block_waves(d, Row<DT>::E);
        const Deal deal{team_threads, 64 * waves / team_threads};
        return f(L, VMAX, deal, waves, ceil_div(tokens, (int64_t)deal.teams));
    };
    const int64_t vecs = ceil_div(d, Row<DT>::E);
    const integral_constant<int, 1> one{};
    if (vecs <= 8) return with(integral_constant<int, 8>{}, one, 8);
    if (vecs <= 16) return with(integral_constant<int, 16>{}, one, 16);
    if (vecs <= 32) return with(integral_constant<int, 32>{}, one, 32);
    const integral_constant<int, 64> wave{};
    if (vecs <= 1024) return with(wave, one, 64 * (int)ceil_div(vecs, 64));
    return with(wave, integral_constant<int, 16 / Row<DT>::E>{}, 1024);   // up to NORM_MAX_D values
}

template <sbn_dtype DT, bool LAYER> sbn_status forward_as(const NormArgs &n, hipStream_t stream)
{
    return dealt<DT>(n.tokens, n.d, [&](auto L, auto VMAX, const Deal &deal, int waves, int64_t all) {
        const int64_t blocks = std::min(all, staying_blocks(waves, FORWARD_WAVES));
        hipLaunchKernelGGL((norm_kernel<DT, LAYER, decltype(L)::value, decltype(VMAX)::value>), dim3((unsigned)blocks), dim3(64 * waves), 0, stream, n, deal);
        return check_launch("norm_kernel");
    });
}

template <sbn_dtype DT, bool LAYER> sbn_status backward_as(const NormArgs &n, float *dgain, float *dbias, hipStream_t stream)
{
    return dealt<DT>(n.tokens, n.d, [&](auto L, auto VMAX, const Deal &deal, int waves, int64_t all) {
        const int blocks = (int)std::min(all, staying_blocks(waves, BACKWARD_WAVES));
        hipLaunchKernelGGL((norm_backward_kernel<DT, LAYER, decltype(L)::value, decltype(VMAX)::value>), dim3(blocks), dim3(64 * waves), 0, stream, n, deal);
        if (dgain || dbias) hipLaunchKernelGGL(norm_shares_kernel, dim3((unsigned)ceil_div(n.d, 32), 2), dim3(1024), 0, stream, n.partials, blocks, n.d, dgain, dbias);
        return check_launch("norm_backward_kernel");
    });
}

}  // namespace

size_t norm_workspace_bytes(int64_t, int64_t d) { return (size_t)2 * most_shares(d) * d * sizeof(float); }

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
    n.inverse_d = 1.0f / (float)d;
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
    n.inverse_d = 1.0f / (float)d;
    n.want_gain = dgain != nullptr;
    n.want_bias = dbias != nullptr;
    if (dtype == SBN_BF16) return layer ? backward_as<SBN_BF16, true>(n, dgain, dbias, stream) : backward_as<SBN_BF16, false>(n, dgain, dbias, stream);
    return layer ? backward_as<SBN_F32, true>(n, dgain, dbias, stream) : backward_as<SBN_F32, false>(n, dgain, dbias, stream);
}

}  // namespace sbn
