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
#include <initializer_list>
#include <type_traits>

#include "sbn_internal.hpp"
#include "sbn_rows.hpp"

namespace sbn {

namespace {

struct NormArgs {
    const void *X, *R, *dY;   // R: residual (forward), d_residual (backward), or null
    const float *gain, *bias;
    void *Y, *S, *dX;
    float *gain_shares, *bias_shares;   // [blocks][d] each, of dgain and dbias; null: not wanted
    int64_t tokens, d;
    float eps, inverse_d;
};

constexpr int MOST_SUMS = 4;   // of a team at once

// How a launch deals rows to threads.  A team shares a row, VMAX vectors of it to a thread: 8, 16 or 32 lanes of a wavefront, a wavefront, or the
// wavefronts of a block.
//
// Rows whose length is no whole number of vectors begin anywhere in a vector of memory.  Where all rows of a call do so alike, a thread's vectors are
// those of memory, and a row's first vector begins `shift` values in front of it: accesses off the 16-byte grid took up to twice as long (rows of 500
// bf16 values: 95 us against 40 for 512).  A thread meets the same columns in every row of its team, so a team has one shift, that of its first row.  Launches
// in which a team has several rows have a multiple of 8 blocks: its rows lie a multiple of 8 values apart, and all have that shift.  (But for one block with two
// rows to a team, too few to matter: the second goes by the first one's.)
struct Deal {
    int team_threads, teams;   // threads of a team; teams of a block (one where a team is more than a wavefront)
    int shifts;                // whether vectors lie on memory's grid
    int base;                  // what row 0's shift is
};

// a thread's place in the row that its team is at
template <sbn_dtype DT> struct Place {
    static constexpr int E = Row<DT>::E;
    typedef typename Row<DT>::value value;
    int64_t first, total, d;   // of the row, in values of the tensor; values of the tensor, of a row
    int sub, team_threads, shift;

    // the column of vector i's first value: less than 0 for a vector that begins in front of the row
    __device__ __forceinline__ int64_t column(int i) const { return (int64_t)(sub + i * team_threads) * E - shift; }
    __device__ __forceinline__ bool whole(int i) const { return column(i) >= 0 && column(i) + E <= d; }
    __device__ __forceinline__ bool none(int i) const { return column(i) + E <= 0 || column(i) >= d; }
    __device__ __forceinline__ bool inside(int i, int k) const { return column(i) + k >= 0 && column(i) + k < d; }

    // vector i, which is read once.  At a row's ends it comes with values of the rows before and behind (which may be written meanwhile) until only()
    // takes them off: nothing waits for a load before the others are under way
    __device__ __forceinline__ u32x4 load(const void *rows, int i) const
    {
        const int64_t at = first + column(i);
        const value *p = static_cast<const value *>(rows) + at;
        u32x4 v = {0, 0, 0, 0};
        if (none(i)) return v;
        if (at >= 0 && at + E <= total) return Row<DT>::template load<true>(p, 0);
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (inside(i, k)) Row<DT>::set(v, k, p[k]);
        return v;
    }
    __device__ __forceinline__ void only(u32x4 &v, int i) const
    {
        if (whole(i)) return;
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (!inside(i, k)) Row<DT>::clear(v, k);
    }
    __device__ __forceinline__ void store(void *rows, int i, u32x4 v) const
    {
        value *p = static_cast<value *>(rows) + first + column(i);
        if (whole(i))
            Row<DT>::store(p, 0, v);
        else if (!none(i)) {
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (inside(i, k)) p[k] = Row<DT>::get(v, k);
        }
    }
    // fp32 values that go with the columns of vector i
    __device__ __forceinline__ void load_columns(const float *p, float other, int i, float (&g)[E]) const
    {
#pragma unroll
        for (int k = 0; k < E; ++k) g[k] = other;
        if (!p || none(i)) return;
        if (whole(i))
            load_floats<E>(p, column(i), d, other, g);
        else {
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (inside(i, k)) g[k] = p[column(i) + k];
        }
    }
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

template <sbn_dtype DT> __device__ __forceinline__ Place<DT> place_of(const NormArgs &n, const Deal &deal)
{
    const int team = threadIdx.x / deal.team_threads;
    Place<DT> at;
    at.sub = threadIdx.x - team * deal.team_threads;
    at.team_threads = deal.team_threads;
    at.total = n.tokens * n.d;
    at.d = n.d;
    at.first = ((int64_t)blockIdx.x * deal.teams + team) * n.d;
    at.shift = deal.shifts ? (int)((at.first + deal.base) & (Row<DT>::E - 1)) : 0;
    return at;
}

template <sbn_dtype DT, int VMAX> __device__ __forceinline__ void load_columns(float (&g)[VMAX][Row<DT>::E], const float *p, float other, const Place<DT> &at)
{
#pragma unroll
    for (int i = 0; i < VMAX; ++i) at.load_columns(p, other, i, g[i]);
}

// x less mu, zeros outside the row
template <sbn_dtype DT> __device__ __forceinline__ void centre(float (&f)[Row<DT>::E], float mu, const Place<DT> &at, int i)
{
#pragma unroll
    for (int k = 0; k < Row<DT>::E; ++k) f[k] -= mu;
    if (!at.whole(i)) {
#pragma unroll
        for (int k = 0; k < Row<DT>::E; ++k)
            if (!at.inside(i, k)) f[k] = 0.0f;
    }
}

// 1 / sqrt(variance + eps); a variance that rounding took below 0 is 0, and one that is no number stays that
__device__ __forceinline__ float factor_of(float variance, float eps) { return 1.0f / sqrtf((variance < 0.0f ? 0.0f : variance) + eps); }

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
    constexpr bool KEEP = VMAX * E <= 8;   // gain and bias stay in registers
    Place<DT> at = place_of<DT>(n, deal);
    int turn = 0;
    float gain[VMAX][E], bias[VMAX][E];
    if (KEEP) {
        load_columns<DT>(gain, n.gain, 1.0f, at);
        load_columns<DT>(bias, n.bias, 0.0f, at);
    }
    for (; at.first < at.total; at.first += (int64_t)gridDim.x * deal.teams * n.d) {
        u32x4 x[VMAX];
#pragma unroll
        for (int i = 0; i < VMAX; ++i) x[i] = at.load(n.X, i);
        u32x4 res[VMAX];
        if (n.R) {
#pragma unroll
            for (int i = 0; i < VMAX; ++i) res[i] = at.load(n.R, i);
        }
#pragma unroll
        for (int i = 0; i < VMAX; ++i) at.only(x[i], i);
        if (n.R) {
#pragma unroll
            for (int i = 0; i < VMAX; ++i) {
                float a[E], b[E];
                at.only(res[i], i);
                Row<DT>::unpack(x[i], a);
                Row<DT>::unpack(res[i], b);
#pragma unroll
                for (int k = 0; k < E; ++k) a[k] += b[k];
                x[i] = Row<DT>::pack(a);
                at.store(n.S, i, x[i]);
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
                centre<DT>(f, mu, at, i);
#pragma unroll
                for (int k = 0; k < E; ++k) {
                    q[0] += f[k];
                    q[1] += f[k] * f[k];
                }
            }
            team_sums<L>(q, deal, fscratch, turn);
            rest = q[0] * n.inverse_d;
            r = factor_of(q[1] * n.inverse_d - rest * rest, n.eps);
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
        if (!KEEP) {
            load_columns<DT>(gain, n.gain, 1.0f, at);
            load_columns<DT>(bias, n.bias, 0.0f, at);
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
            at.store(n.Y, i, Row<DT>::pack(f));
        }
    }
}

// A thread meets the same columns in every row of its team and adds up their dgain and dbias.  At the end a block adds its teams' sums in LDS and
// leaves one share of both vectors, which the next kernel adds in the order of the blocks: no atomics, the same bits every time.
// Bound by memory: 16384 RMS rows of 2560 bf16 values with d_residual move 336 MB in 57 to 64 us, 5.3 to 5.9 TB/s (a call, with the shares, 62; of the layer form,
// with both shares, 73, and 72 without d_residual).  Three blocks of five wavefronts to each of the 256 processors: as many on all of them (819 blocks: 88 us), and
// no more (four: 72) nor fewer (two: 69).  At most 96 registers, so that five wavefronts find room on a SIMD: with 106 the layer form took 102 us for 67 (without a
// residual, the kernel alone).  For that the layer form of bf16 rows keeps two to four registers in memory, and two instances of the RMS form and of longer rows one
// or two; fp32 rows of more than 2560 values in the layer form ten.
template <sbn_dtype DT, bool LAYER, int L, int VMAX>
__global__ void __launch_bounds__(most_threads(L)) __attribute__((amdgpu_waves_per_eu(VMAX * Row<DT>::E <= 8 ? 5 : 4))) norm_backward_kernel(const NormArgs n, const Deal deal)
{
    constexpr int E = Row<DT>::E;
    __shared__ float scratch[2 * 16 * MOST_SUMS];
    __shared__ float shares[256 * E];   // of the threads of several teams
    constexpr bool KEEP = VMAX * E <= 8;   // gain stays in registers, and d_residual comes with the others
    Place<DT> at = place_of<DT>(n, deal);
    int turn = 0;
    float dgain[VMAX][E], dbias[VMAX][E], gain[VMAX][E];
#pragma unroll
    for (int i = 0; i < VMAX; ++i)
#pragma unroll
        for (int k = 0; k < E; ++k) dgain[i][k] = dbias[i][k] = 0.0f;
    if (KEEP) load_columns<DT>(gain, n.gain, 1.0f, at);
    for (; at.first < at.total; at.first += (int64_t)gridDim.x * deal.teams * n.d) {
        u32x4 x[VMAX], y[VMAX], res[VMAX];
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            x[i] = at.load(n.X, i);
            y[i] = at.load(n.dY, i);
        }
        if (KEEP && n.R) {
#pragma unroll
            for (int i = 0; i < VMAX; ++i) res[i] = at.load(n.R, i);
        }
        if (!KEEP) load_columns<DT>(gain, n.gain, 1.0f, at);
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            at.only(x[i], i);
            at.only(y[i], i);
        }
        const float mu = LAYER ? first_mean<DT, L>(x, n, deal, scratch, turn) : 0.0f;
        // sums of c^2 and a c (layer form: of c and a too), with c = x - mu
        float q[LAYER ? 4 : 2] = {};
#pragma unroll
        for (int i = 0; i < VMAX; ++i) {
            float f[E], a[E];
            Row<DT>::unpack(x[i], f);
            Row<DT>::unpack(y[i], a);
            if (LAYER) centre<DT>(f, mu, at, i);
#pragma unroll
            for (int k = 0; k < E; ++k) {
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
        const float r = factor_of(q[0] * n.inverse_d - rest * rest, n.eps);
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
                Row<DT>::unpack(KEEP ? res[i] : at.load(n.R, i), f);
#pragma unroll
                for (int k = 0; k < E; ++k) a[k] += f[k];
            }
            at.store(n.dX, i, Row<DT>::pack(a));
        }
    }
    const auto leave = [&](const float (&sum)[VMAX][E], float *share) {
        if (deal.teams == 1) {
#pragma unroll
            for (int i = 0; i < VMAX; ++i) {
                if (at.whole(i))
                    store_unit<SBN_F32, E>(share + at.column(i), 0, E, sum[i]);
                else {
#pragma unroll
                    for (int k = 0; k < E; ++k)
                        if (at.inside(i, k)) share[at.column(i) + k] = sum[i][k];
                }
            }
            return;
        }
        // several teams: one vector to a thread, 256 threads
        const int wide = deal.team_threads * E, team = threadIdx.x / deal.team_threads;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (at.inside(0, k)) shares[team * wide + at.column(0) + k] = sum[0][k];
        __syncthreads();
        for (int c = threadIdx.x; c < n.d; c += 256) {
            float s = 0.0f;
            for (int w = 0; w < deal.teams; ++w) s += shares[w * wide + c];
            share[c] = s;
        }
    };
    if (n.gain_shares) leave(dgain, n.gain_shares + (int64_t)blockIdx.x * n.d);
    if (n.bias_shares) leave(dbias, n.bias_shares + (int64_t)blockIdx.x * n.d);
}

// adds the shares of the blocks: 32 columns, 32 runs of blocks
__global__ void __launch_bounds__(1024) norm_shares_kernel(const float *gain_shares, const float *bias_shares, int blocks, int64_t d, float *dgain, float *dbias)
{
    __shared__ float runs[32][33];
    float *out = blockIdx.y ? dbias : dgain;
    if (!out) return;
    const float *in = blockIdx.y ? bias_shares : gain_shares;
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

constexpr int PROCESSORS = 256;
// wavefronts of a processor that stay: as many as its registers hold of the kernel, where that was fastest (see there)
constexpr int FORWARD_WAVES = 25, FORWARD_WAVES_LONG = 20, BACKWARD_WAVES = 16;

// blocks of `waves` wavefronts each that stay until all rows are done, the same number for every processor
int64_t staying_blocks(int waves, int most) { return PROCESSORS * std::max(1, most / waves); }

// rows of a team that one block goes through in the backward rather than leave shares to a second launch (two rows of 2560 bf16 values: 5.4 us against 6.5, three
// 7.0 against 6.5)
constexpr int ONE_BLOCK_ROWS = 2;

// vectors that a row of d values reaches over: rows that are no whole number of them may begin in the middle of one
int64_t vectors_of(int64_t d, int values) { return d % values ? ceil_div(d + values - 1, values) : d / values; }

// Vectors of a thread where a team is more than a wavefront: eight values, or sixteen in rows of more than 2560.  Large blocks fill a processor unevenly
// and wait for each other: rows of 8192 bf16 values 76 us by 16 wavefronts with eight, 67 by eight with sixteen; of 4096 57 by eight, 50 by four; of 2560
// 36 by five and 38 by three.
int vectors_of_thread(int64_t vecs, int values) { return vecs <= 320 * 8 / values ? 8 / values : 16 / values; }

// wavefronts of a block: four with a team or several each, or those of one team
int block_waves(int64_t d, int values)
{
    const int64_t vecs = vectors_of(d, values);
    return vecs <= 64 ? 4 : (int)std::min<int64_t>(16, ceil_div(vecs, 64 * vectors_of_thread(vecs, values)));
}

// The most that a call's shares of one vector hold, in values of either type: staying_blocks() leaves BACKWARD_WAVES wavefronts to a processor (or one block of as
// many), 64 lanes of 8 values each, or of 16 in rows whose vectors reach past 2560 values.  No more blocks than wavefronts, nor than rows.  Never falls as rows or
// values are added, as blocks times values do (1024 blocks of 512 values, 512 of 1001, 768 of 2560): what was made for a program's longest rows serves shorter ones.
int64_t share_values(int64_t tokens, int64_t d)
{
    const int64_t waves = PROCESSORS * BACKWARD_WAVES, of_waves = waves * 64 * (d + Row<SBN_BF16>::E - 1 > 2560 ? 16 : 8);
    return std::min(std::min(waves, tokens) * d, of_waves);
}

// Calls f with the lanes of a team that is part of a wavefront (64: whole wavefronts), the vectors of a thread, the deal, the wavefronts of a block and
// the blocks that give every row a team of its own.  rows: the tensors of the call (or null).
template <sbn_dtype DT, class F> sbn_status dealt(const NormArgs &n, std::initializer_list<const void *> rows, F &&f)
{
    using std::integral_constant;
    constexpr int E = Row<DT>::E;
    const int64_t vecs = vectors_of(n.d, E);
    const auto base = [](const void *p) { return (int)(reinterpret_cast<uintptr_t>(p) / sizeof(typename Row<DT>::value) % E); };
    bool alike = vecs <= 1024 * 16 / E;   // (the longest rows have no room for a vector more)
    for (const void *p : rows) alike = alike && (!p || base(p) == base(n.X));
    // where row 0 lies off the grid, so do rows of whole vectors: they have no room for a shift
    alike = alike && (n.d % E != 0 || base(n.X) == 0);
    const int waves = block_waves(n.d, E);
    const auto with = [&](auto L, auto VMAX) {
        // part of a wavefront, or the wavefronts of the block; more than a vector to a thread only in the latter
        const int team_threads = decltype(L)::value < 64 ? decltype(L)::value : vecs <= 64 ? 64 : 64 * waves;
        const Deal deal{team_threads, 64 * waves / team_threads, alike, base(n.X)};
        return f(L, VMAX, deal, waves, ceil_div(n.tokens, (int64_t)deal.teams));
    };
    const integral_constant<int, 1> one{};
    if (vecs <= 8) return with(integral_constant<int, 8>{}, one);
    if (vecs <= 16) return with(integral_constant<int, 16>{}, one);
    if (vecs <= 32) return with(integral_constant<int, 32>{}, one);
    const integral_constant<int, 64> wave{};
    if (vecs <= 64) return with(wave, one);
    if (vectors_of_thread(vecs, E) == 8 / E) return with(wave, integral_constant<int, 8 / E>{});
    return with(wave, integral_constant<int, 16 / E>{});   // up to NORM_MAX_D values
}

template <sbn_dtype DT, bool LAYER> sbn_status forward_as(const NormArgs &n, hipStream_t stream)
{
    return dealt<DT>(n, {n.R, n.S, n.Y}, [&](auto L, auto VMAX, const Deal &deal, int waves, int64_t all) {
        const int64_t blocks = std::min(all, staying_blocks(waves, decltype(VMAX)::value * Row<DT>::E > 8 ? FORWARD_WAVES_LONG : FORWARD_WAVES));
        hipLaunchKernelGGL((norm_kernel<DT, LAYER, decltype(L)::value, decltype(VMAX)::value>), dim3((unsigned)blocks), dim3(64 * waves), 0, stream, n, deal);
        return check_launch("norm_kernel");
    });
}

template <sbn_dtype DT, bool LAYER> sbn_status backward_as(NormArgs &n, float *dgain, float *dbias, float *workspace, hipStream_t stream)
{
    return dealt<DT>(n, {n.dY, n.R, n.dX}, [&](auto L, auto VMAX, const Deal &deal, int waves, int64_t all) {
        // where there are few rows, two blocks to a processor, or four rows to a team: shares cost as well (1531 rows of 1001: 13 + 8 us by 766 blocks, 12 + 4 by 512);
        // a multiple of 8 unless every team has one row, so that a team's rows begin alike (5000 rows of 777 bf16 values: 17.6 us by 1256 blocks, 18.2 by 1250; 2500 of 1001,
        // by 632 and 625: 13.6 and 13.9)
        const int64_t few = std::max<int64_t>(2 * PROCESSORS, ceil_div(ceil_div(all, 4), 8) * 8);
        const int blocks = all <= ONE_BLOCK_ROWS ? 1 : (int)std::min({all, staying_blocks(waves, BACKWARD_WAVES), few});
        // one block's shares are the sums
        n.gain_shares = !dgain ? nullptr : blocks == 1 ? dgain : workspace;
        n.bias_shares = !dbias ? nullptr : blocks == 1 ? dbias : workspace + blocks * n.d;
        hipLaunchKernelGGL((norm_backward_kernel<DT, LAYER, decltype(L)::value, decltype(VMAX)::value>), dim3(blocks), dim3(64 * waves), 0, stream, n, deal);
        if ((dgain || dbias) && blocks > 1)
            hipLaunchKernelGGL(norm_shares_kernel, dim3((unsigned)ceil_div(n.d, 32), 2), dim3(1024), 0, stream, n.gain_shares, n.bias_shares, blocks, n.d, dgain, dbias);
        return check_launch("norm_backward_kernel");
    });
}

}  // namespace

size_t norm_workspace_bytes(int64_t tokens, int64_t d) { return (size_t)2 * share_values(tokens, d) * sizeof(float); }

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
    n.tokens = tokens;
    n.d = d;
    n.eps = eps;
    n.inverse_d = 1.0f / (float)d;
    float *const ws = static_cast<float *>(workspace);
    if (dtype == SBN_BF16) return layer ? backward_as<SBN_BF16, true>(n, dgain, dbias, ws, stream) : backward_as<SBN_BF16, false>(n, dgain, dbias, ws, stream);
    return layer ? backward_as<SBN_F32, true>(n, dgain, dbias, ws, stream) : backward_as<SBN_F32, false>(n, dgain, dbias, ws, stream);
}

}  // namespace sbn
