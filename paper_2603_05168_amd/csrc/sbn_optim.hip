// The optimizer step over many tensors: the norm of all gradients, and AdamW with moments in fp32 or in 8 bits.
//
//   m' = beta1 m + (1 - beta1) g,   v' = beta2 v + ((1 - beta2) g) g          (g scaled first where a factor is given)
//   p' = p (1 - lr decay) - (lr / (1 - beta1^t)) m' / (sqrt(v' / (1 - beta2^t)) + eps)
// Bound by memory: bf16 weights and gradients with fp32 moments move 22 bytes per weight, with moments in 8 bits 10.1.
//
// Moments in 8 bits: 32 consecutive values share an exponent e (a byte, as of fp32), that of their largest magnitude.  A code is the upper part of
// the fp32 pattern, exponent and three bits of mantissa, counted from the pattern `below` binades under e: rounding is an addition below the cut,
// and codes and values are a shift and a sum apart.  m: a sign and seven bits (15 binades), v: eight bits (31 binades).  Code 0 is 0; a v that is
// not zero keeps the lowest code, so that what it divides does not blow up.
#include <algorithm>
#include <climits>
#include <cmath>

#include "sbn_internal.hpp"
#include "sbn_rows.hpp"

namespace sbn {

namespace {

constexpr int THREADS = 256;
constexpr int STEP = THREADS * 8;             // values of a block at once
// Values of a block at most.  Short pieces keep the stores of all blocks near each other in memory (79M weights with fp32 moments: 305 us, by 8 steps 336, by
// 16 347); with moments in 8 bits what a block does once weighs too (317M weights: 608 by one step, 574 by two, 576 by four, 581 by eight, 607 by 16).
constexpr int64_t CHUNK_32BIT = STEP, CHUNK_8BIT = 4 * STEP;

struct AdamWItem {
    void *p;
    const void *g;
    void *m, *v;
    uint8_t *m_scales, *v_scales;
    uint32_t n;
    float decay;
};
constexpr int ADAMW_LAUNCH_MAX = 64;   // tensors of a launch: their table is a kernel argument, and a wavefront looks through it at once

struct AdamWArgs {
    int first_block[ADAMW_LAUNCH_MAX];   // of a tensor; behind the last one the number of blocks
    AdamWItem items[ADAMW_LAUNCH_MAX];
    const float *lr, *clip;
    const int64_t *step;
    double log_beta1, log_beta2;
    float beta1, less_beta1, beta2, less_beta2;   // less_beta: 1 - beta
    float eps;
    uint32_t seed_low, seed_high;
    int first_item;   // place in the call of items[0]
    uint32_t chunk;   // values of a block
};
static_assert(sizeof(AdamWArgs) <= 4096, "kernel arguments");

// the tensor of a block: how many begin at or in front of it, less one
__device__ __forceinline__ int tensor_of(const int *first_block, int block)
{
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(first_block[threadIdx.x & 63] <= block)) - 1);
}

__device__ __forceinline__ float lane_value(float x, int lane) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), lane)); }

// 1 - beta^t from the logarithm of beta: to a few steps of fp32, where powers in double took as long as a thousand values
__device__ __forceinline__ float less_power(double log_beta, double t) { return -expm1f((float)(t * log_beta)); }

// 32 random bits of a counter and two keys: two rounds of a multiplication between shifts, the multipliers from the digits of the golden ratio and
// of pi.  The rounding needs no more than bits that are even on average and not the same for neighbours, moments or steps.
__device__ __forceinline__ uint32_t mix(uint32_t x, uint32_t key0, uint32_t key1)
{
    x = (x ^ (x >> 16) ^ (key0 ^ (key0 >> 16))) * 0x9E3779B1u;   // x ^ key0, shifted and added to itself
    x = (x ^ (x >> 15)) + key1;
    x *= 0x85A308D3u;
    return x ^ (x >> 16);
}

constexpr int M_BELOW = 15, V_BELOW = 31;

// A value's pattern lies in its upper 16 bits, so two values are decoded, and their codes made, at once.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));

// the upper halves of two patterns, the first one's in the low half
__device__ __forceinline__ uint32_t upper_halves(uint32_t first, uint32_t second) { return __builtin_amdgcn_perm(second, first, 0x07060302u); }

// the values of four codes
template <int BELOW> __device__ __forceinline__ void values_of(uint32_t codes, uint32_t exponent, float *f)
{
    const u16x2 offset = (u16x2)(uint16_t)((exponent - BELOW) << 7);   // 8 codes to a binade, a code at bit 4
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t x = __builtin_amdgcn_perm(0, codes, j ? 0x030c020cu : 0x010c000cu);   // two codes, in the upper byte of each half
        const u16x2 low = __builtin_bit_cast(u16x2, (BELOW == M_BELOW ? x & 0x7f007f00u : x) >> 4);
        // the offset where the code is not 0: less than any 2^16 - low
        uint32_t both = __builtin_bit_cast(uint32_t, (u16x2)(low + __builtin_elementwise_min((u16x2)(-low), offset)));
        if (BELOW == M_BELOW) both |= x & 0x80008000u;
        f[2 * j] = __uint_as_float(both << 16);
        f[2 * j + 1] = __uint_as_float(both & 0xffff0000u);
    }
}

// 0 for 0, else 1, in one instruction (the compiler makes two of a minimum)
__device__ __forceinline__ uint32_t not_zero(uint32_t x)
{
    uint32_t y;
    asm("v_min_u32 %0, 1, %1" : "=v"(y) : "v"(x));
    return y;
}

// the codes of four values; half: what rounding adds to their patterns
template <int BELOW> __device__ __forceinline__ uint32_t codes_of(const float *x, uint32_t exponent, const uint32_t (&half)[4])
{
    const uint32_t offset = (exponent - BELOW) << 23;
    i16x2 q[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        uint32_t t[2], sign[2], some[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t bits = __float_as_uint(x[2 * j + k]), a = BELOW == V_BELOW ? bits : bits & 0x7fffffffu;   // (v has no sign)
            t[k] = a + (half[2 * j + k] - offset);   // the code, less its offset, above bit 20
            sign[k] = bits;
            some[k] = BELOW == V_BELOW ? not_zero(a) : 0;
        }
        const i16x2 code = __builtin_bit_cast(i16x2, upper_halves(t[0], t[1])) >> (int16_t)4;
        if constexpr (BELOW == V_BELOW)
            q[j] = __builtin_elementwise_max(code, __builtin_bit_cast(i16x2, some[0] | some[1] << 16));
        else
            q[j] = __builtin_bit_cast(i16x2, __builtin_bit_cast(uint32_t, __builtin_elementwise_max(code, (i16x2)(int16_t)0)) |
                                                 ((upper_halves(sign[0], sign[1]) >> 8) & 0x00800080u));
    }
    return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, q[1]), __builtin_bit_cast(uint32_t, q[0]), 0x06040200u);
}
__device__ __forceinline__ uint32_t nearest(float x) { return 0x7ffffu + ((__float_as_uint(x) >> 20) & 1u); }

// the exponent that 32 values share, four lanes with eight each
template <int BELOW> __device__ __forceinline__ uint32_t shared_exponent(const float (&x)[8])
{
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max(top, BELOW == V_BELOW ? __float_as_uint(x[k]) : __float_as_uint(x[k]) & 0x7fffffffu);
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xb1, 0xf, 0xf, true));   // quad_perm: lane ^ 1, lane ^ 2
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4e, 0xf, 0xf, true));
    return min(max((top + 0xfffffu) >> 23, (uint32_t)BELOW), 255u);   // one more where rounding may reach the next binade
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// What a thread has of a tensor: eight weights with their gradients and moments.  All of it is read and written once a step, and weights, gradients and fp32
// moments go past the caches (nontemporal): what a step leaves in the memory side's cache has to leave it while the next kernel reads.  The norm of 79M
// gradients and a step with fp32 moments took 30 + 347 us (30 + 305 now), with stores through the caches 52 + 330; with 8-bit moments for 317M weights 94 + 602
// (94 + 576 now), through the caches 94 + 643.  (Codes go through the caches, eight bytes to a thread: past them 623, their loads alone 598 for 583.)
template <sbn_dtype PT, sbn_dtype GT, bool BITS8> struct Eight {
    float p[8], g[8], m[8], v[8];

    template <bool WHOLE> __device__ __forceinline__ void load(const AdamWItem &it, uint32_t at)
    {
        const uint32_t unit = at / 8;
        if (WHOLE) {
            load_whole<PT>(it.p, at, p);
            load_whole<GT>(it.g, at, g);
        } else {
            load_unit<PT, 8>(it.p, unit, it.n, p);
            load_unit<GT, 8>(it.g, unit, it.n, g);
        }
        if constexpr (BITS8) {
            u32x2 mc = static_cast<const u32x2 *>(it.m)[unit], vc = static_cast<const u32x2 *>(it.v)[unit];
            const uint32_t me = it.m_scales[at / 32], ve = it.v_scales[at / 32];
            if (!WHOLE) {   // what pads the last 32 is zero
                mc = first_bytes(mc, (int64_t)it.n - at);
                vc = first_bytes(vc, (int64_t)it.n - at);
            }
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
                values_of<M_BELOW>(mc[k / 4], me, m + k);
                values_of<V_BELOW>(vc[k / 4], ve, v + k);
            }
        } else if (WHOLE) {
            load_whole<SBN_F32>(it.m, at, m);
            load_whole<SBN_F32>(it.v, at, v);
        } else {
            load_unit<SBN_F32, 8>(it.m, unit, it.n, m);
            load_unit<SBN_F32, 8>(it.v, unit, it.n, v);
        }
    }
    // CUT: bf16 weights are the upper halves of what p holds
    template <bool WHOLE, bool CUT> __device__ __forceinline__ void store(const AdamWItem &it, uint32_t at) const
    {
        const uint32_t unit = at / 8;
        if constexpr (CUT) {
            u32x4 w;
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = upper_halves(__float_as_uint(p[2 * k]), __float_as_uint(p[2 * k + 1]));
            if (WHOLE)
                Row<PT>::template store<true>(it.p, unit, w);
            else
                store_vec<PT>(it.p, unit, it.n, w);
        } else if (WHOLE)
            store_whole<PT>(it.p, at, p);
        else
            store_unit<PT, 8>(it.p, unit, it.n, p);
        if constexpr (!BITS8) {
            if (WHOLE) {
                store_whole<SBN_F32>(it.m, at, m);
                store_whole<SBN_F32>(it.v, at, v);
            } else {
                store_unit<SBN_F32, 8>(it.m, unit, it.n, m);
                store_unit<SBN_F32, 8>(it.v, unit, it.n, v);
            }
        }
    }

private:
    template <sbn_dtype DT> static __device__ __forceinline__ void load_whole(const void *p, uint32_t at, float (&f)[8])
    {
        constexpr int E = Row<DT>::E;
        const void *here = static_cast<const typename Row<DT>::value *>(p) + at;
#pragma unroll
        for (int j = 0; j < 8 / E; ++j) {
            float part[E];
            Row<DT>::unpack(Row<DT>::template load<true>(here, j), part);
#pragma unroll
            for (int k = 0; k < E; ++k) f[j * E + k] = part[k];
        }
    }
    template <sbn_dtype DT> static __device__ __forceinline__ void store_whole(void *p, uint32_t at, const float (&f)[8])
    {
        constexpr int E = Row<DT>::E;
        void *here = static_cast<typename Row<DT>::value *>(p) + at;
#pragma unroll
        for (int j = 0; j < 8 / E; ++j) {
            float part[E];
#pragma unroll
            for (int k = 0; k < E; ++k) part[k] = f[j * E + k];
            Row<DT>::template store<true>(here, j, Row<DT>::pack(part));
        }
    }
    static __device__ __forceinline__ u32x2 first_bytes(u32x2 c, int64_t n)
    {
        const uint64_t all = (uint64_t)c[1] << 32 | c[0], some = n >= 8 ? all : n <= 0 ? 0 : all & (((uint64_t)1 << (8 * n)) - 1);
        return (u32x2){(uint32_t)some, (uint32_t)(some >> 32)};
    }
};

template <sbn_dtype PT, sbn_dtype GT, bool BITS8, bool STOCHASTIC> __global__ void __launch_bounds__(THREADS) adamw_kernel(const AdamWArgs a)
{
    float factor = 1.0f;
    if (a.clip) {
        factor = *a.clip;
        if (!(fabsf(factor) <= 3.4028235e38f)) return;   // gradients that are not finite: no step
    }
    const int which = tensor_of(a.first_block, blockIdx.x);
    const AdamWItem it = a.items[which];
    const int64_t step = *a.step;
    const float given = *a.lr, lr = given == given ? given : __uint_as_float(0x7fc00000u);   // (a NaN whose pattern rounding does not run over)
    const float keep = (float)(1.0 - (double)lr * (double)it.decay);
    // both powers at once, in lanes of their own: rate = lr / (1 - beta1^t), of_v = 1 / sqrt(1 - beta2^t)
    const bool second = threadIdx.x & 1;
    const float power = less_power(second ? a.log_beta2 : a.log_beta1, (double)step), of = (second ? 1.0f : lr) / (second ? sqrtf(power) : power);
    const float rate = lane_value(of, 0), of_v = lane_value(of, 1);
    const float b1 = a.beta1, c1 = a.less_beta1, b2 = a.beta2, c2 = a.less_beta2;
    // v_sqrt_f32 and v_rcp_f32 are good to a step of fp32 and take less than half the time of the correctly rounded root and quotient, but make zero of
    // numbers below 2^-126: with an eps that is nothing beside such a root they must not be met
    const bool exactly = a.eps < 1e-12f;
    uint32_t key0 = 0, key1 = 0;
    if (STOCHASTIC) {
        key0 = mix(a.seed_low, a.seed_high, 0);
        key0 = mix(key0, (uint32_t)step, (uint32_t)(step >> 32));
        key0 = mix(key0, (uint32_t)(a.first_item + which), 0);
        key1 = mix(key0, 0x243F6A88u, 0);
    }
    const uint32_t begin = (blockIdx.x - a.first_block[which]) * a.chunk;   // at most 2^31 values
    const uint32_t end = (min(it.n, begin + a.chunk) + 31) / 32 * 32;
    // four threads have the 32 values that share an exponent, and go through the loop together
    for (uint32_t at = begin + threadIdx.x * 8; at < end; at += STEP) {
        Eight<PT, GT, BITS8> e;
        const bool whole = at + 8 <= it.n;
        if (whole)
            e.template load<true>(it, at);
        else
            e.template load<false>(it, at);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float s = e.g[k] * factor;   // (a factor of one changes nothing)
            e.m[k] = e.m[k] * b1 + s * c1;
            e.v[k] = e.v[k] * b2 + s * c2 * s;
        }
        if (!exactly) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                e.p[k] = fmaf(-rate * e.m[k], __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(e.v[k]), of_v, a.eps)), e.p[k] * keep);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) e.p[k] = e.p[k] * keep - rate * e.m[k] / (sqrtf(e.v[k]) * of_v + a.eps);
        }
        // 16 bits for the rounding of every p, m and v: two values to a hash
        const auto noise = [&](int j, int k) {
            const uint32_t bits = mix(3 * (at / 2 + k / 2) + j, key0, key1);
            return k & 1 ? bits >> 16 : bits & 0xffffu;
        };
        constexpr bool CUT = PT == SBN_BF16 && STOCHASTIC;
        if constexpr (CUT) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float rounded = __uint_as_float(__float_as_uint(e.p[k]) + noise(0, k));
                // the pattern of a NaN in fp32 could run over to that of a zero; those that come of bf16 and 8 bits, or of infinities, do not reach so far
                e.p[k] = (GT == SBN_BF16 && BITS8) || e.p[k] == e.p[k] ? rounded : e.p[k];
            }
        }
        if (whole)
            e.template store<true, CUT>(it, at);
        else
            e.template store<false, CUT>(it, at);
        if constexpr (BITS8) {
            const uint32_t me = shared_exponent<M_BELOW>(e.m), ve = shared_exponent<V_BELOW>(e.v);
            u32x2 mc, vc;
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
                uint32_t m_half[4], v_half[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    m_half[i] = STOCHASTIC ? noise(1, k + i) * 16 + 8 : nearest(e.m[k + i]);
                    v_half[i] = STOCHASTIC ? noise(2, k + i) * 16 + 8 : nearest(e.v[k + i]);
                }
                mc[k / 4] = codes_of<M_BELOW>(e.m + k, me, m_half);
                vc[k / 4] = codes_of<V_BELOW>(e.v + k, ve, v_half);
            }
            static_cast<u32x2 *>(it.m)[at / 8] = mc;
            static_cast<u32x2 *>(it.v)[at / 8] = vc;
            if (at % 32 == 0) {
                it.m_scales[at / 32] = (uint8_t)me;
                it.v_scales[at / 32] = (uint8_t)ve;
            }
        }
    }
}

template <sbn_dtype OUT, int BELOW> __global__ void __launch_bounds__(256) state_values_kernel(const uint2 *codes, const uint8_t *scales, int64_t n, void *out)
{
    const int64_t unit = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (unit * 8 >= n) return;
    const uint2 c = codes[unit];
    const uint32_t e = scales[unit / 4];
    float f[8];
    values_of<BELOW>(c.x, e, f);
    values_of<BELOW>(c.y, e, f + 4);
    store_unit<OUT, 8>(out, unit, n, f);
}

// ---- the norm of all gradients ----------------------------------------------------------------------------------------------------
constexpr int GRAD_NORM_LAUNCH_MAX = 64;
constexpr int64_t MEMORY_CACHE = 256 << 20;   // bytes of the memory side's cache
// Values of a block: 64 KB, or 32 where that is not four blocks to a processor (a call on 4M values in fp32 12.4 -> 6.2 us, on 2M in bf16 6.9 -> 6.3; the
// kernels alone now take 4.4 and 2.2, 4.1 and 2.0, and calls up to 8.8 where the host is slower than they).
int64_t grad_norm_chunk(int count, const int64_t *sizes, sbn_dtype dtype)
{
    const int64_t size = dtype == SBN_BF16 ? 2 : 4;
    int64_t values = 0;
    for (int i = 0; i < count; ++i) values += sizes[i];
    return (values * size < 4 * 256 * 32768 ? 32768 : 65536) / size;
}
constexpr int64_t GRAD_NORM_CHUNK_LEAST = 32768 / 4;

struct GradNormArgs {
    int first_block[GRAD_NORM_LAUNCH_MAX];
    const void *g[GRAD_NORM_LAUNCH_MAX];
    int64_t n[GRAD_NORM_LAUNCH_MAX];
    int64_t chunk;   // values of a block
    double *sums;
};

__device__ __forceinline__ double block_sum(double s, double *scratch)
{
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += scratch[w];
    return s;
}

// Squares in double: those of fp32 gradients reach past the range of fp32.  ONCE: the gradients are more than the memory side's cache holds, and go past it
// (317M in bf16: 94 us against 143); else they are left there for the step (79M: 30 + 347 us against 27 + 369).
template <sbn_dtype GT, bool ONCE> __global__ void __launch_bounds__(256) square_sums_kernel(const GradNormArgs a)
{
    __shared__ double scratch[4];
    const int which = tensor_of(a.first_block, blockIdx.x);
    const void *g = a.g[which];
    const int64_t n = a.n[which], begin = (int64_t)((int)blockIdx.x - a.first_block[which]) * a.chunk;
    const int64_t end = min(n, begin + a.chunk);
    double s = 0.0;
    constexpr int E = Row<GT>::E, AT_ONCE = 8;
    for (int64_t at = begin + threadIdx.x * E; at < end; at += 256 * E * AT_ONCE) {
        u32x4 x[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) x[j] = load_vec<GT, ONCE>(g, at / E + 256 * j, end);
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            float f[E];
            Row<GT>::unpack(x[j], f);
#pragma unroll
            for (int k = 0; k < E; ++k) s = fma((double)f[k], (double)f[k], s);
        }
    }
    s = block_sum(s, scratch);
    if (threadIdx.x == 0) a.sums[blockIdx.x] = s;
}

__global__ void __launch_bounds__(1024) grad_norm_kernel(const double *sums, int64_t blocks, float max_norm, float *out)
{
    __shared__ double scratch[16];
    double s = 0.0;
#pragma unroll 8
    for (int64_t b = threadIdx.x; b < blocks; b += 1024) s += sums[b];
    s = block_sum(s, scratch);
    if (threadIdx.x == 0) {
        const double norm = sqrt(s);
        out[0] = (float)norm;
        out[1] = isfinite(norm) ? (float)fmin(1.0, (double)max_norm / norm) : __uint_as_float(0x7fc00000u);
    }
}

template <sbn_dtype PT, sbn_dtype GT, bool BITS8> void launch_adamw_as(const AdamWArgs &a, int64_t blocks, bool stochastic, hipStream_t stream)
{
    if (stochastic)
        hipLaunchKernelGGL((adamw_kernel<PT, GT, BITS8, true>), dim3((unsigned)blocks), dim3(THREADS), 0, stream, a);
    else
        hipLaunchKernelGGL((adamw_kernel<PT, GT, BITS8, false>), dim3((unsigned)blocks), dim3(THREADS), 0, stream, a);
}
template <sbn_dtype PT, sbn_dtype GT> void launch_adamw_bits(const AdamWArgs &a, int64_t blocks, bool bits8, bool stochastic, hipStream_t stream)
{
    bits8 ? launch_adamw_as<PT, GT, true>(a, blocks, stochastic, stream) : launch_adamw_as<PT, GT, false>(a, blocks, stochastic, stream);
}

}  // namespace

// One sum to a block of the shortest length, whichever the call takes: it never falls as tensors or values are added, so that a buffer for all gradients serves
// a part of them (by the blocks' own length 8M values took 7816 bytes, and 8.7M 4256).
size_t grad_norm_workspace_bytes(int count, const int64_t *sizes)
{
    int64_t blocks = 0;
    for (int i = 0; i < count; ++i) blocks += ceil_div(sizes[i], GRAD_NORM_CHUNK_LEAST);
    return (size_t)blocks * sizeof(double);
}

sbn_status launch_grad_norm(int count, const void *const *grads, sbn_dtype dtype, const int64_t *sizes, float max_norm, float *out, void *workspace, hipStream_t stream)
{
    double *sums = static_cast<double *>(workspace);
    const int64_t chunk = grad_norm_chunk(count, sizes, dtype);
    int64_t all = 0, values = 0;
    for (int i = 0; i < count; ++i) values += sizes[i];
    const bool once = values * (dtype == SBN_BF16 ? 2 : 4) > MEMORY_CACHE;
    for (int first = 0; first < count; first += GRAD_NORM_LAUNCH_MAX) {
        GradNormArgs a;
        a.sums = sums + all;
        a.chunk = chunk;
        const int here = std::min(count - first, GRAD_NORM_LAUNCH_MAX);
        int64_t blocks = 0;
        for (int i = 0; i < GRAD_NORM_LAUNCH_MAX; ++i) {
            a.g[i] = i < here ? grads[first + i] : nullptr;
            a.n[i] = i < here ? sizes[first + i] : 0;
            a.first_block[i] = i < here ? (int)blocks : INT_MAX;
            blocks += ceil_div(a.n[i], chunk);
        }
        const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, stream, a); };
        if (dtype == SBN_BF16)
            once ? launch(square_sums_kernel<SBN_BF16, true>) : launch(square_sums_kernel<SBN_BF16, false>);
        else
            once ? launch(square_sums_kernel<SBN_F32, true>) : launch(square_sums_kernel<SBN_F32, false>);
        all += blocks;
    }
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(1024), 0, stream, sums, all, max_norm, out);
    return check_launch("grad_norm_kernel");
}

sbn_status launch_adamw(const AdamWCall &c, hipStream_t stream)
{
    const bool bits8 = c.m_scales != nullptr;
    for (int first = 0; first < c.count; first += ADAMW_LAUNCH_MAX) {
        AdamWArgs a;
        a.lr = c.lr;
        a.clip = c.clip;
        a.step = c.step;
        a.log_beta1 = std::log(c.beta1);
        a.log_beta2 = std::log(c.beta2);
        a.beta1 = (float)c.beta1;
        a.less_beta1 = (float)(1.0 - c.beta1);
        a.beta2 = (float)c.beta2;
        a.less_beta2 = (float)(1.0 - c.beta2);
        a.eps = (float)c.eps;
        a.seed_low = c.seed ? (uint32_t)*c.seed : 0;
        a.seed_high = c.seed ? (uint32_t)(*c.seed >> 32) : 0;
        const int here = std::min(c.count - first, ADAMW_LAUNCH_MAX);
        a.first_item = first;
        int64_t values = 0;
        for (int i = 0; i < here; ++i) values += c.sizes[first + i];
        // four blocks to a processor at least where there are values for them
        a.chunk = (uint32_t)std::max<int64_t>(STEP, std::min(bits8 ? CHUNK_8BIT : CHUNK_32BIT, values / (256 * 4) / STEP * STEP));
        int64_t blocks = 0;
        for (int i = 0; i < ADAMW_LAUNCH_MAX; ++i) {
            const int j = first + i;
            a.first_block[i] = i < here ? (int)blocks : INT_MAX;
            if (i >= here) {
                a.items[i] = AdamWItem{};
                continue;
            }
            a.items[i] = AdamWItem{c.params[j], c.grads[j], c.m[j], c.v[j], bits8 ? c.m_scales[j] : nullptr, bits8 ? c.v_scales[j] : nullptr, (uint32_t)c.sizes[j],
                                   c.weight_decay ? c.weight_decay[j] : 0.0f};
            blocks += ceil_div(c.sizes[j], (int64_t)a.chunk);
        }
        if (c.param_dtype == SBN_BF16)
            c.grad_dtype == SBN_BF16 ? launch_adamw_bits<SBN_BF16, SBN_BF16>(a, blocks, bits8, c.seed != nullptr, stream)
                                     : launch_adamw_bits<SBN_BF16, SBN_F32>(a, blocks, bits8, c.seed != nullptr, stream);
        else
            c.grad_dtype == SBN_BF16 ? launch_adamw_bits<SBN_F32, SBN_BF16>(a, blocks, bits8, c.seed != nullptr, stream)
                                     : launch_adamw_bits<SBN_F32, SBN_F32>(a, blocks, bits8, c.seed != nullptr, stream);
    }
    return check_launch("adamw_kernel");
}

sbn_status launch_adamw_state_values(const void *codes, const uint8_t *scales, int64_t n, bool second, void *out, sbn_dtype dtype, hipStream_t stream)
{
    const auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(n, 2048)), dim3(256), 0, stream, static_cast<const uint2 *>(codes), scales, n, out);
    };
    if (dtype == SBN_BF16)
        second ? launch(state_values_kernel<SBN_BF16, V_BELOW>) : launch(state_values_kernel<SBN_BF16, M_BELOW>);
    else
        second ? launch(state_values_kernel<SBN_F32, V_BELOW>) : launch(state_values_kernel<SBN_F32, M_BELOW>);
    return check_launch("state_values_kernel");
}

}  // namespace sbn
