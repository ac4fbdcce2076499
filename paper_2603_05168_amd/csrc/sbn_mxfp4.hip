// Microscaled 4-bit floating point: blocks of 32 consecutive values of a row share a scale 2^(s - 127) (one byte), a value is a sign and one
// of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  Rows are padded with zeros to whole 128 columns; two codes lie in a byte, the even column in the low half.
//   s = max(exponent field of the block's largest magnitude - 2, 0),  code = magnitude / 2^(s - 127) rounded to the nearest (ties to the even
//   code), at most 6
// The product runs on v_mfma_scale_f32_32x32x64_f8f6f4, which takes both operands and their scales as they are stored and adds up in fp32.
#include <algorithm>

#include "sbn_internal.hpp"
#include "sbn_mfma.hpp"

namespace sbn {

namespace {

constexpr int GROUP = 32, PAD = 128;

// 2^(s - 127) and its inverse
__device__ __forceinline__ float scale_value(const uint32_t s) { return __uint_as_float(s ? s << 23 : 0x00400000u); }
__device__ __forceinline__ float scale_inverse(const uint32_t s) { return __uint_as_float((254u - s) << 23); }

// ---- quantize ----------------------------------------------------------------------------------------------------------------------
// A lane takes eight values of a row, four neighbouring lanes a block.
template <bool BF16>
__device__ __forceinline__ void load8(const void *src, const int64_t at, float (&x)[8])
{
    if constexpr (BF16) {
        const uint4 v = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(src) + at);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
        const v4f lo = *reinterpret_cast<const v4f *>(static_cast<const float *>(src) + at), hi = *reinterpret_cast<const v4f *>(static_cast<const float *>(src) + at + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = lo[i];
            x[4 + i] = hi[i];
        }
    }
}

// codes of eight values (a word), s: scale of the block that four neighbouring lanes hold
__device__ __forceinline__ uint32_t quantize8(const float (&x)[8], uint32_t &s)
{
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[i]));
    most = fmaxf(most, __shfl_xor(most, 1));
    most = fmaxf(most, __shfl_xor(most, 2));
    const uint32_t field = __float_as_uint(most) >> 23;
    s = field > 2 ? field - 2 : 0u;
    const float inv = scale_inverse(s);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0] * inv, x[1] * inv, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2] * inv, x[3] * inv, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4] * inv, x[5] * inv, 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6] * inv, x[7] * inv, 1.0f, 3);
    return w;
}

template <bool BF16>
__global__ void __launch_bounds__(256) mxfp4_quantize_kernel(const void *X, int64_t rows, int cols, int vectors, uint32_t *codes, uint8_t *scales)
{
    // vectors: of eight values in a padded row, a multiple of 16
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * vectors) return;   // whole blocks of four lanes
    const int64_t row = i / vectors;
    const int col = 8 * (int)(i - row * vectors);
    float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (col < cols) load8<BF16>(X, row * cols + col, x);
    uint32_t s;
    codes[i] = quantize8(x, s);
    if ((threadIdx.x & 3) == 0) scales[i >> 2] = (uint8_t)s;
}

template <bool BF16>
__global__ void __launch_bounds__(256) mxfp4_dequantize_kernel(const uint32_t *codes, const uint8_t *scales, int64_t rows, int cols, int vectors, void *Y)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int across = cols / 8;
    if (i >= rows * across) return;
    const int64_t row = i / across;
    const int v = (int)(i - row * across);
    const uint32_t w = codes[row * vectors + v];
    const float scale = scale_value(scales[(row * vectors + v) >> 2]);
    typedef float v2f __attribute__((ext_vector_type(2)));
    const v2f p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3)};
    const int64_t at = row * cols + 8 * v;
    if constexpr (BF16) {
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)   // exact: two significant bits, so the high half of the fp32 value
            o[k] = __builtin_amdgcn_perm(__float_as_uint(p[k][1] * scale), __float_as_uint(p[k][0] * scale), 0x07060302u);
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(Y) + at) = make_uint4(o[0], o[1], o[2], o[3]);
    } else {
        v4f *const to = reinterpret_cast<v4f *>(static_cast<float *>(Y) + at);
        to[0] = v4f{p[0][0] * scale, p[0][1] * scale, p[1][0] * scale, p[1][1] * scale};
        to[1] = v4f{p[2][0] * scale, p[2][1] * scale, p[3][0] * scale, p[3][1] * scale};
    }
}

// ---- block tile product -----------------------------------------------------------------------------------------------------------------
// Y[t, o] = sum_k q(X)[t, k] W[o, k] (+ bias[o]) for block tiles of 256 x 256 (o x t; eight wavefronts of 128 x 64) or 128 x 128 (four of 64 x 64, two
// blocks per multiprocessor).  Stages of 256 k (128 bytes of a row, and its eight scales) come by LDS-DMA into two buffers; a stage is
// consumed in quarters of 64 k, quarter u being the blocks u and 4 + u of the stage: a lane's scales of a stage are then one word, whose byte
// u the instruction picks.
constexpr int STAGE_BYTES = 128, STAGE_SCALES = 8;
template <bool BIG> struct MxTile {
    static constexpr int N = BIG ? 256 : 128, M = N, WAVES = BIG ? 8 : 4;
    static constexpr int WP = BIG ? 4 : 2, WQ = 2;
    static constexpr int CODES = N * STAGE_BYTES, SCALES = N * STAGE_SCALES;
    static constexpr int STAGE = 2 * (CODES + SCALES), LDS = 2 * STAGE;      // P codes, Q codes, P scales, Q scales
    static constexpr int ROW = WP * 128;                                     // bytes of a staged row of results
    static_assert(WAVES * 32 * ROW <= LDS, "results are staged in the idle stages");
};
struct MxArgs {
    const uint8_t *P, *Q;      // codes of W [N, pitch] and of X [M, pitch]
    const uint8_t *sp, *sq;    // their scales, [., pitch / 16]
    int64_t pitch;             // bytes of a row, a multiple of 64
    int N, M;
    const float *bias;
    float *Y;                  // [M, N]
    int tiles_n, tiles_m;
};

// one dword per lane through a buffer resource (see lds_dma16_buffer): lane l deposits at lds_addr + 4 l
__device__ __forceinline__ void lds_dma4_buffer(const v4i rsrc, uint32_t voff, uint32_t soff, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" : : "s"(lds_addr), "v"(voff), "s"(rsrc), "s"(soff) : "memory", "m0");
}

template <bool BIG>
__global__ void __launch_bounds__(64 * MxTile<BIG>::WAVES) mxfp4_tile_kernel(MxArgs g)
{
    using S = MxTile<BIG>;
    constexpr int WP = S::WP, WQ = S::WQ, SLOTS = WP * WQ;
    extern __shared__ __attribute__((aligned(1024))) uint8_t dlds[];
    const int nb = g.tiles_n * g.tiles_m, per = (nb + 7) >> 3;
    const int id = ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3);   // an XCD takes a contiguous eighth
    if (((int)blockIdx.x >> 3) >= per || id >= nb) return;
    const int tn = id % g.tiles_n, tm = id / g.tiles_n;
    const int n0 = tn * S::N, m0 = tm * S::M;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave & 1, wm = wave >> 1, r = lane & 31, c = lane >> 5;
    const uint32_t lds0 = lds_address(dlds);
    const int nk = (int)((g.pitch + STAGE_BYTES - 1) / STAGE_BYTES);
    const bool half_last = (g.pitch & (STAGE_BYTES - 1)) != 0;             // the last stage is half a stage

    // rows past the matrix, and what is past its end, read as zeros
    const uint32_t pitch = (uint32_t)g.pitch, spitch = pitch / 16;
    const int prows = std::min(S::N, g.N - n0), qrows = std::min(S::M, g.M - m0);
    const int pbytes = prows * (int)pitch, qbytes = qrows * (int)pitch;
    v4i pb = buffer_of(g.P + (int64_t)n0 * pitch, pbytes), qb = buffer_of(g.Q + (int64_t)m0 * pitch, qbytes);
    v4i spb = buffer_of(g.sp + (int64_t)n0 * spitch, pbytes / 16), sqb = buffer_of(g.sq + (int64_t)m0 * spitch, qbytes / 16);
    uint32_t off[4];   // the same of both operands
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = 32 * wave + 8 * i + (lane >> 3);
        off[i] = (uint32_t)row * pitch + 16u * ((lane & 7) ^ ((row >> 1) & 7));
    }
    const uint32_t soff = (uint32_t)(32 * wave + (lane >> 1)) * spitch + 4u * (lane & 1);
    auto request = [&](const int kt, const int i) {   // instruction i < 10 of stage kt; past the last one zeros are deposited
        if (i == 0) {   // (no branch: the compiler would move the matrix instructions behind it)
            const bool some = kt < nk;
            pb[2] = some ? pbytes : 0;
            qb[2] = some ? qbytes : 0;
            spb[2] = some ? pbytes / 16 : 0;
            sqb[2] = some ? qbytes / 16 : 0;
        }
        const uint32_t at = lds0 + (kt & 1) * S::STAGE, k = (uint32_t)kt * STAGE_BYTES;
        if (i < 4) lds_dma16_buffer(pb, off[i], k, at + wave * 4096 + i * 1024);
        else if (i < 8) lds_dma16_buffer(qb, off[i - 4], k, at + S::CODES + wave * 4096 + (i - 4) * 1024);
        else if (i == 8) lds_dma4_buffer(spb, soff, k / 16, at + 2 * S::CODES + wave * 256);
        else lds_dma4_buffer(sqb, soff, k / 16, at + 2 * S::CODES + S::SCALES + wave * 256);
    };
    // the second half of a last stage that is half a stage: zeros in place of what the next row begins with
    auto zero_tail = [&](const uint32_t at) {
        typedef __attribute__((address_space(3))) v4i *lds_v4i;
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int gran = (lane & 7) ^ (((32 * wave + 8 * i + (lane >> 3)) >> 1) & 7);
            if (gran >= 4) {
                *(lds_v4i)(uintptr_t)(lds0 + at + wave * 4096 + i * 1024 + 16 * lane) = v4i{0, 0, 0, 0};
                *(lds_v4i)(uintptr_t)(lds0 + at + S::CODES + wave * 4096 + i * 1024 + 16 * lane) = v4i{0, 0, 0, 0};
            }
        }
    };
    // granule 4 c + u of a row in quarter u: u flips bits of the address
    const uint32_t slot0 = 16 * ((4 * c) ^ ((r >> 1) & 7));
    const uint32_t pa = lds0 + (wn * 32 * WP + r) * 128 + slot0, qa = lds0 + S::CODES + (wm * 32 * WQ + r) * 128 + slot0;
    const uint32_t psa = lds0 + 2 * S::CODES + (wn * 32 * WP + r) * 8 + 4 * c, qsa = lds0 + 2 * S::CODES + S::SCALES + (wm * 32 * WQ + r) * 8 + 4 * c;
    typedef __attribute__((address_space(3))) const v4i *lds_v4i;
    typedef __attribute__((address_space(3))) const int *lds_int;

    v16f acc[WP][WQ];
#pragma unroll
    for (int a = 0; a < WP; ++a)
#pragma unroll
        for (int b = 0; b < WQ; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;
    v4i fp[2][WP], fq[2][WQ];
    int sp[WP], sq[WQ], sp_next[WP], sq_next[WQ];   // scales of a stage
    auto read_one = [&](const uint32_t at, const int u, const int i) {
        if (i < WP) fp[u & 1][i] = *(lds_v4i)(uintptr_t)((pa ^ (16 * u)) + at + i * 32 * 128);
        else fq[u & 1][i - WP] = *(lds_v4i)(uintptr_t)((qa ^ (16 * u)) + at + (i - WP) * 32 * 128);
    };
    auto read_scales = [&](const uint32_t at) {
#pragma unroll
        for (int a = 0; a < WP; ++a) sp_next[a] = *(lds_int)(uintptr_t)(psa + at + a * 32 * 8);
#pragma unroll
        for (int b = 0; b < WQ; ++b) sq_next[b] = *(lds_int)(uintptr_t)(qsa + at + b * 32 * 8);
    };
    auto wide = [](const v4i x) { return v8i{x[0], x[1], x[2], x[3], 0, 0, 0, 0}; };   // 4-bit operands are four registers
    auto quarter = [&](const int u, auto &&side) {
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            const int a = s / WQ, b = s % WQ;
            const v8i x = wide(fp[u & 1][a]), y = wide(fq[u & 1][b]);
            if (u == 0) acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, acc[a][b], 4, 4, 0, sp[a], 0, sq[b]);
            if (u == 1) acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, acc[a][b], 4, 4, 1, sp[a], 1, sq[b]);
            if (u == 2) acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, acc[a][b], 4, 4, 2, sp[a], 2, sq[b]);
            if (u == 3) acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, acc[a][b], 4, 4, 3, sp[a], 3, sq[b]);
            side(s);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    constexpr int READS = WP + WQ;
    auto spread = [&](const int s, const int n, auto &&op) {
#pragma unroll
        for (int k = 0; k < n; ++k)
            if (k * SLOTS / n == s) op(k);
    };
    // Step kt: quarters 0 to 2 read the fragments of the next quarter; then stage kt + 1 must have landed and every wavefront holds the last
    // fragments of stage kt, so behind the barrier the last quarter reads the first fragments of stage kt + 1 and stage kt + 2 is asked for.
    auto take_scales = [&] {
#pragma unroll
        for (int a = 0; a < WP; ++a) sp[a] = sp_next[a];
#pragma unroll
        for (int b = 0; b < WQ; ++b) sq[b] = sq_next[b];
    };
#pragma unroll
    for (int i = 0; i < 10; ++i) request(0, i);
#pragma unroll
    for (int i = 0; i < 10; ++i) request(1, i);
    SBN_WAIT_VMCNT(10);
    if (half_last && nk == 1) zero_tail(0);
    __syncthreads();
    read_scales(0);
    take_scales();
#pragma unroll
    for (int i = 0; i < READS; ++i) read_one(0, 0, i);
    uint32_t at = 0;
    for (int kt = 0; kt < nk; ++kt) {
        const uint32_t next = S::STAGE - at;
#pragma unroll
        for (int u = 0; u < 3; ++u)
            quarter(u, [&](const int s) { spread(s, READS, [&](const int k) { read_one(at, u + 1, k); }); });
        SBN_WAIT_VMCNT(0);
        if (half_last && kt + 2 == nk) zero_tail(next);
        __syncthreads();
        quarter(3, [&](const int s) {
            if (s == 0) read_scales(next);
            spread(s, READS, [&](const int k) { read_one(next, 0, k); });
            spread(s, 10, [&](const int k) { request(kt + 2, k); });
        });
        take_scales();
        at = next;
    }
    SBN_WAIT_VMCNT(0);   // the surplus stages have landed
    __syncthreads();

    // Result: 32 tokens at a time through the idle stages (granules of 16 bytes XOR-swizzled with the row), so that whole rows of the
    // wavefront's outputs leave
    typedef float v4f_u __attribute__((ext_vector_type(4), aligned(4)));
    uint8_t *const stg = dlds + wave * 32 * S::ROW;
    constexpr int LPR = S::ROW / 16, J = 32 * LPR / 64;
    const int nw = n0 + wn * 32 * WP, n = nw + 4 * (lane % LPR), mw = m0 + wm * 32 * WQ;
    v4f bias = {0.0f, 0.0f, 0.0f, 0.0f};
    if (g.bias)
#pragma unroll
        for (int i = 0; i < 4; ++i) bias[i] = n + i < g.N ? g.bias[n + i] : 0.0f;
#pragma unroll
    for (int b = 0; b < WQ; ++b) {
        asm volatile("" ::: "memory");
#pragma unroll
        for (int a = 0; a < WP; ++a)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<v4f *>(stg + r * S::ROW + 16 * ((8 * a + 2 * q + c) ^ (r & 15))) =
                    v4f{acc[a][b][4 * q], acc[a][b][4 * q + 1], acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]};
        asm volatile("" ::: "memory");
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int row = (64 / LPR) * j + lane / LPR, m = mw + 32 * b + row;
            v4f x = *reinterpret_cast<const v4f *>(stg + row * S::ROW + 16 * ((lane % LPR) ^ (row & 15)));
            if (g.bias) x += bias;
            if (m >= g.M) continue;
            float *const to = g.Y + (int64_t)m * g.N + n;
            if (n + 4 <= g.N) *reinterpret_cast<v4f_u *>(to) = x;
            else
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (n + i < g.N) to[i] = x[i];
        }
    }
}

template <bool BIG>
sbn_status launch_tile(MxArgs &g, hipStream_t stream)
{
    using S = MxTile<BIG>;
    g.tiles_n = (int)ceil_div(g.N, S::N);
    g.tiles_m = (int)ceil_div(g.M, S::M);
    static thread_local bool raised = false;
    if (!raised) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&mxfp4_tile_kernel<BIG>), hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
        if (e != hipSuccess) { set_hip_error(e, "hipFuncSetAttribute"); return SBN_EHIP; }
        raised = true;
    }
    const int64_t blocks = ceil_div((int64_t)g.tiles_n * g.tiles_m, 8) * 8;
    hipLaunchKernelGGL(mxfp4_tile_kernel<BIG>, dim3((unsigned)blocks), dim3(64 * S::WAVES), S::LDS, stream, g);
    return check_launch("mxfp4_tile_kernel");
}

int64_t padded(int64_t cols) { return ceil_div(cols, PAD) * PAD; }

}  // namespace

void mxfp4_bytes(int64_t rows, int64_t cols, size_t &codes, size_t &scales)
{
    codes = (size_t)(rows * padded(cols) / 2);
    scales = (size_t)(rows * padded(cols) / GROUP);
}

size_t mxfp4_workspace_bytes(int64_t tokens, int64_t d_in)
{
    size_t codes, scales;
    mxfp4_bytes(tokens, d_in, codes, scales);
    return align_up(codes, 256) + align_up(scales, 256);
}

sbn_status launch_mxfp4_quantize(const void *X, sbn_dtype dtype, int64_t rows, int64_t cols, uint8_t *codes, uint8_t *scales, hipStream_t stream)
{
    const int64_t vectors = padded(cols) / 8;
    const dim3 grid((unsigned)ceil_div(rows * vectors, 256)), block(256);
    uint32_t *const words = reinterpret_cast<uint32_t *>(codes);
    if (dtype == SBN_BF16) hipLaunchKernelGGL(mxfp4_quantize_kernel<true>, grid, block, 0, stream, X, rows, (int)cols, (int)vectors, words, scales);
    else hipLaunchKernelGGL(mxfp4_quantize_kernel<false>, grid, block, 0, stream, X, rows, (int)cols, (int)vectors, words, scales);
    return check_launch("mxfp4_quantize_kernel");
}

sbn_status launch_mxfp4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *Y, sbn_dtype dtype, hipStream_t stream)
{
    const int64_t vectors = padded(cols) / 8;
    const dim3 grid((unsigned)ceil_div(rows * (cols / 8), 256)), block(256);
    const uint32_t *const words = reinterpret_cast<const uint32_t *>(codes);
    if (dtype == SBN_BF16) hipLaunchKernelGGL(mxfp4_dequantize_kernel<true>, grid, block, 0, stream, words, scales, rows, (int)cols, (int)vectors, Y);
    else hipLaunchKernelGGL(mxfp4_dequantize_kernel<false>, grid, block, 0, stream, words, scales, rows, (int)cols, (int)vectors, Y);
    return check_launch("mxfp4_dequantize_kernel");
}

sbn_status launch_mxfp4_linear(const void *X, int64_t tokens, int64_t d_in, int64_t d_out, const uint8_t *codes, const uint8_t *scales, const float *bias,
                               float *Y, void *workspace, hipStream_t stream)
{
    size_t code_bytes, scale_bytes;
    mxfp4_bytes(tokens, d_in, code_bytes, scale_bytes);
    uint8_t *const xc = static_cast<uint8_t *>(workspace), *const xs = xc + align_up(code_bytes, 256);
    const sbn_status st = launch_mxfp4_quantize(X, SBN_BF16, tokens, d_in, xc, xs, stream);
    if (st != SBN_OK) return st;
    MxArgs g{codes, xc, scales, xs, padded(d_in) / 2, (int)d_out, (int)tokens, bias, Y, 0, 0};
    return launch_tile<false>(g, stream);
}

}  // namespace sbn
