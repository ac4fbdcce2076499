// Microscaled 4-bit floating point: blocks of 32 consecutive values of a row share a scale 2^(s - 127) (one byte), a value is a sign and one
// of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  Rows are padded with zeros to whole 128 columns; two codes lie in a byte, the even column in the low half.
//   s = max(exponent field of the block's largest magnitude - 2, 0),  code = magnitude / 2^(s - 127) rounded to the nearest (ties to the even
//   code), at most 6
// The product runs on v_mfma_scale_f32_32x32x64_f8f6f4, which takes both operands and their scales as they are stored and adds up in fp32.
#include <algorithm>
#include <atomic>
#include <cmath>

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

// codes of eight values (a word), s: scale of the block that four neighbouring lanes hold.  Values are finite: the maximum drops a NaN, which the
// conversion turns into a 6; of an infinity s is 253.
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

// PER vectors of eight values per lane, 256 apart.  Scales: block by block of a row, or, for the products, [stages of 2^stage_shift columns, rows, blocks
// of a stage].
template <bool BF16, int PER>
__global__ void __launch_bounds__(256) mxfp4_quantize_kernel(const void *X, uint32_t rows, int cols, uint32_t vectors, uint32_t *codes, uint8_t *scales,
                                                                int stage_shift)
{
    // vectors: in a padded row, a multiple of 16.  All together they are at most 2^32 (2^27 tokens of a product, whose rows are padded to 256 columns): the
    // last one's number has 32 bits, their count may have 33
    const uint32_t first = blockIdx.x * 256 * PER + threadIdx.x, last = rows * vectors - 1;
    float x[PER][8];
    uint32_t row[PER], col[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const uint32_t i = first + 256 * p;
        row[p] = i / vectors;
        col[p] = 8 * (i - row[p] * vectors);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[p][e] = 0.0f;
        if (i <= last && (int)col[p] < cols) load8<BF16>(X, (int64_t)row[p] * cols + col[p], x[p]);
    }
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const uint32_t i = first + 256 * p;
        if (i > last) return;   // whole blocks of four lanes
        uint32_t s;
        codes[i] = quantize8(x[p], s);
        if ((threadIdx.x & 3) == 0) {
            const int in_stage = stage_shift - 5;   // log2 of the blocks of a stage
            scales[stage_shift ? ((((int64_t)(col[p] >> stage_shift)) * rows + row[p]) << in_stage) + ((col[p] >> 5) & ((1u << in_stage) - 1)) : i >> 2] = (uint8_t)s;
        }
    }
}

template <bool BF16, int PER>
__global__ void __launch_bounds__(256) mxfp4_dequantize_kernel(const uint32_t *codes, const uint8_t *scales, uint32_t rows, uint32_t cols, uint32_t vectors, void *Y)
{
    const uint32_t first = blockIdx.x * 256 * PER + threadIdx.x, across = cols / 8, all = rows * across;
    uint32_t w[PER], s[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const uint32_t i = std::min(first + 256 * p, all - 1), row = i / across, at = row * vectors + (i - row * across);
        w[p] = codes[at];
        s[p] = scales[at >> 2];
    }
    typedef float v2f __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const uint32_t i = first + 256 * p;
        if (i >= all) return;
        const float scale = scale_value(s[p]);
        const v2f v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[p], 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[p], 1.0f, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[p], 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[p], 1.0f, 3)};
        const int64_t at = 8 * (int64_t)i;
        if constexpr (BF16) {
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)   // exact: two significant bits, so the high half of the fp32 value
                o[k] = __builtin_amdgcn_perm(__float_as_uint(v[k][1] * scale), __float_as_uint(v[k][0] * scale), 0x07060302u);
            *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(Y) + at) = make_uint4(o[0], o[1], o[2], o[3]);
        } else {
            v4f *const to = reinterpret_cast<v4f *>(static_cast<float *>(Y) + at);
            to[0] = v4f{v[0][0] * scale, v[0][1] * scale, v[1][0] * scale, v[1][1] * scale};
            to[1] = v4f{v[2][0] * scale, v[2][1] * scale, v[3][0] * scale, v[3][1] * scale};
        }
    }
}

// ---- block tile product -----------------------------------------------------------------------------------------------------------------
// Y[t, o] = sum_k q(X)[t, k] W[o, k] (+ bias[o]) for block tiles of 256 x 256 (o x t; eight wavefronts of 128 x 64), 128 x 128 (four of 64 x 64, two
// blocks per multiprocessor) and 64 x 64 (four of 32 x 32, four blocks).  Stages of 256 k (128 bytes of a row, a whole line) come by LDS-DMA into
// two slots; a stage is consumed in quarters of 64 k, quarter u being the blocks u and 4 + u of the stage: a lane's four scales of a stage are
// one word, and the instruction picks byte u.  Scales of X lie together per stage (the quantizer writes them so); those of W are rows apart,
// so four stages of them are asked for at once: a request for 4 bytes of a row costs as much as one for its line.
// An instruction on 4-bit operands has four times the products of one on bf16 in the same time, so its feeding and what surrounds it bound the
// product: a stage of the large tile takes 1.44 us, 1.17 without its requests and 0.98 its matrix instructions at 2.1 GHz; a tile's first
// stages, its way through LDS and its stores some 16 us more (4096 x 2560 -> 131072, us per tile: 37.6, 25 without stores, 21 without
// results; 30.7 with stores past the caches).  Half the stage in three slots for two blocks per multiprocessor was slower
// (64 bytes of a row are half a line: 81.7 us against 68.2 at 4096 x 2560 -> 6912), and so were requests spread over the stage.  Counters at that
// size (60 us): matrix pipe 24 % of the cycles, conflicts in 31 % of the LDS cycles (W's scales lie 32 bytes apart: four rows of a read to a bank, at
// least), 146 MB read for 15 (tiles in row order: W for every row of tiles and XCD).
constexpr int STAGE_BYTES = 128, STAGE_SCALES = 8;   // of a row and stage
template <int WP_, int WQ_, int WM> struct MxTile {
    static constexpr int WP = WP_, WQ = WQ_, WAVES = 2 * WM;                 // 32 x 32 tiles of a wavefront
    static constexpr int N = 64 * WP, M = 32 * WM * WQ;
    static constexpr int CHUNK_STAGES = 4;                                   // whose scales of W come together
    static constexpr int P = N * STAGE_BYTES, Q = M * STAGE_BYTES, SQ = M * STAGE_SCALES, STAGE = P + Q + SQ;   // in this order
    static constexpr int CHUNK_ROW = STAGE_SCALES * CHUNK_STAGES, CHUNK = N * CHUNK_ROW;      // scales of W of some stages
    static constexpr int CHUNKS = 2 * STAGE, LDS = CHUNKS + 2 * CHUNK;
    static constexpr int PI = N / (8 * WAVES), QI = M / (8 * WAVES);                          // requests (8 rows each) of a wavefront and stage
    static constexpr int REQUESTS = PI + QI + 1, CI = CHUNK / (256 * WAVES);                  // with X's scales; of a chunk
    // results of the large tiles, taken from some 40 MB on, leave past the caches, us through them and past: 4096 x 2560 -> 131072 1204 and 981, -> 6912 65.9
    // and 65.5, -> 2560 33.0 and 31.1; 1500 x 2560 -> 6912 30.8 and 28.4
    static constexpr bool PAST_CACHES = WP == 4;
    static constexpr int OUT = WP * 128;                                     // bytes of a staged row of results
    static_assert(WAVES * 32 * OUT <= CHUNKS, "results are staged in the idle stages");
};
using MxLarge = MxTile<4, 2, 4>;
using MxMiddle = MxTile<2, 2, 2>;
using MxSmall = MxTile<1, 1, 2>;
struct MxArgs {
    const uint8_t *P, *Q;      // codes of W [N, pitch] and of X [M, qpitch]
    const uint8_t *sp, *sq;    // their scales, [N, pitch / 16] and [stages, M, scales of a stage]
    int64_t pitch, qpitch;     // bytes of a row: a multiple of 64 (W) and of 128 (X)
    int N, M, stages;
    const float *bias;
    float *Y;                  // [M, N]
    int tiles_n, tiles_m;
};

// one dword per lane through a buffer resource (see lds_dma16_buffer): lane l deposits at lds_addr + 4 l
__device__ __forceinline__ void lds_dma4_buffer(const v4i rsrc, uint32_t voff, uint32_t soff, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" : : "s"(lds_addr), "v"(voff), "s"(rsrc), "s"(soff) : "memory", "m0");
}

template <class S>
__global__ void __launch_bounds__(64 * S::WAVES, 2) mxfp4_tile_kernel(MxArgs g)
{
    constexpr int WP = S::WP, WQ = S::WQ, TILES = WP * WQ;
    extern __shared__ __attribute__((aligned(1024))) uint8_t dlds[];
    const int nb = g.tiles_n * g.tiles_m, per = (nb + 7) >> 3;
    const int id = ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3);   // an XCD takes a contiguous eighth
    if (((int)blockIdx.x >> 3) >= per || id >= nb) return;
    const int tn = id % g.tiles_n, tm = id / g.tiles_n;
    const int n0 = tn * S::N, m0 = tm * S::M;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave & 1, wm = wave >> 1, r = lane & 31, c = lane >> 5;
    const uint32_t lds0 = lds_address(dlds);
    const int nk = g.stages;

    // Rows past the matrix read as zeros.  A last stage of W that is half a stage goes on into the next row: X holds zeros there.
    const uint32_t pitch = (uint32_t)g.pitch, qpitch = (uint32_t)g.qpitch, spitch = pitch / 16;
    const int prows = std::min(S::N, g.N - n0), qrows = std::min(S::M, g.M - m0);
    const int pbytes = prows * (int)pitch, qbytes = qrows * (int)qpitch;
    v4i pb = buffer_of(g.P + (int64_t)n0 * pitch, pbytes), qb = buffer_of(g.Q + (int64_t)m0 * qpitch, qbytes);
    const v4i spb = buffer_of(g.sp + (int64_t)n0 * spitch, pbytes / 16);
    v4i sqb = buffer_of(g.sq + (int64_t)m0 * STAGE_SCALES, 0);
    const uint64_t sqstep = (uint64_t)g.M * STAGE_SCALES;
    // Codes: one instruction fills 1 KB, lane l granule l % 8 of row l / 8 holding granule (l % 8) ^ swizzle: 16 rows of one granule lie in
    // different banks.
    auto swizzle = [](const int row) { return (row >> 1) & 7; };
    uint32_t poff[S::PI], qoff[S::QI];
#pragma unroll
    for (int i = 0; i < S::PI; ++i) {
        const int row = 8 * (S::PI * wave + i) + lane / 8;
        poff[i] = (uint32_t)row * pitch + 16u * ((lane % 8) ^ swizzle(row));
    }
#pragma unroll
    for (int i = 0; i < S::QI; ++i) {
        const int row = 8 * (S::QI * wave + i) + lane / 8;
        qoff[i] = (uint32_t)row * qpitch + 16u * ((lane % 8) ^ swizzle(row));
    }
    // scales of X: 256 bytes of what lies together (by two wavefronts where there are more of them, so that all have as many requests in
    // flight); of W: rows of CHUNK_ROW bytes
    constexpr int CL = S::CHUNK_ROW / 4;
    const int qw = wave % (S::SQ / 256);
    const uint32_t spoff = (uint32_t)(lane / CL) * spitch + 4u * (lane % CL);
    auto request = [&](const int kt, const uint32_t slot, const int i) {   // instruction i of stage kt; past the last one zeros are deposited
        if (i == 0) {   // (no branch: the compiler would move the matrix instructions behind it)
            const bool some = kt < nk;
            pb[2] = some ? pbytes : 0;
            qb[2] = some ? qbytes : 0;
            const uint64_t base = (uint64_t)(uintptr_t)(g.sq + (int64_t)m0 * STAGE_SCALES) + (uint64_t)kt * sqstep;
            sqb[0] = (int)(uint32_t)base;
            sqb[1] = (int)(uint32_t)(base >> 32);
            sqb[2] = some ? qrows * STAGE_SCALES : 0;
        }
        const uint32_t at = lds0 + slot, k = (uint32_t)kt * STAGE_BYTES;
        if (i < S::PI) lds_dma16_buffer(pb, poff[i], k, at + (S::PI * wave + i) * 1024);
        else if (i < S::PI + S::QI) lds_dma16_buffer(qb, qoff[i - S::PI], k, at + S::P + (S::QI * wave + i - S::PI) * 1024);
        else lds_dma4_buffer(sqb, 256 * qw + 4 * lane, 0, at + S::P + S::Q + 256 * qw);
    };
    auto request_chunk = [&](const int kt) {   // scales of W of the stages kt .. kt + CHUNK_STAGES - 1
        const uint32_t at = lds0 + S::CHUNKS + (kt / S::CHUNK_STAGES & 1) * S::CHUNK;
#pragma unroll
        for (int i = 0; i < S::CI; ++i) {
            const int row = 64 / CL * (S::CI * wave + i);
            lds_dma4_buffer(spb, spoff, row * spitch + kt * STAGE_SCALES, at + row * S::CHUNK_ROW);
        }
    };
    // granule 4 c + u of a row in quarter u: u flips bits of the address
    const uint32_t slot0 = 16 * ((4 * c) ^ swizzle(r));
    const uint32_t pa = lds0 + (wn * 32 * WP + r) * STAGE_BYTES + slot0, qa = lds0 + S::P + (wm * 32 * WQ + r) * STAGE_BYTES + slot0;
    const uint32_t psa = lds0 + S::CHUNKS + (wn * 32 * WP + r) * S::CHUNK_ROW + 4 * c, qsa = lds0 + S::P + S::Q + (wm * 32 * WQ + r) * STAGE_SCALES + 4 * c;
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
    int sp[WP], sq[WQ];   // scales of a stage
    constexpr int READS = WP + WQ;
    auto read_one = [&](const uint32_t at, const int u, const int i) {
        if (i < WP) fp[u & 1][i] = *(lds_v4i)(uintptr_t)((pa ^ (16 * u)) + at + i * 32 * STAGE_BYTES);
        else fq[u & 1][i - WP] = *(lds_v4i)(uintptr_t)((qa ^ (16 * u)) + at + (i - WP) * 32 * STAGE_BYTES);
    };
    auto read_scales = [&](const int kt, const uint32_t at) {
        const uint32_t chunk = (kt / S::CHUNK_STAGES & 1) * S::CHUNK + (kt % S::CHUNK_STAGES) * STAGE_SCALES;
#pragma unroll
        for (int a = 0; a < WP; ++a) sp[a] = *(lds_int)(uintptr_t)(psa + chunk + a * 32 * S::CHUNK_ROW);
#pragma unroll
        for (int b = 0; b < WQ; ++b) sq[b] = *(lds_int)(uintptr_t)(qsa + at + b * 32 * STAGE_SCALES);
    };
    auto wide = [](const v4i x) { return v8i{x[0], x[1], x[2], x[3], 0, 0, 0, 0}; };   // 4-bit operands are four registers
    auto quarter = [&](const int u, auto &&side) {
#pragma unroll
        for (int s = 0; s < TILES; ++s) {
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
    auto spread = [&](const int s, const int n, auto &&op) {
#pragma unroll
        for (int k = 0; k < n; ++k)
            if (k * TILES / n == s) op(k);
    };
    // Stage kt: quarters 0 to 2 read the fragments of the next quarter; then stage kt + 1 must have landed and every wavefront holds the
    // last fragments of stage kt, so behind the barrier the last quarter reads the first fragments of stage kt + 1 and asks for stage kt + 2
    // in the slot of stage kt.
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        if (st == 0) request_chunk(0);
#pragma unroll
        for (int i = 0; i < S::REQUESTS; ++i) request(st, st * S::STAGE, i);
    }
    SBN_WAIT_VMCNT(S::REQUESTS);
    __syncthreads();
    read_scales(0, 0);
#pragma unroll
    for (int i = 0; i < READS; ++i) read_one(0, 0, i);
    uint32_t at = 0;
    for (int kt = 0; kt < nk; ++kt) {
        const uint32_t next = at ? 0 : S::STAGE;
#pragma unroll
        for (int u = 0; u < 3; ++u)
            quarter(u, [&](const int s) { spread(s, READS, [&](const int k) { read_one(at, u + 1, k); }); });
        SBN_WAIT_VMCNT(0);
        __syncthreads();
        if ((kt + 2) % S::CHUNK_STAGES == 0) request_chunk(kt + 2);   // (past the last row's end: zeros)
        quarter(3, [&](const int s) {
            spread(s, READS, [&](const int k) { read_one(next, 0, k); });
            spread(s, S::REQUESTS, [&](const int k) { request(kt + 2, at, k); });
            if (s == TILES - 1) read_scales(kt + 1, next);   // behind their last use
        });
        at = next;
    }
    SBN_WAIT_VMCNT(0);   // the surplus stages have landed
    __syncthreads();

    // Result: 32 tokens at a time through the idle stages (granules of 16 bytes XOR-swizzled with the row), so that whole rows of the
    // wavefront's outputs leave
    typedef float v4f_u __attribute__((ext_vector_type(4), aligned(4)));
    uint8_t *const stg = dlds + wave * 32 * S::OUT;
    constexpr int LPR = S::OUT / 16, J = 32 * LPR / 64, SWIZZLE = LPR < 16 ? LPR - 1 : 15;
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
                *reinterpret_cast<v4f *>(stg + r * S::OUT + 16 * ((8 * a + 2 * q + c) ^ (r & SWIZZLE))) =
                    v4f{acc[a][b][4 * q], acc[a][b][4 * q + 1], acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]};
        asm volatile("" ::: "memory");
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int row = (64 / LPR) * j + lane / LPR, m = mw + 32 * b + row;
            v4f x = *reinterpret_cast<const v4f *>(stg + row * S::OUT + 16 * ((lane % LPR) ^ (row & SWIZZLE)));
            if (g.bias) x += bias;
            if (m >= g.M) continue;
            float *const to = g.Y + (int64_t)m * g.N + n;
            if (n + 4 <= g.N) {
                if (S::PAST_CACHES) __builtin_nontemporal_store(x, reinterpret_cast<v4f_u *>(to));
                else *reinterpret_cast<v4f_u *>(to) = x;
            } else
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (n + i < g.N) to[i] = x[i];
        }
    }
}

template <class S> int64_t tile_blocks(int64_t N, int64_t M) { return ceil_div(ceil_div(N, S::N) * ceil_div(M, S::M), 8) * 8; }

template <class S>
sbn_status launch_tile(MxArgs g, hipStream_t stream)
{
    g.tiles_n = (int)ceil_div(g.N, S::N);
    g.tiles_m = (int)ceil_div(g.M, S::M);
    static thread_local bool raised = false;
    if (!raised) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&mxfp4_tile_kernel<S>), hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
        if (e != hipSuccess) { set_hip_error(e, "hipFuncSetAttribute"); return SBN_EHIP; }
        raised = true;
    }
    hipLaunchKernelGGL(mxfp4_tile_kernel<S>, dim3((unsigned)tile_blocks<S>(g.N, g.M)), dim3(64 * S::WAVES), S::LDS, stream, g);
    return check_launch("mxfp4_tile_kernel");
}

// ---- few tokens ---------------------------------------------------------------------------------------------------------------------------
// The same product where W is what has to be moved: a block takes 32 rows of W at a time, its wavefronts share the dimensions in stages of 256,
// and their sums meet in LDS.  A wavefront's stages of W come by LDS-DMA into a part of its own (whole lines are asked for; a lane's operands lie in 32
// rows), two at a time, without a barrier; the tokens' operands are read from the L2 into registers.  Quantizing them here as well, by the lane that
// multiplies them, cost more than the launch it saved (one token x 2560 -> 6912: 8.6 us against 6.2, -> 131072: 46 against 30).
// 2560 -> 131072 takes 28 us at one token, 6.3 TB/s of codes and scales: the read stream of the board; -> 6912 at 32 tokens 5.0, a launch and its chain.

constexpr int FEW_ROWS = 32, FEW_STAGE = FEW_ROWS * (STAGE_BYTES + STAGE_SCALES), FEW_PITCH = FEW_ROWS + 4;
constexpr int FEW_WAVES = 8, LDS_BYTES = 160 * 1024;
int few_lds(int tokens) { return 2 * FEW_STAGE + 2 * tokens * FEW_PITCH * 4; }   // of a wavefront: two stages, its sums of two tiles

template <int TG>
__global__ void __launch_bounds__(512) mxfp4_few_kernel(MxArgs g)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t dlds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int r = lane & 31, c = lane >> 5;
    const uint32_t pitch = (uint32_t)g.pitch, spitch = pitch / 16;
    const int stages = g.stages;
    const int tiles = (g.N + FEW_ROWS - 1) / FEW_ROWS;
    const uint32_t lds0 = lds_address(dlds) + wave * 2 * FEW_STAGE;
    float *const sums = reinterpret_cast<float *>(dlds + waves * 2 * FEW_STAGE);   // [2][waves][g.M][FEW_PITCH]
    uint32_t off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = 8 * i + (lane >> 3);
        off[i] = (uint32_t)row * pitch + 16u * ((lane & 7) ^ ((row >> 1) & 7));
    }
    const uint32_t soff = (uint32_t)(lane >> 1) * spitch + 4u * (lane & 1);
    // W of a stage, to buffer e
    auto request = [&](const int tile, const int st, const int e) {
        const int64_t o0 = (int64_t)tile * FEW_ROWS;
        const int rows = std::min(FEW_ROWS, g.N - (int)o0);
        const v4i pb = buffer_of(g.P + o0 * pitch, rows * (int)pitch), spb = buffer_of(g.sp + o0 * spitch, rows * (int)spitch);
#pragma unroll
        for (int i = 0; i < 4; ++i) lds_dma16_buffer(pb, off[i], (uint32_t)st * STAGE_BYTES, lds0 + e * FEW_STAGE + i * 1024);
        lds_dma4_buffer(spb, soff, (uint32_t)st * STAGE_SCALES, lds0 + e * FEW_STAGE + FEW_ROWS * STAGE_BYTES);
    };
    v4i q[2][TG][4], p[2][4];
    int sq[2][TG], sp[2];
    // the tokens' operands of a stage
    auto load_tokens = [&](const int st, const int e) {
#pragma unroll
        for (int i = 0; i < TG; ++i) {
            const int64_t t = std::min(32 * i + r, g.M - 1);   // past the last the last one again
            const uint8_t *const row = g.Q + t * g.qpitch + st * STAGE_BYTES + 64 * c;
#pragma unroll
            for (int u = 0; u < 4; ++u) q[e][i][u] = *reinterpret_cast<const v4i *>(row + 16 * u);
            sq[e][i] = *reinterpret_cast<const int *>(g.sq + ((int64_t)st * g.M + t) * STAGE_SCALES + 4 * c);
        }
    };
    typedef __attribute__((address_space(3))) const v4i *lds_v4i;
    typedef __attribute__((address_space(3))) const int *lds_int;
    auto read_words = [&](const int e) {
        const uint32_t at = lds0 + e * FEW_STAGE;
#pragma unroll
        for (int u = 0; u < 4; ++u) p[e][u] = *(lds_v4i)(uintptr_t)(at + r * 128 + 16 * ((4 * c + u) ^ ((r >> 1) & 7)));
        sp[e] = *(lds_int)(uintptr_t)(at + FEW_ROWS * STAGE_BYTES + 8 * r + 4 * c);
    };
    v16f acc[TG];
    auto wide = [](const v4i x) { return v8i{x[0], x[1], x[2], x[3], 0, 0, 0, 0}; };
    auto multiply = [&](const int e) {
#pragma unroll
        for (int i = 0; i < TG; ++i) {
            acc[i] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(p[e][0]), wide(q[e][i][0]), acc[i], 4, 4, 0, sp[e], 0, sq[e][i]);
            acc[i] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(p[e][1]), wide(q[e][i][1]), acc[i], 4, 4, 1, sp[e], 1, sq[e][i]);
            acc[i] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(p[e][2]), wide(q[e][i][2]), acc[i], 4, 4, 2, sp[e], 2, sq[e][i]);
            acc[i] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(p[e][3]), wide(q[e][i][3]), acc[i], 4, 4, 3, sp[e], 3, sq[e][i]);
        }
    };
    // A wavefront's stages wave, wave + waves, ... of a tile, two at a time
    auto request_two = [&](const int tile, const int st) {
        request(tile, st, 0);
        if (st + waves < stages) request(tile, st + waves, 1);
    };
    const bool kept = stages <= 2 * waves;   // the tokens' operands stay in registers from tile to tile
    int tile = blockIdx.x;
    request_two(tile, wave);
    for (int parity = 0; tile < tiles; tile += gridDim.x, parity ^= 1) {
#pragma unroll
        for (int i = 0; i < TG; ++i)
#pragma unroll
            for (int x = 0; x < 16; ++x) acc[i][x] = 0.0f;
        for (int st = wave; st < stages; st += 2 * waves) {
            const bool two = st + waves < stages;
            if (!kept || tile == (int)blockIdx.x) {
                load_tokens(st, 0);
                if (two) load_tokens(st + waves, 1);
            }
            SBN_WAIT_VMCNT(0);
            asm volatile("" ::: "memory");   // the words have landed
            read_words(0);
            if (two) read_words(1);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // and are out of LDS before the next ones are asked for
            if (st + 2 * waves < stages) request_two(tile, st + 2 * waves);
            else if (tile + (int)gridDim.x < tiles) request_two(tile + gridDim.x, wave);
            multiply(0);
            if (two) multiply(1);
        }
        float *const part = sums + (parity * waves + wave) * g.M * FEW_PITCH;
#pragma unroll
        for (int i = 0; i < TG; ++i)
            if (32 * i + r < g.M)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    *reinterpret_cast<v4f *>(part + (32 * i + r) * FEW_PITCH + 8 * x + 4 * c) = v4f{acc[i][4 * x], acc[i][4 * x + 1], acc[i][4 * x + 2], acc[i][4 * x + 3]};
        // (asynchronous loads go on: no __syncthreads, which would wait for them.  One barrier per tile: the sums of the tile after the next
        // one are written behind the next one's barrier)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        typedef float v4f_u __attribute__((ext_vector_type(4), aligned(4)));
        for (int at = threadIdx.x; at < 8 * g.M; at += blockDim.x) {
            const int t = at >> 3, n = 4 * (at & 7);
            v4f x = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int w = 0; w < waves; ++w) x += *reinterpret_cast<const v4f *>(sums + ((parity * waves + w) * g.M + t) * FEW_PITCH + n);
            const int o = tile * FEW_ROWS + n;
            float *const to = g.Y + (int64_t)t * g.N + o;
            if (o + 4 <= g.N) {
                if (g.bias) x += *reinterpret_cast<const v4f_u *>(g.bias + o);
                *reinterpret_cast<v4f_u *>(to) = x;
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (o + i < g.N) to[i] = x[i] + (g.bias ? g.bias[o + i] : 0.0f);
            }
        }
    }
}

template <int TG>
sbn_status launch_few(const MxArgs &g, hipStream_t stream)
{
    // as many wavefronts as have the same number of stages, up to eight, or as many as LDS has room for
    const int most = std::min(FEW_WAVES, LDS_BYTES / few_lds(g.M)), waves = (int)ceil_div(g.stages, ceil_div(g.stages, most));
    static thread_local bool raised = false;
    if (!raised) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&mxfp4_few_kernel<TG>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS_BYTES);
        if (e != hipSuccess) { set_hip_error(e, "hipFuncSetAttribute"); return SBN_EHIP; }
        raised = true;
    }
    // as many blocks as fit the device, with the same number of tiles each
    const int lds = waves * few_lds(g.M), fit = std::max(1, std::min(LDS_BYTES / lds, 16 / waves));
    const int64_t tiles = ceil_div(g.N, FEW_ROWS), rounds = ceil_div(tiles, 256 * fit);
    hipLaunchKernelGGL(mxfp4_few_kernel<TG>, dim3((unsigned)ceil_div(tiles, rounds)), dim3(64 * waves), lds, stream, g);
    return check_launch("mxfp4_few_kernel");
}

std::atomic<int> g_tiles{-1};   // of the test hook

int64_t padded(int64_t cols) { return ceil_div(cols, PAD) * PAD; }

}  // namespace

void set_mxfp4_tiles(int size) { g_tiles.store(size, std::memory_order_relaxed); }

void mxfp4_bytes(int64_t rows, int64_t cols, size_t &codes, size_t &scales)
{
    codes = (size_t)(rows * padded(cols) / 2);
    scales = (size_t)(rows * padded(cols) / GROUP);
}

// X in the workspace: rows of whole stages (256 columns) of codes, then the scales stage by stage
static int64_t stages_of(int64_t d_in) { return ceil_div(d_in, 256); }
static size_t x_code_bytes(int64_t tokens, int64_t d_in) { return align_up((size_t)(tokens * stages_of(d_in) * STAGE_BYTES), 256); }
size_t mxfp4_workspace_bytes(int64_t tokens, int64_t d_in)
{
    return x_code_bytes(tokens, d_in) + align_up((size_t)(tokens * stages_of(d_in) * STAGE_SCALES), 256);
}

// Bound by what they move.  131072 x 2560 of bf16, us with 1 / 2 / 4 vectors per lane: quantize 177 / 169 / 180 (5.0 TB/s, what a copy reaches), back
// 150 / 134 / 131 (6.5); few blocks keep one vector per lane
template <bool BF16>
static void launch_quantize(const void *X, int64_t rows, int64_t cols, int64_t vectors, uint8_t *codes, uint8_t *scales, int stage_shift, hipStream_t stream)
{
    uint32_t *const words = reinterpret_cast<uint32_t *>(codes);
    const int64_t blocks = ceil_div(rows * vectors, 256);
    if (blocks >= 4096)
        hipLaunchKernelGGL((mxfp4_quantize_kernel<BF16, 2>), dim3((unsigned)ceil_div(blocks, 2)), dim3(256), 0, stream, X, (uint32_t)rows, (int)cols, (uint32_t)vectors, words,
                           scales, stage_shift);
    else
        hipLaunchKernelGGL((mxfp4_quantize_kernel<BF16, 1>), dim3((unsigned)blocks), dim3(256), 0, stream, X, (uint32_t)rows, (int)cols, (uint32_t)vectors, words, scales,
                           stage_shift);
}

sbn_status launch_mxfp4_quantize(const void *X, sbn_dtype dtype, int64_t rows, int64_t cols, uint8_t *codes, uint8_t *scales, hipStream_t stream)
{
    if (dtype == SBN_BF16) launch_quantize<true>(X, rows, cols, padded(cols) / 8, codes, scales, 0, stream);
    else launch_quantize<false>(X, rows, cols, padded(cols) / 8, codes, scales, 0, stream);
    return check_launch("mxfp4_quantize_kernel");
}

template <bool BF16>
static void launch_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *Y, hipStream_t stream)
{
    const uint32_t *const words = reinterpret_cast<const uint32_t *>(codes);
    const int64_t blocks = ceil_div(rows * (cols / 8), 256);
    const uint32_t vectors = (uint32_t)(padded(cols) / 8);
    if (blocks >= 4096)
        hipLaunchKernelGGL((mxfp4_dequantize_kernel<BF16, 4>), dim3((unsigned)ceil_div(blocks, 4)), dim3(256), 0, stream, words, scales, (uint32_t)rows, (uint32_t)cols, vectors, Y);
    else
        hipLaunchKernelGGL((mxfp4_dequantize_kernel<BF16, 1>), dim3((unsigned)blocks), dim3(256), 0, stream, words, scales, (uint32_t)rows, (uint32_t)cols, vectors, Y);
}

sbn_status launch_mxfp4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *Y, sbn_dtype dtype, hipStream_t stream)
{
    if (dtype == SBN_BF16) launch_dequantize<true>(codes, scales, rows, cols, Y, stream);
    else launch_dequantize<false>(codes, scales, rows, cols, Y, stream);
    return check_launch("mxfp4_dequantize_kernel");
}

// Estimated us of a product in tiles of one size: one tile alone, or every multiprocessor's share of them, `each` us of the multiprocessor.  The
// figures are fits to products of 65 to 8192 tokens, 1000 -> 20000, 2560 -> 6912 and 131072, 4096 -> 4096 (2560 -> 6912, us, small / middle /
// large: 128 tokens 10.4 / 14.7 / 24.1, 512 21.3 / 18.7 / 28.6, 4096 110 / 81 / 68).  A launch has fewer than 2^32 threads, so some 2^36 outputs and
// more do not go to the small tiles (the large ones have room for all that a call takes).
template <class S>
static float tiles_us(const int64_t N, const int64_t M, const float alone, const float each)
{
    if (tile_blocks<S>(N, M) * 64 * S::WAVES >= (int64_t)1 << 32) return INFINITY;
    return std::max(alone, each * (float)ceil_div(ceil_div(N, S::N) * ceil_div(M, S::M), 256));
}

// 0, 1, 2: small, middle, large tiles
static int choose_tile(const int64_t N, const int64_t M, const int64_t stages)
{
    const float large = tiles_us<MxLarge>(N, M, 1.05f * stages + 12.0f, 1.44f * stages + 16.0f), middle = tiles_us<MxMiddle>(N, M, 0.65f * stages + 6.2f, 0.48f * stages + 6.5f),
                small = tiles_us<MxSmall>(N, M, 0.38f * stages + 4.6f, 0.28f * stages + 1.1f);
    return large <= std::min(middle, small) ? 2 : middle <= small ? 1 : 0;
}

int64_t mxfp4_tile_threads(int64_t tokens, int64_t d_in, int64_t d_out, int *size)
{
    *size = choose_tile(d_out, tokens, stages_of(d_in));
    return *size == 0 ? tile_blocks<MxSmall>(d_out, tokens) * 64 * MxSmall::WAVES
                      : *size == 1 ? tile_blocks<MxMiddle>(d_out, tokens) * 64 * MxMiddle::WAVES : tile_blocks<MxLarge>(d_out, tokens) * 64 * MxLarge::WAVES;
}

sbn_status launch_mxfp4_linear(const void *X, int64_t tokens, int64_t d_in, int64_t d_out, const uint8_t *codes, const uint8_t *scales, const float *bias,
                               float *Y, void *workspace, hipStream_t stream)
{
    const int64_t stages = stages_of(d_in);
    uint8_t *const xc = static_cast<uint8_t *>(workspace), *const xs = xc + x_code_bytes(tokens, d_in);
    launch_quantize<true>(X, tokens, d_in, stages * 32, xc, xs, 8, stream);
    const sbn_status st = check_launch("mxfp4_quantize_kernel");
    if (st != SBN_OK) return st;
    MxArgs g{codes, xc, scales, xs, padded(d_in) / 2, stages * STAGE_BYTES, (int)d_out, (int)tokens, (int)stages, bias, Y, 0, 0};
    // 64 tokens, few and small tiles: 2560 -> 6912 8.9 and 10.4 us, 4096 -> 4096 10.8 and 12.6
    const int forced = g_tiles.load(std::memory_order_relaxed);
    if (tokens <= 32 && forced < 0) return launch_few<1>(g, stream);
    if (tokens <= 64 && forced < 0) return launch_few<2>(g, stream);
    const int size = forced >= 0 ? forced : choose_tile(g.N, g.M, stages);
    return size == 0 ? launch_tile<MxSmall>(g, stream) : size == 1 ? launch_tile<MxMiddle>(g, stream) : launch_tile<MxLarge>(g, stream);
}

}  // namespace sbn
