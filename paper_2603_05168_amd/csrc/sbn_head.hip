// The output head in training: softmax cross entropy and distillation from a teacher's top logits over a vocabulary, without keeping
// the logits.  H [tokens, d] and W [vocab, d] are bf16, z = H W^T, and per token t
//   ce = lse(z) - z_y,                                         lse(x) = log sum_v exp x_v
//   kd = tau^2 sum_v q_v (log q_v - (z_v / tau - lse(z / tau))),   q = softmax(a / tau) over the teacher's entries
//   G  = d_ce (softmax(z) - onehot(y)) + d_kd tau (softmax(z / tau) - q),   dH = G W,   dW = G^T H
// Forward: one product whose tiles leave a maximum and sums of exponentials per token and the words of a wavefront (128, 64 or 32); they
// are joined in a fixed order.  Backward: the vocabulary is cut into pieces; the logits of a piece are made once more, turned into G (bf16) on their
// way out, and both gradients' products read G.  All products run on the bf16 matrix cores (v_mfma_f32_32x32x16_bf16, fp32
// accumulation).  Nothing is added atomically: results do not depend on the order of blocks.
#include <algorithm>
#include <atomic>

#include "sbn_internal.hpp"
#include "sbn_mfma.hpp"

namespace sbn {

namespace {

constexpr float LOG2E = 1.4426950408889634f;

// two values rounded to bf16 (to nearest, ties to even), lo in the low half: v_cvt_pk_bf16_f32
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v2f{lo, hi}, v2bf));
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }   // v_exp_f32: 1 ulp

// ---- block tile product -------------------------------------------------------------------------------------------------------------
// acc[n, m] = sum_k P[n, k] Q[m, k] for a block tile of 256 x 256 (eight wavefronts of 128 x 64), 128 x 128 (four of 64 x 64, two blocks per
// multiprocessor) or 64 x 64 (four of 32 x 32, two blocks).  Either operand lies with k contiguous ([rows, ld]) or the other way round ([k, ld],
// "transposed": read from LDS by ds_read_b64_tr_b16).  Stages of 64 k come by LDS-DMA into a ring of 2 AHEAD + 1 slots that the operands
// take in turns, so that P lies in LDS AHEAD stages ahead and Q one less; a stage is consumed in quarters of 16 k, the fragments of the next
// quarter are read and the requests for later stages issued between the matrix instructions of the current one.
constexpr int STAGE_K = 64;
enum { TINY, SMALL, BIG };
template <int SIZE> struct HeadTile {
    static constexpr int N = SIZE == BIG ? 256 : SIZE == SMALL ? 128 : 64, M = N;
    static constexpr int WAVES = SIZE == BIG ? 8 : 4, WN = 2, WM = WAVES / WN;   // wavefronts along n and m
    static constexpr int WP = N / WN / 32, WQ = M / WM / 32;                     // 32 x 32 tiles of a wavefront: 4 x 2, 2 x 2 or 1 x 1
    static constexpr int AHEAD = SIZE == TINY ? 4 : 2;
    static constexpr int SLOT = N * STAGE_K * 2, SLOTS = 2 * AHEAD + 1;          // one operand's share of a stage
    static constexpr int REQUESTS = SLOT / (1024 * WAVES);                       // of a wavefront, operand and stage
    static constexpr int LDS = SLOTS * SLOT;
    // results leave through the ring's last slot, some rows (columns m) of a wavefront at a time: a next tile's first stages may be in the others
    static constexpr int ROW = WP * 128, STAGING = SLOT / WAVES, ROWS = STAGING / ROW;
    static constexpr int STAGED = (SLOTS - 1) * SLOT;
};

// The lane, as a value that the compiler knows nothing of: what a tile's parts derive from it is made again in each of them, for all of it at once
// does not fit the registers
__device__ __forceinline__ int lane_here()
{
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}

struct Operand {
    const uint16_t *base;   // row 0, k 0
    int64_t ld;
    int rows, k;            // what the matrix has (k: from the product's first k on)
};

// The requests of one operand: instructions of 1 KB.  Rows and k past the matrix read as zeros or as what zero_tail overwrites; stages past the
// last fetch nothing.  A buffer's size has 32 bits and ends with the rows of the tile.
template <int SIZE, bool TRANSPOSED> struct Requests {
    using S = HeadTile<SIZE>;
    static constexpr int I = S::REQUESTS;
    v4i buffer;
    uint32_t off[I], bytes, bytes_last;
    uint64_t step;
    int nk, kleft, wave;

    __device__ __forceinline__ void set(const Operand &op, int row0, int nk_, int wave_, int lane)
    {
        nk = __builtin_amdgcn_readfirstlane(nk_);
        wave = wave_;
        const uint32_t pitch = 2u * (uint32_t)op.ld;
        kleft = op.k - (nk - 1) * STAGE_K;
        kleft = kleft < STAGE_K ? kleft : STAGE_K;
        if constexpr (TRANSPOSED) {
            // a stage is 64 k rows of S::N values; slot s of row k holds granule s ^ f(k), f = 4 (k & 3) | 2 ((k >> 2) & 1): the four k rows that a
            // transposing read of 16 lanes takes lie in different banks
            auto up_to_end = [&](const int k) { return (uint32_t)std::min((uint64_t)k * pitch - 2u * (uint32_t)row0, (uint64_t)0xfffffff0u); };
            bytes = up_to_end(STAGE_K);
            bytes_last = up_to_end(kleft);
            step = (uint64_t)op.ld * (STAGE_K * 2);
            asm volatile("" : "+s"(step));
            buffer = buffer_of(op.base + row0, nk > 1 ? bytes : bytes_last);
            constexpr int GPR = S::N / 8, RPI = 64 / GPR;   // granules of a k row, k rows per instruction
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const int k = RPI * (I * wave + i) + lane / GPR;
                const int gran = (lane % GPR) ^ (4 * (k & 3) | 2 * ((k >> 2) & 1)) % GPR;
                off[i] = (uint32_t)k * pitch + 16u * gran;
            }
        } else {
            // one instruction fills 8 rows x 128 bytes: lane l row l / 8, slot l % 8 holding granule slot ^ ((row >> 1) & 7)
            const int rows = op.rows - row0 < S::N ? op.rows - row0 : S::N;
            bytes = (uint32_t)(rows - 1) * pitch + 2 * STAGE_K;
            bytes_last = (uint32_t)(rows - 1) * pitch + 2 * kleft;
            step = 2 * STAGE_K;
            buffer = buffer_of(op.base + (int64_t)row0 * op.ld, nk > 1 ? bytes : bytes_last);
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const int row = 8 * (I * wave + i) + (lane >> 3);
                off[i] = (uint32_t)row * pitch + 16u * ((lane & 7) ^ ((row >> 1) & 7));
            }
        }
    }
    // instruction i of stage kt; the last one moves on to the next stage
    __device__ __forceinline__ void issue(const int kt, const uint32_t slot, const int i)
    {
        lds_dma16_buffer(buffer, off[i], 0, slot + (I * wave + i) * 1024);
        if (i + 1 < I) return;
        const uint64_t base = ((uint64_t)(uint32_t)buffer[1] << 32 | (uint32_t)buffer[0]) + step;
        // (the same in all lanes; where the compiler does not see it, it would not hold them in scalar registers)
        buffer[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)base);
        buffer[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32));
        buffer[2] = __builtin_amdgcn_readfirstlane(kt + 2 < nk ? (int)bytes : kt + 2 == nk ? (int)bytes_last : 0);
    }
    // k of the last stage past a row's end: the next row was fetched in their place.  A lane overwrites what it asked for itself, behind
    // its own wait and in front of the barrier that publishes the stage.
    __device__ __forceinline__ void zero_tail(const uint32_t slot) const
    {
        if constexpr (TRANSPOSED) return;
        typedef __attribute__((address_space(3))) v4i *lds_v4i;
        const int lane = lane_here();   // (volatile: not in front of the wait)
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int k = 8 * ((lane & 7) ^ (((8 * (I * wave + i) + (lane >> 3)) >> 1) & 7));
            if (k >= kleft) *(lds_v4i)(uintptr_t)(slot + (I * wave + i) * 1024 + 16 * lane) = v4i{0, 0, 0, 0};
        }
    }
};

// The fragments of one operand: W tiles of 32 rows, eight k of a row per lane.
template <int SIZE, bool TRANSPOSED, int W> struct Fragments {
    using S = HeadTile<SIZE>;
    typedef __attribute__((address_space(3))) const v8bf *lds_v8bf;
    typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) v4bf *lds_v4bf;
    static constexpr int READS = TRANSPOSED ? 2 * W : W, ADDRESSES = TRANSPOSED ? 2 * W : 4;
    uint32_t at[ADDRESSES];
    v8bf f[2][W];

    __device__ __forceinline__ Fragments(const uint32_t slot, const int part, const int lane)   // part: of the tile's rows, 32 W each
    {
        const int r = lane & 31, c = lane >> 5;
        if constexpr (TRANSPOSED) {
            // lane l of a group of 16 supplies the address of k row k0 + (l >> 2), columns 4 (l & 3) .. + 3 and gets four k of column l;
            // two reads (h = 0, 1) make the eight k of a fragment
            const int rr = (lane & 15) >> 2;
#pragma unroll
            for (int b = 0; b < W; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int gran = (part * 32 * W + 32 * b) / 8 + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
                    at[2 * b + h] = slot + (8 * c + 4 * h + rr) * (2 * S::N) + 16 * (gran ^ (4 * rr | 2 * h) % (S::N / 8)) + 8 * (lane & 1);
                }
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u) at[u] = slot + (part * 32 * W + r) * 128 + 16 * ((2 * u + c) ^ ((r >> 1) & 7));
        }
    }
    __device__ __forceinline__ void read(const int u, const int i)   // read i of quarter u
    {
        if constexpr (TRANSPOSED) {
            const v4bf v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_v4bf)(uintptr_t)(at[i] + 16 * u * (2 * S::N)));
            if (i & 1) f[u & 1][i >> 1].hi = v; else f[u & 1][i >> 1].lo = v;
        } else {
            f[u & 1][i] = *(lds_v8bf)(uintptr_t)(at[u] + i * 32 * 128);
        }
    }
    __device__ __forceinline__ void move(const uint32_t by)
    {
#pragma unroll
        for (int i = 0; i < ADDRESSES; ++i) at[i] += by;
    }
};

// A tile's product in two parts, so that a block that takes one tile after the other asks for a tile's first stages in front of the last one's
// results: begin, then run.
template <int SIZE, bool PT, bool QT> struct TileProduct {
    using S = HeadTile<SIZE>;
    static constexpr int WP = S::WP, WQ = S::WQ, TILES = WP * WQ, I = S::REQUESTS, D = S::AHEAD;
    Requests<SIZE, PT> rp;
    Requests<SIZE, QT> rq;
    int nk;

    __device__ __forceinline__ void begin(const Operand &p, const Operand &q, const int n0, const int m0, const int stages, uint8_t *lds)
    {
        const int lane = lane_here(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint32_t lds0 = lds_address(lds);
        nk = stages;
        rp.set(p, n0, nk, wave, lane);
        rq.set(q, m0, nk, wave, lane);
#pragma unroll
        for (int j = 0; j < 2 * D; ++j)
#pragma unroll
            for (int i = 0; i < I; ++i) {
                if (j & 1) rq.issue(j >> 1, lds0 + j * S::SLOT, i);
                else rp.issue(j >> 1, lds0 + j * S::SLOT, i);
            }
    }

    __device__ __forceinline__ void run(uint8_t *lds, v16f (&acc)[WP][WQ])
    {
        const int lane = lane_here(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint32_t lds0 = lds_address(lds);
        Fragments<SIZE, PT, WP> fp(lds0, wave & 1, lane);
        Fragments<SIZE, QT, WQ> fq(lds0 + S::SLOT, wave >> 1, lane);
        constexpr int READS = fp.READS + fq.READS;
#pragma unroll
        for (int a = 0; a < WP; ++a)
#pragma unroll
            for (int b = 0; b < WQ; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;
        auto read_one = [&](const int u, const int i) {
            if (i < fp.READS) fp.read(u, i);
            else fq.read(u, i - fp.READS);
        };
        auto advance = [](const uint32_t slot) { return slot < (S::SLOTS - 2u) * S::SLOT ? slot + 2u * S::SLOT : slot - (S::SLOTS - 2u) * S::SLOT; };   // two slots further on
        // a quarter step: side(s) is issued after instruction s; the source order is the intended issue order
        auto quarter = [&](const int u, auto &&side) {
#pragma unroll
            for (int s = 0; s < TILES; ++s) {
                const int a = s / WQ, b = s % WQ;
                acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp.f[u & 1][a], fq.f[u & 1][b], acc[a][b], 0, 0, 0);
                side(s);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto spread = [&](const int s, const int n, auto &&op) {   // operations [0, n) over the instructions of a quarter step
#pragma unroll
            for (int k = 0; k < n; ++k)
                if (k * TILES / n == s) op(k);
        };
        // The ring holds P(0), Q(0), P(1), Q(1), ...  Step kt: quarters 0 to 2 read the fragments of the next quarter; then stage kt + 1 must have
        // landed and every wavefront holds the last fragments of stage kt, so behind the barrier the last quarter reads the first fragments of
        // stage kt + 1 and asks for Q(kt + D) in the slot of P(kt), and the first two quarters of the next step for P(kt + D + 1) in that of Q(kt).
        SBN_WAIT_VMCNT((2 * D - 2) * I);   // (what was issued behind begin is waited for as well)
        asm volatile("" ::: "memory");
        if (nk == 1) {
            if (rp.kleft < STAGE_K) rp.zero_tail(lds0);
            if (rq.kleft < STAGE_K) rq.zero_tail(lds0 + S::SLOT);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < READS; ++i) read_one(0, i);
        uint32_t sp = 0, sq = S::SLOT;
        for (int kt = 0; kt < nk; ++kt) {
            const uint32_t sp_next = advance(sp), sq_next = advance(sq);
            const uint32_t free = sp ? sp - S::SLOT : (S::SLOTS - 1u) * S::SLOT;   // of Q(kt - 1)
#pragma unroll
            for (int u = 0; u < 3; ++u)
                quarter(u, [&](const int s) {
                    spread(s, READS, [&](const int k) { read_one(u + 1, k); });
                    if (u < 2) spread(s, I / 2, [&](const int k) { rp.issue(kt + D, lds0 + free, I / 2 * u + k); });
                });
            SBN_WAIT_VMCNT((2 * D - 3) * I);   // P(kt + 2) and what follows it may fly
            if (kt + 2 == nk) {
                if (rp.kleft < STAGE_K) rp.zero_tail(lds0 + sp_next);
                if (rq.kleft < STAGE_K) rq.zero_tail(lds0 + sq_next);
            }
            __syncthreads();
            fp.move(sp_next - sp);
            fq.move(sq_next - sq);
            quarter(3, [&](const int s) {
                spread(s, READS, [&](const int k) { read_one(0, k); });
                spread(s, I, [&](const int k) { rq.issue(kt + D, lds0 + sp, k); });
            });
            sp = sp_next;
            sq = sq_next;
        }
        SBN_WAIT_VMCNT(0);   // the surplus stages have landed
        __syncthreads();
    }
};

// Part of a wavefront's columns b of its result to its part of LDS in fp32: ROWS columns m from 32 b + first on become rows, granules of 16 bytes
// (four n) XOR-swizzled with the row.
template <int SIZE, int ROWS>
__device__ __forceinline__ void stage_columns(const v16f (&acc)[HeadTile<SIZE>::WP][HeadTile<SIZE>::WQ], const int b, const int first, uint8_t *stg, const int lane)
{
    using S = HeadTile<SIZE>;
    constexpr int SWIZZLE = S::ROW / 16 < 16 ? S::ROW / 16 - 1 : 15;
    const int r = (lane & 31) - first, c = lane >> 5;
    asm volatile("" ::: "memory");   // behind the last columns' reads
    if (ROWS == 32 || (r >= 0 && r < ROWS))
#pragma unroll
        for (int a = 0; a < S::WP; ++a)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<v4f *>(stg + r * S::ROW + 16 * ((8 * a + 2 * q + c) ^ (r & SWIZZLE))) =
                    v4f{acc[a][b][4 * q], acc[a][b][4 * q + 1], acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]};
    asm volatile("" ::: "memory");   // the reads are of what other lanes have written
}
template <int SIZE>
__device__ __forceinline__ float *staged(uint8_t *stg, const int row, const int n)
{
    constexpr int SWIZZLE = HeadTile<SIZE>::ROW / 16 < 16 ? HeadTile<SIZE>::ROW / 16 - 1 : 15;
    return reinterpret_cast<float *>(stg + row * HeadTile<SIZE>::ROW + 16 * ((n >> 2) ^ (row & SWIZZLE)) + 4 * (n & 3));
}
// Tile order: consecutive tiles form super-tiles of 8 x 8
__device__ __forceinline__ void tile_in_order(const int tiles_n, const int tiles_m, const int id, int &tn, int &tm)
{
    const int band_tiles = 8 * tiles_n;
    const int nbands = (tiles_m + 7) >> 3;
    int band = id / band_tiles;
    band = band < nbands - 1 ? band : nbands - 1;
    const int h = band == nbands - 1 ? tiles_m - 8 * band : 8;      // tile rows of this band
    const int rem = id - band * band_tiles;
    const int ncols = (tiles_n + 7) >> 3;
    int col = rem / (8 * h);
    col = col < ncols - 1 ? col : ncols - 1;
    const int rem2 = rem - col * 8 * h;
    tn = 8 * col + rem2 / h;
    tm = 8 * band + rem2 % h;
}
// Blocks go to the eight XCDs round-robin and every XCD has its own L2, so XCD x takes a contiguous eighth of `all` in order.  The numbers that pad
// them to a multiple of eight get one past the end.
__device__ __forceinline__ int place_of_block(const int all, const int bid)
{
    const int per = (all + 7) >> 3, at = bid >> 3;
    return at < per ? (bid & 7) * per + at : all;
}
__device__ __forceinline__ bool tile_of_block(const int tiles_n, const int tiles_m, const int bid, int &tn, int &tm)
{
    const int id = place_of_block(tiles_n * tiles_m, bid);
    if (id >= tiles_n * tiles_m) return false;
    tile_in_order(tiles_n, tiles_m, id, tn, tm);
    return true;
}

// ---- logits --------------------------------------------------------------------------------------------------------------------------
struct LogitsArgs {
    const uint16_t *H, *W;       // W: the piece's first row
    int tokens, d, words;        // words: rows of W in the piece
    int64_t v0, vocab;           // the piece's first word, words of all pieces
    int tiles_n, tiles_m;
    const int64_t *targets;      // with HARD
    // with SOFT: the teacher's entries (see teacher_kernel)
    const int32_t *at;
    const float *q;
    const uint32_t *map;
    const float *some;
    int top_k;
    float tau;
    // forward
    float *m, *s1, *s2;          // [parts, tokens]: maximum, sum of exp(z - m), sum of exp((z - m) / tau)
    float *z_target, *z_top;     // [tokens], [tokens, top_k]
    // backward
    const float *lse1, *lse2, *d1, *d2;
    uint16_t *G;                 // [tokens, ldg]
    uint16_t *rest;              // [tokens, ldg]: what rounding to bf16 left over of G; null: not asked for (tiles of 64 and 128 alone)
    int64_t ldg;
};

// The teacher's entries among the 32 tokens from m on and the wavefront's words from v on: each(row, word - v, entry).  A wavefront asks one bit
// per token and 64 words first; lists are read where it is set only.
template <int WORDS, class Each>
__device__ __forceinline__ void entries_here(const LogitsArgs &g, const uint32_t hits, const int m, const int64_t v, const int lane, Each &&each)
{
    for (uint32_t left = hits; left; left &= left - 1) {
        const int row = __builtin_ctz(left);
        const int64_t first = (int64_t)(m + row) * g.top_k;
        for (int j = lane; j < g.top_k; j += 64) {
            const int64_t n = g.at[first + j] - v;
            if (n >= 0 && n < WORDS) each(row, (int)n, first + j);
        }
    }
}
template <int WORDS>
__device__ __forceinline__ uint32_t rows_with_entries(const LogitsArgs &g, const int t, const int64_t v)
{
    constexpr uint32_t MASK = WORDS == 128 ? 3u : 1u;
    const uint32_t word = t < g.tokens ? g.map[(v >> 11) * g.tokens + t] : 0u;
    return (uint32_t)__ballot((word >> ((v >> 6) & 31)) & MASK);   // the lanes of the upper half hold the same tokens
}

// What d_ce has in common: the significand of the first one of the first 64 tokens that counts.  G is divided by it before it is rounded to bf16 and
// the products' sums are multiplied by it: with one d_ce for all tokens (a mean) -d_ce (1 - p) has the same rounding error in every token,
// which sums keep (0.0039 of the norm of dH and dW at 16384 tokens, 0.0019 this way), whereas -2^e (1 - p) is exact where p is small.  Any
// value in [1, 2) is right; ranges do not change.  Read in front of a product, looked at behind it.
struct CommonFactor {
    int64_t target = -1;
    float d = 0.0f;
    __device__ __forceinline__ CommonFactor(const int64_t *targets, const float *d1, const int tokens)
    {
        const int t = threadIdx.x & 63;
        if (targets && t < tokens) {
            target = targets[t];
            d = d1[t];
        }
    }
    __device__ __forceinline__ float value(const int64_t vocab) const
    {
        const uint32_t bits = __float_as_uint(d) & 0x7fffffffu;
        const uint64_t some = __ballot(target >= 0 && target < vocab && bits >= 0x00800000u && bits < 0x7f800000u);
        return some ? __uint_as_float((__builtin_amdgcn_readlane(bits, __builtin_ctzll(some)) & 0x007fffffu) | 0x3f800000u) : 1.0f;
    }
};

// What two rounded values left over, rounded in turn; nothing of one that has no finite value
__device__ __forceinline__ uint32_t rest_of(const uint32_t rounded, const float lo, const float hi)
{
    const float a = __builtin_bit_cast(float, rounded << 16), b = __builtin_bit_cast(float, rounded & 0xffff0000u);
    return pack_bf16(__builtin_fabsf(a) < INFINITY ? lo - a : 0.0f, __builtin_fabsf(b) < INFINITY ? hi - b : 0.0f);
}

// what belongs to a lane's tokens, asked for in front of a tile's product
template <int WQ, bool GRAD, bool HARD, bool SOFT> struct TokenValues {
    int64_t target[WQ];
    float d1[WQ], lse1[WQ], d2[WQ], lse2[WQ], some[WQ];
    __device__ __forceinline__ void load(const LogitsArgs &g, const int m0)
    {
        const int r = lane_here() & 31;
#pragma unroll
        for (int b = 0; b < WQ; ++b) {
            const int t = std::min(m0 + 32 * b + r, g.tokens - 1);
            if (HARD) target[b] = g.targets[t];
            if (HARD && GRAD) {
                d1[b] = g.d1[t];
                lse1[b] = g.lse1[t];
            }
            if (SOFT && GRAD) {
                d2[b] = g.d2[t];
                lse2[b] = g.lse2[t];
                some[b] = g.some[t];
            }
        }
    }
};

// Forward, a block takes tile after tile, gridDim.x apart: the next one's first stages come in under the sums of the last one (16384 tokens x
// 131072 words x 2560: 8.68 ms with a block per tile, 8.63 so; 1531 x 50001 x 1000 164 us and 160).  Backward, results need LDS: with all of it for
// a block per tile G takes 181 us at 1531 x 50001 x 1000, with the slot that a next tile's first stages leave 206.
// Many tokens are bound by the matrix pipe at the clock that power leaves: 2048 x 32000 x 2560 262 to 296 us (1.13 to 1.28 PFLOP/s, the pipe busy
// in 71 % of the cycles), 16384 tokens x 131072 8.7 ms forward (1.26) and 9.6 in eight pieces backward (1.14), where G leaves; with few dimensions
// a tile's sums and results weigh as much as its product (1531 x 50001 x 1000: 0.9 and 0.87, the pipe busy in 44 % of the backward pass).  One
// token by the stream of W: 131072 x 2560 112 us, 6.0 TB/s.
template <int SIZE, bool GRAD, bool HARD, bool SOFT>
__global__ void __launch_bounds__(64 * HeadTile<SIZE>::WAVES, 2) logits_kernel(LogitsArgs g)
{
    using S = HeadTile<SIZE>;
    constexpr int WP = S::WP, WQ = S::WQ, WORDS = 32 * WP;
    constexpr int LPR = S::ROW / 32;   // G: lanes per row
    constexpr int ROWS = GRAD ? 32 : S::ROWS;                       // staged at a time
    static_assert(S::WAVES * 32 * S::ROW <= S::LDS, "32 columns of every wavefront are staged in the idle ring");
    extern __shared__ __attribute__((aligned(1024))) uint8_t dlds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint8_t *const stg = GRAD ? dlds + wave * 32 * S::ROW : dlds + S::STAGED + wave * S::STAGING;
    const float k1 = LOG2E, k2 = SOFT ? LOG2E / g.tau : 0.0f;
    const int jobs = (g.tiles_n * g.tiles_m + 7) / 8 * 8;
    int job = blockIdx.x, tn, tm;
    auto next_tile = [&] {
        for (; job < jobs; job += gridDim.x)
            if (tile_of_block(g.tiles_n, g.tiles_m, job, tn, tm)) return true;
        return false;
    };
    if (!next_tile()) return;
    TokenValues<WQ, GRAD, HARD, SOFT> now, next;
    TileProduct<SIZE, false, false> product;
    const Operand p{g.W, g.d, g.words, g.d}, q{g.H, g.d, g.tokens, g.d};
    const int stages = (g.d + STAGE_K - 1) / STAGE_K;
    const CommonFactor common(GRAD && HARD ? g.targets : nullptr, g.d1, g.tokens);
    now.load(g, tm * S::M + (wave >> 1) * 32 * WQ);
    product.begin(p, q, tn * S::N, tm * S::M, stages, dlds);
    const float inv = GRAD && HARD ? 1.0f / common.value(g.vocab) : 1.0f;
    for (bool more = true; more;) {
        v16f acc[WP][WQ];
        product.run(dlds, acc);
        const int part = 2 * tn + (wave & 1);
        const int n0 = tn * S::N + (wave & 1) * WORDS;      // of the piece
        const int m0 = tm * S::M + (wave >> 1) * 32 * WQ;
        const int64_t v = g.v0 + n0;
        const int left = g.words - n0;                      // words that the wavefront has
        if constexpr (GRAD) {
            more = false;
        } else {
            job += gridDim.x;
            more = next_tile();
        }
        if (more) {
            next.load(g, tm * S::M + (wave >> 1) * 32 * WQ);
            product.begin(p, q, tn * S::N, tm * S::M, stages, dlds);
        }
        const int lane = lane_here(), r = lane & 31, c = lane >> 5;
#pragma unroll
        for (int b = 0; b < WQ; ++b) {
            const int t = m0 + 32 * b + r;
            const bool inside = t < g.tokens;
            const bool kept = HARD && inside && now.target[b] >= 0 && now.target[b] < g.vocab;
            const int64_t y = kept ? now.target[b] - v : -1;   // relative to the wavefront's words
            const bool here = y >= 0 && y < (left < WORDS ? left : WORDS);
            const uint32_t hits = SOFT ? rows_with_entries<WORDS>(g, t, v) : 0u;
            if constexpr (!GRAD) {
                if (HARD && __any(here)) {
                    float z = 0.0f;
#pragma unroll
                    for (int a = 0; a < WP; ++a)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if ((int)y == 32 * a + 8 * (i >> 2) + 4 * c + (i & 3)) z = acc[a][b][i];
                    if (here && (((int)y >> 2) & 1) == c) g.z_target[t] = z;
                }
                if (SOFT && hits)
#pragma unroll
                    for (int row0 = 0; row0 < 32; row0 += ROWS) {
                        const uint32_t some = hits & ((uint32_t)((1ull << ROWS) - 1) << row0);
                        if (!some) continue;
                        stage_columns<SIZE, ROWS>(acc, b, row0, stg, lane);
                        entries_here<WORDS>(g, some, m0 + 32 * b, v, lane, [&](int row, int n, int64_t e) { g.z_top[e] = *staged<SIZE>(stg, row - row0, n); });
                    }
                if (left < WORDS) {
#pragma unroll
                    for (int a = 0; a < WP; ++a)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (32 * a + 8 * (i >> 2) + 4 * c + (i & 3) >= left) acc[a][b][i] = -INFINITY;
                }
                float most = -INFINITY;
#pragma unroll
                for (int a = 0; a < WP; ++a)
#pragma unroll
                    for (int i = 0; i < 16; ++i) most = fmaxf(most, acc[a][b][i]);
                most = fmaxf(most, __shfl_xor(most, 32));
                const float base = most == -INFINITY ? 0.0f : most;   // no word here: sums of zeros
                const float base1 = base * k1, base2 = base * k2;
                float sum1 = 0.0f, sum2 = 0.0f;
#pragma unroll
                for (int a = 0; a < WP; ++a)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float z = acc[a][b][i];
                        if (HARD) sum1 += exp2_fast(__builtin_fmaf(z, k1, -base1));
                        if (SOFT) sum2 += exp2_fast(__builtin_fmaf(z, k2, -base2));
                    }
                if (HARD) sum1 += __shfl_xor(sum1, 32);
                if (SOFT) sum2 += __shfl_xor(sum2, 32);
                if (inside && c == 0) {
                    const int64_t at = (int64_t)part * g.tokens + t;
                    g.m[at] = most;
                    if (HARD) g.s1[at] = sum1;
                    if (SOFT) g.s2[at] = sum2;
                }
            } else {
                // exp(z - lse) as 2^(z log2 e - lse log2 e); a token without a share has none whatever its lse
                float c1 = 0.0f, c2 = 0.0f, l1 = INFINITY, l2 = INFINITY;
                if (HARD && kept) c1 = now.d1[b] * inv;
                if (HARD && c1 != 0.0f) l1 = now.lse1[b] * LOG2E;
                if (SOFT && inside && now.some[b] != 0.0f) c2 = now.d2[b] * g.tau * inv;
                if (SOFT && c2 != 0.0f) l2 = now.lse2[b] * LOG2E;
#pragma unroll
                for (int a = 0; a < WP; ++a)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float z = acc[a][b][i];
                        float e = 0.0f;
                        if (HARD) e = c1 * exp2_fast(__builtin_fmaf(z, k1, -l1));
                        if (SOFT) e = __builtin_fmaf(c2, exp2_fast(__builtin_fmaf(z, k2, -l2)), e);
                        acc[a][b][i] = e;
                    }
                if (HARD && __any(here)) {
                    const float less = here ? c1 : 0.0f;
#pragma unroll
                    for (int a = 0; a < WP; ++a)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if ((int)y == 32 * a + 8 * (i >> 2) + 4 * c + (i & 3)) acc[a][b][i] -= less;
                }
                stage_columns<SIZE, 32>(acc, b, 0, stg, lane);
                if (SOFT && hits) {
                    entries_here<WORDS>(g, hits, m0 + 32 * b, v, lane, [&](int row, int m, int64_t e) {
                        float *const x = staged<SIZE>(stg, row, m);
                        *x = __builtin_fmaf(-(g.d2[m0 + 32 * b + row] * g.tau * inv), g.q[e], *x);   // every word once per token: no two lanes at one place
                    });
                    asm volatile("" ::: "memory");
                }
                const int n = 8 * (lane % LPR);
#pragma unroll
                for (int j = 0; j < LPR / 2; ++j) {
                    const int row = 64 / LPR * j + lane / LPR, tt = m0 + 32 * b + row;
                    v4f lo = *reinterpret_cast<const v4f *>(staged<SIZE>(stg, row, n)), hi = *reinterpret_cast<const v4f *>(staged<SIZE>(stg, row, n + 4));
                    if (left < WORDS) {   // columns that pad a row of G
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (n + i >= left) lo[i] = 0.0f;
                            if (n + 4 + i >= left) hi[i] = 0.0f;
                        }
                    }
                    if (tt < g.tokens && n0 + n < g.ldg) {
                        const uint4 words = make_uint4(pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]), pack_bf16(hi[0], hi[1]), pack_bf16(hi[2], hi[3]));
                        *reinterpret_cast<uint4 *>(g.G + tt * g.ldg + n0 + n) = words;
                        if (SIZE != BIG && g.rest != nullptr)
                            *reinterpret_cast<uint4 *>(g.rest + tt * g.ldg + n0 + n) = make_uint4(rest_of(words.x, lo[0], lo[1]), rest_of(words.y, lo[2], lo[3]),
                                                                                                  rest_of(words.z, hi[0], hi[1]), rest_of(words.w, hi[2], hi[3]));
                    }
                }
            }
        }
        now = next;
    }
}

// ---- the teacher -----------------------------------------------------------------------------------------------------------------------
// A wavefront per token: q = softmax(a / tau) over the valid entries (an index of the vocabulary, a logit that is not -inf; a NaN or +inf makes the
// token's q NaN).  A word that a list holds more than once counts once, with the sum of its probabilities: at[t, j] is entry j's word where it is the list's first of that word
// and -1 elsewhere, so that no two entries of a token meet in one place later.  map[w, t]: bit i of word w says that the token has an entry
// among the words 64 (32 w + i) .. + 63.
// Latency and the search of the list: 4096 tokens x 64 entries 13 us, 37 x 7 4.2.
struct TeacherArgs {
    const int64_t *idx;
    const void *logits;
    int tokens, top_k, map_words;
    int64_t vocab;
    float tau;
    int32_t *at;
    float *q, *some;
    uint32_t *map;
};

__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int i = 1; i < 64; i *= 2) x = fmaxf(x, __shfl_xor(x, i));
    return x;
}
__device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int i = 1; i < 64; i *= 2) x += __shfl_xor(x, i);
    return x;
}

template <bool BF16>
__global__ void __launch_bounds__(256) teacher_kernel(TeacherArgs g)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t dlds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.x * 4 + wave;
    int32_t *const word = reinterpret_cast<int32_t *>(dlds) + wave * (2 * g.top_k + g.map_words);
    float *const share = reinterpret_cast<float *>(word + g.top_k);
    uint32_t *const map = reinterpret_cast<uint32_t *>(share + g.top_k);
    if (t >= g.tokens) return;   // a wavefront keeps to itself: no barrier below
    const int64_t first = (int64_t)t * g.top_k;
    float most = -INFINITY;
    bool mine = false;
    for (int j = lane; j < g.top_k; j += 64) {
        const int64_t i = g.idx[first + j];
        const float a = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t *>(g.logits)[first + j] << 16) : static_cast<const float *>(g.logits)[first + j];
        const bool valid = i >= 0 && i < g.vocab && a != -INFINITY;
        mine |= valid;
        word[j] = valid ? (int32_t)i : -1;
        share[j] = a;
        if (valid) most = fmaxf(most, a);
    }
    for (int w = lane; w < g.map_words; w += 64) map[w] = 0;
    most = wave_max(most);
    float total = 0.0f;
    for (int j = lane; j < g.top_k; j += 64) {
        const float e = word[j] >= 0 ? expf((share[j] - most) / g.tau) : 0.0f;
        share[j] = e;
        total += e;
    }
    total = wave_sum(total);
    const bool some = __any(mine);
    asm volatile("" ::: "memory");   // LDS operations of a wavefront are done in order
    for (int j = lane; j < g.top_k; j += 64) {
        const int32_t w = word[j];
        float e = share[j];
        bool again = false;
        if (w >= 0) {
            for (int i = 0; i < j; ++i) again |= word[i] == w;
            for (int i = j + 1; i < g.top_k; ++i)
                if (word[i] == w) e += share[i];
            if (!again) atomicOr(&map[w >> 11], 1u << ((w >> 6) & 31));
        }
        g.at[first + j] = again ? -1 : w;
        g.q[first + j] = some ? e / total : 0.0f;
    }
    asm volatile("" ::: "memory");
    for (int w = lane; w < g.map_words; w += 64) g.map[(int64_t)w * g.tokens + t] = map[w];
    if (lane == 0) g.some[t] = some ? 1.0f : 0.0f;
}

// ---- losses from the parts of their sums ---------------------------------------------------------------------------------------------------
struct JoinArgs {
    const float *m, *s1, *s2;
    int parts, tokens, top_k, across;   // across: tokens of a block, a power of two
    int64_t vocab;
    const int64_t *targets;
    const float *z_target, *z_top, *q, *some;
    const int32_t *at;
    float tau;
    float *ce, *kd, *lse1, *lse2;
};

// A block takes `across` tokens; the slices of a token, 256 / across threads, share its parts and entries.  Their sums meet by shuffles and once in LDS.
// Bound by its reads: 16384 tokens x 1024 parts (134 MB) 33 us, 4.1 TB/s; few tokens by one chain of reads, 3.4 us at 16 x 1000.
template <bool HARD, bool SOFT>
__global__ void __launch_bounds__(256) join_kernel(JoinArgs g)
{
    __shared__ float waves[4][4][64];
    const int slices = 256 / g.across, slice = threadIdx.x / g.across, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.x * g.across + threadIdx.x % g.across;
    const bool inside = t < g.tokens;
    const float k2 = SOFT ? LOG2E / g.tau : 0.0f;
    int64_t y = -1;
    float z_target = 0.0f;
    if (HARD && inside) {
        y = g.targets[t];
        z_target = g.z_target[t];   // of a token that counts
    }
    float m = -INFINITY, s1 = 0.0f, s2 = 0.0f;
    auto add = [&](const float om, const float o1, const float o2) {
        const float to = fmaxf(m, om), base = to == -INFINITY ? 0.0f : to;
        const float mine = m - base, its = om - base;
        if (HARD) s1 = s1 * exp2_fast(mine * LOG2E) + o1 * exp2_fast(its * LOG2E);
        if (SOFT) s2 = s2 * exp2_fast(mine * k2) + o2 * exp2_fast(its * k2);
        m = to;
    };
    for (int p = slice; p < g.parts; p += 4 * slices) {
        float om[4], o1[4], o2[4];   // asked for together
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t at = (int64_t)std::min(p + i * slices, g.parts - 1) * g.tokens + std::min(t, g.tokens - 1);
            om[i] = p + i * slices < g.parts ? g.m[at] : -INFINITY;
            o1[i] = HARD ? g.s1[at] : 0.0f;
            o2[i] = SOFT ? g.s2[at] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (p + i * slices < g.parts) add(om[i], o1[i], o2[i]);   // also where the maximum is -inf: the part may be of NaN, which no maximum shows
    }
    for (int x = g.across; x < 64; x *= 2) add(__shfl_xor(m, x), __shfl_xor(s1, x), __shfl_xor(s2, x));   // the same sum in both lanes
    waves[0][wave][lane] = m;
    waves[1][wave][lane] = s1;
    waves[2][wave][lane] = s2;
    __syncthreads();
    m = -INFINITY;
    s1 = s2 = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) add(waves[0][w][lane], waves[1][w][lane], waves[2][w][lane]);
    const float lse1 = HARD ? m + logf(s1) : 0.0f, lse2 = SOFT ? m / g.tau + logf(s2) : 0.0f;
    if (inside && slice == 0) {
        if (HARD) {
            g.lse1[t] = lse1;
            g.ce[t] = y >= 0 && y < g.vocab ? lse1 - z_target : 0.0f;
        }
        if (SOFT) g.lse2[t] = lse2;
    }
    if constexpr (SOFT) {
        float sum = 0.0f;
        if (inside)
            for (int j = slice; j < g.top_k; j += slices) {
                const int64_t e = (int64_t)t * g.top_k + j;
                const float q = g.q[e];
                if (g.at[e] >= 0 && q != 0.0f) sum += q * (logf(q) - g.z_top[e] / g.tau + lse2);
            }
        for (int x = g.across; x < 64; x *= 2) sum += __shfl_xor(sum, x);
        waves[3][wave][lane] = sum;
        __syncthreads();
        if (inside && slice == 0) {
            sum = waves[3][0][lane] + waves[3][1][lane] + waves[3][2][lane] + waves[3][3][lane];
            g.kd[t] = g.some[t] != 0.0f ? g.tau * g.tau * sum : 0.0f;
        }
    }
}

// ---- gradients -------------------------------------------------------------------------------------------------------------------------
// The two products of a piece in one launch, the longer contraction first.  The contraction of either may be cut into splits that leave
// their sums in fp32 side by side; dH adds up over the pieces of the vocabulary in fp32 as well.
struct GradientArgs {
    Operand P, Q;              // P transposed; Q transposed (dW) or not (dH)
    int N, M, stages;          // of the result; k stages of the whole contraction
    int splits, per;           // stages of a split
    uint16_t *C;               // bf16 [M, N], or null:
    float *part;               // fp32 [splits, M, N]
    int add;                   // to what part holds
    int tiles_n, tiles_m;
};
struct GradientPair {
    GradientArgs dw, dh;
    int dw_first, job0;        // the first block of the second product
    const int64_t *targets;    // of G's common factor (null: 1)
    const float *d1;
    int tokens;
    int64_t vocab;
};

template <int SIZE>
__device__ __forceinline__ void gradient_results(const GradientArgs &g, const v16f (&acc)[HeadTile<SIZE>::WP][HeadTile<SIZE>::WQ], uint8_t *lds, const int n0,
                                                 const int m0, const int split, const float factor)
{
    using S = HeadTile<SIZE>;
    static_assert(S::WAVES * 32 * S::ROW <= S::LDS, "32 columns of every wavefront are staged in the idle ring");
    const int lane = lane_here(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint8_t *const stg = lds + wave * 32 * S::ROW;
    const int nw = n0 + (wave & 1) * 32 * S::WP, mw = m0 + (wave >> 1) * 32 * S::WQ;
    float *const part = g.part + ((int64_t)split * g.M + mw) * g.N + nw;
#pragma unroll
    for (int b = 0; b < S::WQ; ++b) {
        stage_columns<SIZE, 32>(acc, b, 0, stg, lane);
        if (g.C) {
            constexpr int LPR = S::ROW / 32;
            const int n = 8 * (lane % LPR);
#pragma unroll
            for (int j = 0; j < LPR / 2; ++j) {
                const int row = 64 / LPR * j + lane / LPR, m = 32 * b + row;
                const v4f lo = *reinterpret_cast<const v4f *>(staged<SIZE>(stg, row, n)) * factor, hi = *reinterpret_cast<const v4f *>(staged<SIZE>(stg, row, n + 4)) * factor;
                if (mw + m < g.M && nw + n < g.N)
                    *reinterpret_cast<uint4 *>(g.C + (int64_t)(mw + m) * g.N + nw + n) =
                        make_uint4(pack_bf16(lo[0], lo[1]), pack_bf16(lo[2], lo[3]), pack_bf16(hi[0], hi[1]), pack_bf16(hi[2], hi[3]));
            }
        } else {
            constexpr int LPR = S::ROW / 16;
            const int n = 4 * (lane % LPR);
#pragma unroll
            for (int j = 0; j < LPR / 2; ++j) {
                const int row = 64 / LPR * j + lane / LPR, m = 32 * b + row;
                v4f x = *reinterpret_cast<const v4f *>(staged<SIZE>(stg, row, n)) * factor;
                if (mw + m < g.M && nw + n < g.N) {
                    v4f *const to = reinterpret_cast<v4f *>(part + (int64_t)m * g.N + n);
                    if (g.add) x += *to;
                    *to = x;
                }
            }
        }
    }
}

template <int SIZE, bool QT>
__device__ __forceinline__ void gradient_tile(const GradientArgs &g, uint8_t *lds, const int job, const CommonFactor &common, const int64_t vocab)
{
    using S = HeadTile<SIZE>;
    // The tiles of a split follow one another and so lie on as few XCDs as there are for each: they read the same k of both operands, which only these
    // L2s ask for then (dH of 1531 x 50001 x 1000 in four splits of 24 tiles: 863 MB read with every split on all XCDs, 420 so).  The tiles of dW
    // that share the same words' G, the larger operand where tokens are few, follow one another.
    const int tiles = g.tiles_n * g.tiles_m, id = place_of_block(tiles * g.splits, job);
    if (id >= tiles * g.splits) return;
    int split = id / tiles, tn, tm;
    if constexpr (QT) tile_in_order(g.tiles_m, g.tiles_n, id - split * tiles, tm, tn);
    else tile_in_order(g.tiles_n, g.tiles_m, id - split * tiles, tn, tm);
    split = __builtin_amdgcn_readfirstlane(split);
    const int k0 = split * g.per * STAGE_K, left = g.stages - split * g.per, stages = left < g.per ? left : g.per;
    if (stages <= 0) return;   // of a last piece that has fewer of them; nothing to add
    Operand p = g.P, q = g.Q;
    p.base += (int64_t)k0 * p.ld;
    p.k -= k0;
    q.base += (int64_t)k0 * (QT ? q.ld : 1);
    q.k -= k0;
    TileProduct<SIZE, true, QT> product;
    product.begin(p, q, tn * S::N, tm * S::M, stages, lds);
    v16f acc[S::WP][S::WQ];
    product.run(lds, acc);
    gradient_results<SIZE>(g, acc, lds, tn * S::N, tm * S::M, split, common.value(vocab));
}

// A block per tile: taken one after the other by a block, as the logits are, they took 3 to 10 % longer (the two products' tiles are not alike,
// and the device deals them out as multiprocessors become free).  Bound by the matrix pipe: 16384 tokens x 16384 words x 2560 in 2.1 ms (1.3 PFLOP/s;
// large library products of these two forms reach 0.91 and 0.97), 1531 x 50001 x 1000 in 290 to 320 us (1.0), where dW has 24 stages to a tile
// and some 18 us beside them.
template <int SIZE>
__global__ void __launch_bounds__(64 * HeadTile<SIZE>::WAVES, 2) gradient_kernel(GradientPair pair)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t dlds[];
    const CommonFactor common(pair.targets, pair.d1, pair.tokens);
    const bool second = (int)blockIdx.x >= pair.job0;
    const int job = (int)blockIdx.x - (second ? pair.job0 : 0);
    if (second != (pair.dw_first != 0)) gradient_tile<SIZE, true>(pair.dw, dlds, job, common, pair.vocab);
    else gradient_tile<SIZE, false>(pair.dh, dlds, job, common, pair.vocab);
}

// bf16 sums of fp32 parts.  A block takes 256 / SLICES groups of four values, a slice of its threads every SLICES-th part: with few values and
// many parts (37 x 1000 in 32) one thread for all of them took 11 us.
// 16384 x 2560 40 us: 252 MB at 6.2 TB/s.
template <int SLICES>
__global__ void __launch_bounds__(256) sum_parts_kernel(const float *part, int64_t n, int parts, uint16_t *out, int64_t first)
{
    constexpr int ACROSS = 256 / SLICES;
    __shared__ v4f sums[256];
    const int slice = threadIdx.x / ACROSS;
    const int64_t i = first + ((int64_t)blockIdx.x * ACROSS + threadIdx.x % ACROSS) * 4;
    v4f x = {0.0f, 0.0f, 0.0f, 0.0f};
    if (i < n)
        for (int p = slice; p < parts; p += SLICES) x += *reinterpret_cast<const v4f *>(part + p * n + i);
    if constexpr (SLICES > 1) {
        sums[threadIdx.x] = x;
        __syncthreads();
        if (slice) return;
#pragma unroll
        for (int s = 1; s < SLICES; ++s) x += sums[threadIdx.x + s * ACROSS];
    }
    if (i < n) *reinterpret_cast<uint2 *>(out + i) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
}

// ---- few tokens ------------------------------------------------------------------------------------------------------------------------
// Gradients of up to 64 tokens in one launch.  dH reads W: small tiles as above, the words cut into splits.  dW is written and little else: its
// contraction is the tokens, at most four steps of 16, so a wavefront takes 128 words x 128 columns from registers.  A lane reads four
// neighbouring columns (words) of eight tokens of H (G) and sorts them into four fragments by byte permutations; column j of a lane's four is
// a product's column, so a lane's results are neighbours again and rows leave in 256 bytes.
// Bound by what it moves: 37 x 32001 x 1000 27 us for 71 MB read and 72 written, 5.3 TB/s (33 where it takes G's rests as well).  An XCD takes
// neighbouring tiles: rows that are not whole lines share them (dealt out in turns, W came 1.8 times: 34 us), and tiles of one split share G
// (64 x 32000 x 2560, whole lines: 4 us).
struct FewGradients {
    GradientArgs dh;
    int dh_blocks, dw_per;   // multiples of eight; of the others, an XCD's share
    const uint16_t *H, *G, *rest;
    int64_t ldg;
    int tokens, d, words;
    uint16_t *dW;
    int across;               // groups of 128 columns
    const int64_t *targets;
    const float *d1;
    int64_t vocab;
};

// fragment j: column k + j of COLUMNS, rows first + 8 c .. + 7 (the last one again past it)
template <int COLUMNS>
__device__ __forceinline__ void column_fragments(const uint16_t *base, const int64_t ld, const int first, const int last, const int64_t k, const int c, v8bf (&f)[COLUMNS])
{
    typedef unsigned v4u __attribute__((ext_vector_type(4)));
    uint32_t raw[8][COLUMNS / 2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint16_t *const row = base + (int64_t)std::min(first + 8 * c + e, last) * ld + k;
        if constexpr (COLUMNS == 4) {
            const uint2 x = *reinterpret_cast<const uint2 *>(row);
            raw[e][0] = x.x;
            raw[e][1] = x.y;
        } else raw[e][0] = *reinterpret_cast<const uint32_t *>(row);
    }
#pragma unroll
    for (int j = 0; j < COLUMNS; ++j) {
        v4u o;
#pragma unroll
        for (int p = 0; p < 4; ++p) o[p] = __builtin_amdgcn_perm(raw[2 * p + 1][j / 2], raw[2 * p][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
        f[j] = __builtin_bit_cast(v8bf, o);
    }
}
// the same with zeros past the last one
template <int COLUMNS>
__device__ __forceinline__ void token_fragments(const uint16_t *base, const int64_t ld, const int first, const int tokens, const int64_t k, const int c, v8bf (&f)[COLUMNS])
{
    column_fragments(base, ld, first, tokens - 1, k, c, f);
    if (first + 16 > tokens) {
        typedef unsigned v4u __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int j = 0; j < COLUMNS; ++j) {
            v4u x = __builtin_bit_cast(v4u, f[j]);
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const int left = tokens - (first + 8 * c + 2 * p);
                x[p] = left >= 2 ? x[p] : left == 1 ? x[p] & 0xffffu : 0u;
            }
            f[j] = __builtin_bit_cast(v8bf, x);
        }
    }
}

template <int STEPS, bool REST>   // of 16 tokens; with what rounding left over of G
__global__ void __launch_bounds__(256, 2) few_gradient_kernel(FewGradients g)
{
    using S = HeadTile<SMALL>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t dlds[];
    const CommonFactor common(g.targets, g.d1, g.tokens);
    if ((int)blockIdx.x < g.dh_blocks) {
        const int id = ((int)blockIdx.x & 7) * (g.dh_blocks >> 3) + ((int)blockIdx.x >> 3);
        const int tn = id % g.dh.tiles_n, split = id / g.dh.tiles_n;
        if (split >= g.dh.splits) return;
        const int s0 = split * g.dh.per, nk = std::min(g.dh.stages - s0, g.dh.per);
        Operand p = g.dh.P, q = g.dh.Q;
        p.base += (int64_t)s0 * STAGE_K * p.ld;
        p.k -= s0 * STAGE_K;
        q.base += s0 * STAGE_K;
        q.k -= s0 * STAGE_K;
        v16f acc[S::WP][S::WQ];
        TileProduct<SMALL, true, false> product;
        product.begin(p, q, tn * S::N, 0, nk, dlds);
        product.run(dlds, acc);
        gradient_results<SMALL>(g.dh, acc, dlds, tn * S::N, 0, split, common.value(g.vocab));
        return;
    }
    const int lane = threadIdx.x & 63, r = lane & 31, c = lane >> 5;
    const int job = (int)blockIdx.x - g.dh_blocks;
    const int id = ((job & 7) * g.dw_per + (job >> 3)) * 4 + (threadIdx.x >> 6);
    const int col = id % g.across * 128 + 4 * r, v0 = id / g.across * 128;
    if (v0 >= g.words) return;
    constexpr int AT_ONCE = STEPS >= 3 && REST ? 2 : 4;   // words of a lane: what the registers hold
    v8bf h[STEPS][4], a[STEPS][AT_ONCE], b[REST ? STEPS : 1][AT_ONCE];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) column_fragments(g.H, g.d, 16 * s, g.tokens - 1, std::min(col, g.d - 4), c, h[s]);
    const float factor = common.value(g.vocab);
#pragma unroll
    for (int w0 = 0; w0 < 4; w0 += AT_ONCE) {
        const int64_t k = std::min((int64_t)v0 + 4 * r, g.ldg - 4) + w0;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            int half = c;
            if (AT_ONCE == 2) {   // neither all of them asked for at once nor their addresses kept: the registers hold no more
                asm volatile("" : "+v"(half));
                __builtin_amdgcn_sched_barrier(0);
            }
            token_fragments(g.G, g.ldg, 16 * s, g.tokens, k, half, a[s]);
            if constexpr (REST) token_fragments(g.rest, g.ldg, 16 * s, g.tokens, k, half, b[s]);
        }
#pragma unroll
        for (int w = 0; w < AT_ONCE; ++w) {   // words v0 + 4 row + w0 + w
            if (AT_ONCE == 2) __builtin_amdgcn_sched_barrier(0);
            v16f acc[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[j][e] = 0.0f;
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[s][w], h[s][j], acc[j], 0, 0, 0);
                    if constexpr (REST) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[s][w], h[s][j], acc[j], 0, 0, 0);
                }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int v = v0 + 4 * (8 * (e >> 2) + 4 * c + (e & 3)) + w0 + w;
                if (v < g.words && col < g.d)
                    *reinterpret_cast<uint2 *>(g.dW + (int64_t)v * g.d + col) =
                        make_uint2(pack_bf16(acc[0][e] * factor, acc[1][e] * factor), pack_bf16(acc[2][e] * factor, acc[3][e] * factor));
            }
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------------------
constexpr int PLAN_CUS = 256;                          // multiprocessors of the part: a plan depends on sizes alone
// Most of G at a time (512 MB and what pads its rows), but for more than 2^20 tokens, whose pieces have 256 words, and for up to 64 tokens, which take
// the vocabulary whole.  2^25 to 2^27 took within 5 % of it, pieces that the last cache holds too
constexpr int64_t PIECE_ELEMENTS = (int64_t)1 << 28;

std::atomic<int> g_logits_size{-1}, g_gradient_size{-1};   // of the test hook

int edge_of(const int size) { return size == BIG ? 256 : size == SMALL ? 128 : 64; }
int64_t tiles_of(const int64_t n, const int64_t m, const int size) { return ceil_div(n, edge_of(size)) * ceil_div(m, edge_of(size)); }

// Estimated us of tiles of one size: of a tile alone and, where the others run, of a multiprocessor's time for it, by its stages
struct TileTimes {
    float alone_step, alone, step, each;
    float longest(const float stages) const { return alone_step * stages + alone; }
    float share(const float stages) const { return step * stages + each; }
};

// Logits in tiles of 64, 128 and 256; fits to 16 to 1500 tokens, 3000 to 100000 words and 128 to 4096 dimensions (0.3 % over the best of the three on
// average, 15 at most).  Rows that are not whole lines of 128 bytes cost a stage's fetches a second line each, small tiles most.  us measured with
// each size (forward with its join): 16 x 500 x 2560 16.2 / 22.4 / 49.6, 300 x 4000 x 2560 23.2 / 27.1 / 51.7, 1000 x 4000 x 2560 40.0 / 29.7 /
// 51.3, 1000 x 32000 x 2560 269 / 158 / 133, 4000 x 32000 x 64 165 / 78 / 59, 169 x 37331 x 3280 99 / 86 / 64, 400 x 100000 x 3280 696 / 466 / 327.
int logits_size(const int64_t tokens, const int64_t words, const int64_t d)
{
    const int forced = g_logits_size.load(std::memory_order_relaxed);
    if (forced >= 0) return forced;
    static constexpr TileTimes times[] = {{0.22f, 2.9f, 0.2f, 1.8f}, {0.41f, 4.0f, 0.41f, 2.2f}, {0.92f, 6.9f, 1.15f, 6.4f}};
    static constexpr float ragged[] = {1.3f, 1.18f, 1.03f};
    const float stages = (float)ceil_div(d, STAGE_K);
    int best = BIG;
    float least = INFINITY;
    for (int size = BIG; size >= TINY; --size) {
        const TileTimes &t = times[size];
        const float alone = t.longest(stages), share = t.share(d % STAGE_K ? ragged[size] * stages : stages);
        const int64_t tiles = tiles_of(words, tokens, size);
        // (few of them do not slow each other down)
        const float us = std::max(alone, tiles <= PLAN_CUS ? alone + (share - alone) * (float)tiles / PLAN_CUS : (float)ceil_div(tiles, PLAN_CUS) * share);
        if (us < least) least = us, best = size;
    }
    return best;
}

struct BackwardPlan {
    int64_t piece;       // words at a time
    int64_t ldg;         // row length of G
    int size;            // tiles of the gradients' products
    int dw_splits, dh_splits;
    // fp32 results that are still to be added up, [parts, rows, d] (0: the product writes bf16)
    int dw_parts() const { return dw_splits > 1 ? dw_splits : 0; }
    int dh_parts(int64_t vocab) const { return dh_splits > 1 || piece < vocab ? dh_splits : 0; }
};

// Rows of G lie an odd number of lines apart, so that those of a stage go to all channels of a L2 (16384 tokens in pieces of 16384 words: 34.5 ms a
// step with the lines of a row alone, 34.1 so)
int64_t pitch_of(const int64_t cols) { return (cols / STAGE_K | 1) * STAGE_K; }

BackwardPlan plan_backward(const int64_t tokens, const int64_t d, const int64_t vocab)
{
    BackwardPlan plan;
    const int64_t most = std::min(std::max(PIECE_ELEMENTS / tokens / 256 * 256, (int64_t)256), (int64_t)1 << 22);
    const int64_t pieces = ceil_div(vocab, most);
    plan.piece = pieces == 1 ? vocab : ceil_div(ceil_div(vocab, pieces), 256) * 256;
    plan.ldg = ceil_div(plan.piece, STAGE_K) * STAGE_K;
    // fewest us over tile sizes and splits: what the products take, and what a split's parts are to read again at 4 TB/s
    const int64_t dw_stages = ceil_div(tokens, STAGE_K), dh_stages = plan.ldg / STAGE_K;
    // fits to 70 to 5000 tokens, 1500 to 100000 words and 128 to 3280 dimensions, with what surrounds a tile in proportion to what it stores.  us of a
    // backward pass, tiles of 128 and of 256 for the gradients: 65 x 32000 x 512 38 / 60, 1000 x 4000 x 2560 74 / 81, 1000 x 32000 x 2560 503 /
    // 456, 130 x 100000 x 3280 846 / 598, 16000 x 4000 x 2560 921 / 803; of 64 and of 128: 128 x 4000 x 64 12 / 15
    static constexpr TileTimes times[] = {{0.2f, 5.0f, 0.33f, 1.4f}, {0.45f, 6.0f, 0.44f, 3.35f}, {1.1f, 9.0f, 1.42f, 14.5f}};
    static constexpr float ragged[] = {1.5f, 1.3f, 1.0f};   // of what surrounds a tile: rows that are not whole lines leave in parts of them
    const int forced = g_gradient_size.load(std::memory_order_relaxed);
    float best = INFINITY;
    for (int size = TINY; size <= BIG; ++size)
        for (int64_t sw = 1; sw <= 16; sw *= 2)
            for (int64_t sh = 1; sh <= 64; sh *= 2) {
                if (forced >= 0 && forced <= BIG && size != forced) continue;
                if ((sw > 1 && sw * 2 > dw_stages) || (sh > 1 && sh * 2 > dh_stages)) continue;
                const int64_t wt = tiles_of(d, plan.piece, size) * sw, ht = tiles_of(d, tokens, size) * sh;
                const float wk = (float)ceil_div(dw_stages, sw), hk = (float)ceil_div(dh_stages, sh);
                const TileTimes &t = times[size];
                const float more = d % STAGE_K ? (ragged[size] - 1.0f) * t.each : 0.0f;
                // a long tile beside those of a full device takes longer (fewer splits of dH than this asks for: 130 x 100000 x 2560 750 us,
                // 200 x 100000 x 2560 733; 501 and 508 so)
                const float most = std::max(wk, hk), busy = std::min(1.0f, (float)(wt + ht) / (float)((size == BIG ? 1 : 2) * PLAN_CUS));
                const float longest = t.longest(most * (1.0f + 0.4f * busy));
                float us = std::max(longest, ((float)wt * t.share(wk) + (float)ht * t.share(hk) + (float)(wt + ht) * more) / (float)PLAN_CUS);
                if (sw > 1) us += 3.0f + (float)(4 * sw + 2) * (float)plan.piece * (float)d / 4e6f;
                if (sh > 1) us += 3.0f + (float)(4 * sh + 2) * (float)tokens * (float)d / 4e6f;
                if (us < best) {
                    best = us;
                    plan.size = size;
                    plan.dw_splits = (int)sw;
                    plan.dh_splits = (int)sh;
                }
            }
    // no split without a stage
    plan.dw_splits = (int)ceil_div(dw_stages, ceil_div(dw_stages, plan.dw_splits));
    plan.dh_splits = (int)ceil_div(dh_stages, ceil_div(dh_stages, plan.dh_splits));
    return plan;
}

// Workspace, one region after the other
struct HeadRegions {
    size_t bytes = 0;
    size_t take(const size_t n)
    {
        const size_t at = bytes;
        bytes += align_up(n, 256);
        return at;
    }
};
struct TeacherRegions {
    size_t at, q, map, some;
    TeacherRegions(HeadRegions &r, int64_t tokens, int64_t vocab, int64_t top_k)
    {
        at = r.take((size_t)tokens * top_k * 4);
        q = r.take((size_t)tokens * top_k * 4);
        map = r.take((size_t)ceil_div(vocab, 2048) * tokens * 4);
        some = r.take((size_t)tokens * 4);
    }
};

template <class Kernel>
sbn_status with_lds(Kernel kernel, const int bytes)
{
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) return SBN_OK;
    set_hip_error(e, "hipFuncSetAttribute");
    return SBN_EHIP;
}

template <int SIZE, bool GRAD, bool HARD, bool SOFT>
sbn_status launch_logits_as(LogitsArgs &g, hipStream_t stream)
{
    using S = HeadTile<SIZE>;
    g.tiles_n = (int)ceil_div(g.words, S::N);
    g.tiles_m = (int)ceil_div(g.tokens, S::M);
    static thread_local bool raised = false;
    if (!raised) {
        const sbn_status st = with_lds(&logits_kernel<SIZE, GRAD, HARD, SOFT>, S::LDS);
        if (st != SBN_OK) return st;
        raised = true;
    }
    const int64_t all = ceil_div((int64_t)g.tiles_n * g.tiles_m, 8) * 8, blocks = GRAD ? all : std::min(all, (int64_t)(SIZE == BIG ? 1 : 2) * PLAN_CUS);
    hipLaunchKernelGGL((logits_kernel<SIZE, GRAD, HARD, SOFT>), dim3((unsigned)blocks), dim3(64 * S::WAVES), S::LDS, stream, g);
    return check_launch("logits_kernel");
}
template <int SIZE, bool GRAD>
sbn_status launch_logits_of(LogitsArgs &g, bool hard, bool soft, hipStream_t stream)
{
    return !soft ? launch_logits_as<SIZE, GRAD, true, false>(g, stream) : hard ? launch_logits_as<SIZE, GRAD, true, true>(g, stream)
                                                                               : launch_logits_as<SIZE, GRAD, false, true>(g, stream);
}
template <bool GRAD>
sbn_status launch_logits(LogitsArgs &g, int size, bool hard, bool soft, hipStream_t stream)
{
    return size == BIG ? launch_logits_of<BIG, GRAD>(g, hard, soft, stream) : size == SMALL ? launch_logits_of<SMALL, GRAD>(g, hard, soft, stream)
                                                                                             : launch_logits_of<TINY, GRAD>(g, hard, soft, stream);
}

sbn_status launch_teacher(const HeadCall &h, uint8_t *ws, const TeacherRegions &r, LogitsArgs &g, hipStream_t stream)
{
    g.at = reinterpret_cast<int32_t *>(ws + r.at);
    g.q = reinterpret_cast<float *>(ws + r.q);
    g.map = reinterpret_cast<uint32_t *>(ws + r.map);
    g.some = reinterpret_cast<float *>(ws + r.some);
    g.top_k = (int)h.top_k;
    g.tau = h.tau;
    TeacherArgs t{h.top_idx, h.top_logits, (int)h.tokens, (int)h.top_k, (int)ceil_div(h.vocab, 2048), h.vocab, h.tau,
                  const_cast<int32_t *>(g.at), const_cast<float *>(g.q), const_cast<float *>(g.some), const_cast<uint32_t *>(g.map)};
    const unsigned lds = 16u * (2u * t.top_k + t.map_words);
    if (h.top_dtype == SBN_BF16) hipLaunchKernelGGL(teacher_kernel<true>, dim3((unsigned)ceil_div(h.tokens, 4)), dim3(256), lds, stream, t);
    else hipLaunchKernelGGL(teacher_kernel<false>, dim3((unsigned)ceil_div(h.tokens, 4)), dim3(256), lds, stream, t);
    return check_launch("teacher_kernel");
}

LogitsArgs logits_of(const HeadCall &h)
{
    LogitsArgs g{};
    g.H = static_cast<const uint16_t *>(h.H);
    g.W = static_cast<const uint16_t *>(h.W);
    g.tokens = (int)h.tokens;
    g.d = (int)h.d_in;
    g.words = (int)h.vocab;
    g.vocab = h.vocab;
    g.targets = h.targets;
    return g;
}

// Few tokens: splits of the words for dH, as many as give 512 blocks (two per multiprocessor) with eight stages each, and fewer where their
// sums, [tokens, d] floats written and read again per split, would weigh more than a quarter of W
// and more than 2 MB
// They are taken for weights of 2^21 values and more (backward pass of 16 to 64 tokens against the plan below at 65, us: 32000 x 2560 88 / 122,
// 32000 x 512 29 / 38, 32000 x 64 18 / 26, 4000 x 512 16.5 / 16.0, 4000 x 64 13.9 / 11.7)
constexpr int64_t FEW_TOKENS = 64, FEW_VALUES = 1 << 21;
// The gradients of few tokens take G with what its rounding to bf16 left over, as rows behind those of G: of dH a tile has room for them, of dW they
// are read beside G.  A result then has its own rounding alone; without the rests G's comes on top, which many tokens do not average out: G's
// largest values, the targets' and the teacher's, stand nearly alone in a row of dH and of dW.  Errors of dH and dW in 1e-4 of their norms, without
// and with the rests (rounding the results alone costs 16 to 17; the same at 64, 512 and 2048 tokens, a little more with a few):
//   distillation 23 and 17;  cross entropy, d_ce alike in all tokens 17 to 18 and 17 (see CommonFactor), d_ce of any values 23 to 27 and 17
// Cross entropy with d_ce alike has its targets' values unrounded, and where few tokens count these are most of dW: then dW without the rests
// is off by up to 1.8 times as much as with them (1.4 at 16 tokens, 1.2 at 18 and more, over 140 sizes).
// The price, backward pass in us without and with the rests, d x words 256 x 2000 and 2560 x 32000:
//   cross entropy  16 tokens 11.3 / 14.5 and 87 / 89, 32 tokens 11.5 / 15 and 89 / 98, 64 tokens 12 / 18.6 and 101 / 123
//   distillation   16 tokens 16.4 / 19.8 and 91 / 94, 64 tokens 18.7 / 26 and 105 / 128
// So a distillation takes them as far as this way goes, cross entropy as long as the tokens are one step of the matrix instruction.  More tokens
// are bound by the matrix pipe, and the rests would be two of eight products more.
constexpr int REST_TOKENS = 16;
bool takes_rest(const int64_t tokens, const bool soft) { return tokens <= (soft ? FEW_TOKENS : REST_TOKENS); }
bool takes_few(const int64_t tokens, const int64_t d, const int64_t vocab, const bool soft)
{
    const int forced = g_gradient_size.load(std::memory_order_relaxed);
    return tokens <= FEW_TOKENS && (forced >= 0 ? forced > BIG : takes_rest(tokens, soft) || vocab * d >= FEW_VALUES);
}
struct FewPlan {
    int64_t ldg;
    int stages, per, splits;   // of dH
    int rows;                  // of G
    int parts;                 // fp32 [parts, tokens, d] of dH; 1: bf16 at once
};
FewPlan plan_few(const int64_t tokens, const int64_t d, const int64_t vocab, const bool soft)
{
    FewPlan p;
    const bool rest = takes_rest(tokens, soft);
    p.rows = (int)(rest ? 2 * tokens : tokens);
    p.stages = (int)ceil_div(vocab, STAGE_K);
    p.ldg = (int64_t)p.stages * STAGE_K;
    int64_t splits = std::min(ceil_div(2 * PLAN_CUS, ceil_div(d, 128)), ceil_div(p.stages, 8));
    splits = std::max((int64_t)1, std::min(splits, std::max(vocab / (16 * tokens), ((int64_t)1 << 19) / (tokens * d))));
    p.per = (int)ceil_div(p.stages, splits);
    p.splits = (int)ceil_div(p.stages, p.per);
    p.parts = rest ? 2 * p.splits : p.splits;
    return p;
}

int64_t forward_parts(const HeadCall &h) { return 2 * ceil_div(h.vocab, edge_of(logits_size(h.tokens, h.vocab, h.d_in))); }

}  // namespace

void set_head_tiles(int logits, int gradients)
{
    g_logits_size.store(logits > BIG ? -1 : logits, std::memory_order_relaxed);
    g_gradient_size.store(gradients, std::memory_order_relaxed);
}

size_t head_workspace_bytes(int64_t tokens, int64_t d_in, int64_t vocab, int64_t top_k, bool backward)
{
    HeadCall h{};
    h.tokens = tokens;
    h.d_in = d_in;
    h.vocab = vocab;
    HeadRegions r;
    const int64_t parts = forward_parts(h);
    for (int i = 0; i < (top_k ? 3 : 2); ++i) r.take((size_t)parts * tokens * 4);
    r.take((size_t)tokens * 4);
    r.take((size_t)tokens * top_k * 4);
    if (top_k) TeacherRegions(r, tokens, vocab, top_k);
    if (!backward) return r.bytes;
    HeadRegions b;
    if (takes_few(tokens, d_in, vocab, top_k != 0)) {
        const FewPlan plan = plan_few(tokens, d_in, vocab, top_k != 0);
        if (top_k) TeacherRegions(b, tokens, vocab, top_k);
        b.take((size_t)plan.rows * plan.ldg * 2);
        b.take(plan.parts > 1 ? (size_t)plan.parts * tokens * d_in * 4 : 0);
        return std::max(r.bytes, b.bytes);
    }
    const BackwardPlan plan = plan_backward(tokens, d_in, vocab);
    if (top_k) TeacherRegions(b, tokens, vocab, top_k);
    b.take((size_t)tokens * pitch_of(plan.ldg) * 2);
    b.take((size_t)plan.dh_parts(vocab) * tokens * d_in * 4);
    b.take((size_t)plan.dw_parts() * plan.piece * d_in * 4);
    return std::max(r.bytes, b.bytes);
}

sbn_status launch_head_forward(const HeadCall &h, void *workspace, hipStream_t stream)
{
    const bool hard = h.targets != nullptr, soft = h.top_idx != nullptr;
    uint8_t *const ws = static_cast<uint8_t *>(workspace);
    HeadRegions r;
    LogitsArgs g = logits_of(h);
    const int64_t parts = forward_parts(h);
    auto floats = [&](const size_t n) { return reinterpret_cast<float *>(ws + r.take(n * 4)); };
    g.m = floats((size_t)parts * h.tokens);
    g.s1 = floats((size_t)parts * h.tokens);
    g.s2 = soft ? floats((size_t)parts * h.tokens) : nullptr;
    g.z_target = floats((size_t)h.tokens);
    g.z_top = floats((size_t)h.tokens * h.top_k);
    if (soft) {
        const TeacherRegions tr(r, h.tokens, h.vocab, h.top_k);
        const sbn_status st = launch_teacher(h, ws, tr, g, stream);
        if (st != SBN_OK) return st;
    }
    const sbn_status st = launch_logits<false>(g, logits_size(h.tokens, h.vocab, h.d_in), hard, soft, stream);
    if (st != SBN_OK) return st;
    JoinArgs j{g.m, g.s1, g.s2, (int)parts, (int)h.tokens, (int)h.top_k, 1, h.vocab, h.targets, g.z_target, g.z_top, g.q, g.some, g.at, h.tau,
               h.ce, h.kd, h.lse1, h.lse2};
    while (j.across < 32 && h.tokens / (2 * j.across) >= PLAN_CUS) j.across *= 2;
    const dim3 grid((unsigned)ceil_div(h.tokens, j.across)), block(256);
    if (!soft) hipLaunchKernelGGL((join_kernel<true, false>), grid, block, 0, stream, j);
    else if (hard) hipLaunchKernelGGL((join_kernel<true, true>), grid, block, 0, stream, j);
    else hipLaunchKernelGGL((join_kernel<false, true>), grid, block, 0, stream, j);
    return check_launch("join_kernel");
}

template <int SIZE>
static sbn_status launch_gradients(GradientPair &pair, hipStream_t stream)
{
    using S = HeadTile<SIZE>;
    pair.dw_first = pair.dw.per >= pair.dh.per;
    int64_t jobs = 0;
    for (const bool second : {false, true}) {
        GradientArgs &g = second != (pair.dw_first != 0) ? pair.dw : pair.dh;
        g.tiles_n = (int)ceil_div(g.N, S::N);
        g.tiles_m = (int)ceil_div(g.M, S::M);
        if (second) pair.job0 = (int)jobs;
        jobs += g.N ? ceil_div((int64_t)g.tiles_n * g.tiles_m * g.splits, 8) * 8 : 0;   // equal shares, one per XCD
    }
    static thread_local bool raised = false;
    if (!raised) {
        const sbn_status st = with_lds(&gradient_kernel<SIZE>, S::LDS);
        if (st != SBN_OK) return st;
        raised = true;
    }
    hipLaunchKernelGGL(gradient_kernel<SIZE>, dim3((unsigned)jobs), dim3(64 * S::WAVES), S::LDS, stream, pair);
    return check_launch("gradient_kernel");
}

template <int STEPS, bool REST>
static sbn_status launch_few_as(const FewGradients &g, const int64_t blocks, hipStream_t stream)
{
    constexpr int LDS = HeadTile<SMALL>::LDS;
    static thread_local bool raised = false;
    if (!raised) {
        const sbn_status st = with_lds(&few_gradient_kernel<STEPS, REST>, LDS);
        if (st != SBN_OK) return st;
        raised = true;
    }
    hipLaunchKernelGGL((few_gradient_kernel<STEPS, REST>), dim3((unsigned)blocks), dim3(256), LDS, stream, g);
    return check_launch("few_gradient_kernel");
}

static sbn_status launch_few_gradients(const HeadCall &h, const LogitsArgs &l, const FewPlan &plan, float *part, hipStream_t stream)
{
    FewGradients g{};
    g.H = l.H;
    g.G = l.G;
    g.ldg = l.ldg;
    g.tokens = l.tokens;
    g.rest = l.rest;
    g.d = l.d;
    g.words = l.words;
    g.dW = static_cast<uint16_t *>(h.dW);
    g.across = (int)ceil_div(h.d_in, 128);
    g.targets = h.targets;
    g.d1 = h.d_ce;
    g.vocab = h.vocab;
    GradientArgs &a = g.dh;
    a.P = Operand{l.W, l.d, l.d, l.words};
    a.Q = Operand{l.G, l.ldg, plan.rows, (int)l.ldg};
    a.N = l.d;
    a.M = plan.rows;   // (a split's rests are a part of their own)
    a.stages = plan.stages;
    a.per = plan.per;
    a.C = plan.parts > 1 ? nullptr : static_cast<uint16_t *>(h.dH);
    a.part = part;
    a.tiles_n = g.across;
    a.splits = plan.splits;
    g.dh_blocks = h.dH ? (g.across * plan.splits + 7) / 8 * 8 : 0;
    g.dw_per = h.dW ? (int)ceil_div(ceil_div(h.vocab, 128) * g.across, 4 * 8) : 0;
    const int64_t blocks = g.dh_blocks + 8 * (int64_t)g.dw_per;
    if (h.tokens <= REST_TOKENS) return launch_few_as<1, true>(g, blocks, stream);
    const bool rest = l.rest != nullptr;
    if (h.tokens <= 32) return rest ? launch_few_as<2, true>(g, blocks, stream) : launch_few_as<2, false>(g, blocks, stream);
    if (h.tokens <= 48) return rest ? launch_few_as<3, true>(g, blocks, stream) : launch_few_as<3, false>(g, blocks, stream);
    return rest ? launch_few_as<4, true>(g, blocks, stream) : launch_few_as<4, false>(g, blocks, stream);
}

sbn_status launch_head_backward(const HeadCall &h, void *workspace, hipStream_t stream)
{
    const bool hard = h.targets != nullptr, soft = h.top_idx != nullptr;
    uint8_t *const ws = static_cast<uint8_t *>(workspace);
    HeadRegions r;
    LogitsArgs g = logits_of(h);
    sbn_status st;
    if (soft) {
        const TeacherRegions tr(r, h.tokens, h.vocab, h.top_k);
        st = launch_teacher(h, ws, tr, g, stream);
        if (st != SBN_OK) return st;
    }
    g.lse1 = h.lse1;
    g.lse2 = h.lse2;
    g.d1 = h.d_ce;
    g.d2 = h.d_kd;
    auto sum = [&](const float *part, int64_t n, int parts, uint16_t *out) {
        if (n <= (int64_t)1 << 20 && parts >= 4) hipLaunchKernelGGL(sum_parts_kernel<8>, dim3((unsigned)ceil_div(n, 128)), dim3(256), 0, stream, part, n, parts, out, (int64_t)0);
        else   // 2^32 values at a time: a launch has fewer than 2^32 threads
            for (int64_t first = 0; first < n; first += (int64_t)1 << 32) {
                const int64_t here = std::min(n - first, (int64_t)1 << 32);
                hipLaunchKernelGGL(sum_parts_kernel<1>, dim3((unsigned)ceil_div(here, 1024)), dim3(256), 0, stream, part, n, parts, out, first);
            }
        return check_launch("sum_parts_kernel");
    };
    if (takes_few(h.tokens, h.d_in, h.vocab, soft)) {
        const FewPlan plan = plan_few(h.tokens, h.d_in, h.vocab, soft);
        g.ldg = plan.ldg;
        g.G = reinterpret_cast<uint16_t *>(ws + r.take((size_t)plan.rows * plan.ldg * 2));
        if (plan.rows > h.tokens) g.rest = g.G + h.tokens * plan.ldg;
        float *const part = reinterpret_cast<float *>(ws + r.bytes);
        const int size = logits_size(h.tokens, h.vocab, h.d_in);
        st = launch_logits<true>(g, g.rest != nullptr ? std::min(size, (int)SMALL) : size, hard, soft, stream);
        if (st == SBN_OK) st = launch_few_gradients(h, g, plan, part, stream);
        return st != SBN_OK || !h.dH || plan.parts == 1 ? st : sum(part, h.tokens * h.d_in, plan.parts, static_cast<uint16_t *>(h.dH));
    }
    const BackwardPlan plan = plan_backward(h.tokens, h.d_in, h.vocab);
    g.G = reinterpret_cast<uint16_t *>(ws + r.take((size_t)h.tokens * pitch_of(plan.ldg) * 2));
    const int dh_parts = plan.dh_parts(h.vocab), dw_parts = plan.dw_parts();
    float *const dh_part = reinterpret_cast<float *>(ws + r.take((size_t)dh_parts * h.tokens * h.d_in * 4));
    float *const dw_part = reinterpret_cast<float *>(ws + r.take((size_t)dw_parts * plan.piece * h.d_in * 4));
    const int d = (int)h.d_in, tokens = (int)h.tokens;
    for (int64_t v0 = 0; v0 < h.vocab; v0 += plan.piece) {
        const int words = (int)std::min(plan.piece, h.vocab - v0);
        g.W = static_cast<const uint16_t *>(h.W) + v0 * d;
        g.v0 = v0;
        g.words = words;
        const int64_t cols = ceil_div(words, STAGE_K) * STAGE_K;
        g.ldg = pitch_of(cols);
        st = launch_logits<true>(g, logits_size(h.tokens, words, h.d_in), hard, soft, stream);
        if (st != SBN_OK) return st;
        GradientPair pair{};
        pair.targets = h.targets;
        pair.d1 = h.d_ce;
        pair.tokens = tokens;
        pair.vocab = h.vocab;
        if (h.dW) {
            GradientArgs &a = pair.dw;
            a.P = Operand{g.H, d, d, tokens};
            a.Q = Operand{g.G, g.ldg, words, tokens};
            a.N = d;
            a.M = words;
            a.stages = (int)ceil_div(tokens, STAGE_K);
            a.splits = plan.dw_splits;
            a.C = dw_parts ? nullptr : static_cast<uint16_t *>(h.dW) + v0 * d;
            a.part = dw_part;
        }
        if (h.dH) {
            GradientArgs &a = pair.dh;
            a.P = Operand{g.W, d, d, words};
            a.Q = Operand{g.G, g.ldg, tokens, (int)cols};
            a.N = d;
            a.M = tokens;
            a.stages = (int)(cols / STAGE_K);
            a.splits = plan.dh_splits;
            a.C = dh_parts ? nullptr : static_cast<uint16_t *>(h.dH);
            a.part = dh_part;
            a.add = v0 > 0;
        }
        if (h.dW) pair.dw.per = (int)ceil_div(pair.dw.stages, pair.dw.splits);
        if (h.dH) pair.dh.per = (int)ceil_div(pair.dh.stages, pair.dh.splits);
        st = plan.size == BIG ? launch_gradients<BIG>(pair, stream) : plan.size == SMALL ? launch_gradients<SMALL>(pair, stream) : launch_gradients<TINY>(pair, stream);
        if (st != SBN_OK) return st;
        if (h.dW && dw_parts) {
            st = sum(dw_part, (int64_t)words * d, dw_parts, static_cast<uint16_t *>(h.dW) + v0 * d);
            if (st != SBN_OK) return st;
        }
    }
    return h.dH && dh_parts ? sum(dh_part, h.tokens * h.d_in, dh_parts, static_cast<uint16_t *>(h.dH)) : SBN_OK;
}

}  // namespace sbn
