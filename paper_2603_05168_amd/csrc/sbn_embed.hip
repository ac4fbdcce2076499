// Embedding: the rows of a table that the tokens name, and the gradient of the table.
//
//   Y[t,:] = scale E[ids[t],:]             (zeros where the id is outside the table)
//   dE[v,:] = scale sum_{t: ids[t] = v} dY[t,:]   (+ dE[v,:])
// Both are bound by memory: the forward moves the rows, the gradient reads dY once and writes the whole table (or, where it is added to one,
// the rows that are named).
//
// The gradient goes by sorted tokens, so that no two writers meet and a repeated call gives the same bits:
//   sort_kernel   puts the tokens in order of their ids, tokens of one id in their own order.  Ids go to blocks round-robin, which spreads the
//                 frequent ones; a block looks through all ids, counts those of lower blocks (where its share of the order begins) and its own,
//                 and places these.
//   sum_kernel    walks the order in pieces of PIECE tokens, which balances the work however often an id occurs.  An id whose tokens end in the
//                 piece that they begin in, or in the next, is written there; of one that goes on each piece leaves a partial sum in fp32.
//   join_kernel   adds the partial sums of such an id in the order of the pieces.
// Few tokens are not sorted: few_kernel.
#include <algorithm>

#include "sbn_internal.hpp"
#include "sbn_rows.hpp"

namespace sbn {

namespace {

constexpr int SORT_THREADS = 1024;
constexpr int SORT_LOADS = 8;                            // of a thread in a tile, two ids each; one where all tokens fit a tile of so few (less code to fetch)
constexpr int SORT_BITS = 15;                            // of a number up to SORT_OWN, or of a token in a tile
constexpr int SORT_OWN = 16384;                          // ids of the table that one sorting block has at most: their counts lie in LDS
constexpr int PIECE = 8;                                 // tokens of a piece: with 16 the code that a wavefront goes through once, and fetches, costs more than the rows (7 us against 11 at 1024 tokens)

// the sorting blocks are 2^sort_shift() and share out the ids of the table
inline int sort_shift(int64_t vocab)
{
    int shift = 8;
    while (vocab > (int64_t)SORT_OWN << shift) ++shift;
    return shift;
}

// A thread's U columns of a row of U values or more.  The last of a row whose length is no multiple of U begin where they still are all in the row:
// neither loads nor stores have ends to look after, and what two threads write twice is the same.
template <int U> __device__ __forceinline__ int64_t columns(int64_t unit, int64_t d) { return min(unit * U, d - U); }

// U columns of a row as they are in memory
template <sbn_dtype DT, int U> struct Raw {
    static constexpr int E = Row<DT>::E, N = U / E;
    typedef typename Row<DT>::value value;
    u32x4 v[N];
    template <bool ONCE> __device__ __forceinline__ void load(const void *row, int64_t column)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = Row<DT>::template load<ONCE>(static_cast<const value *>(row) + column, j);
    }
    __device__ __forceinline__ void store(void *row, int64_t column) const
    {
#pragma unroll
        for (int j = 0; j < N; ++j) Row<DT>::store(static_cast<value *>(row) + column, j, v[j]);
    }
    // those from column `own` on
    __device__ __forceinline__ void store_own(void *row, int64_t column, int64_t own) const
    {
        if (column == own) return store(row, column);
        value *p = static_cast<value *>(row) + column;
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (column + j * E + k >= own) p[j * E + k] = Row<DT>::get(v[j], k);
    }
    __device__ __forceinline__ void add_to(float (&sum)[U]) const
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float f[E];
            Row<DT>::unpack(v[j], f);
#pragma unroll
            for (int k = 0; k < E; ++k) sum[j * E + k] += f[k];
        }
    }
    static __device__ __forceinline__ Raw of(const float (&sum)[U])
    {
        Raw raw;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float f[E];
#pragma unroll
            for (int k = 0; k < E; ++k) f[k] = sum[j * E + k];
            raw.v[j] = Row<DT>::pack(f);
        }
        return raw;
    }
};

template <sbn_dtype DT> __device__ __forceinline__ float value_at(const void *row, int64_t column) { return Row<DT>::number(static_cast<const typename Row<DT>::value *>(row)[column]); }
template <sbn_dtype DT> __device__ __forceinline__ void set_value(void *row, int64_t column, float f)
{
    static_cast<typename Row<DT>::value *>(row)[column] = Row<DT>::rounded(f);
}

// A wavefront copies a row, four units of it at a time: 168 MB (16384 rows of 2560 bf16 values) in 27 us, where a copy of as much takes 24.
template <sbn_dtype TABLE, sbn_dtype OUT> __global__ void __launch_bounds__(256) embedding_kernel(const void *E, const int64_t *ids, int64_t tokens, int64_t vocab,
                                                                                                  int64_t d, float scale, void *Y)
{
    constexpr int U = unit_of(TABLE, OUT), AT_ONCE = 4;
    const int lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (t >= tokens) return;
    const int64_t id = ids[t];
    const bool inside = id >= 0 && id < vocab;
    const void *from = static_cast<const typename Row<TABLE>::value *>(E) + (inside ? id : 0) * d;
    void *to = static_cast<typename Row<OUT>::value *>(Y) + t * d;
    if (d < U) {
        if (lane < d) set_value<OUT>(to, lane, inside ? value_at<TABLE>(from, lane) * scale : 0.0f);
        return;
    }
    for (int64_t u0 = lane; u0 * U < d; u0 += 64 * AT_ONCE) {
        Raw<TABLE, U> rows[AT_ONCE];
        if (inside) {
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) rows[j].template load<false>(from, columns<U>(u0 + 64 * j, d));
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            if ((u0 + 64 * j) * U >= d) break;
            float f[U] = {};
            if (inside) {
                rows[j].add_to(f);
#pragma unroll
                for (int k = 0; k < U; ++k) f[k] *= scale;
            }
            Raw<OUT, U>::of(f).store(to, columns<U>(u0 + 64 * j, d));
        }
    }
}

struct SortArgs {
    const int64_t *ids;
    int64_t tokens, vocab;
    int *begin;          // [blocks * own + 1]: where the tokens of id k * blocks + b begin in the order, at b * own + k
    int *order;          // [tokens]: the tokens
    int *order_ids;      // [tokens]: their ids
    int own, shift;      // ids of a block; log2 of the blocks
    char *clear;         // the table's gradient, to be cleared by the blocks behind (null: not)
    int64_t clear_bytes;
};

// sum over the lanes up to this one, by DPP (row_shr 1, 2, 4, 8, row_bcast 15, 31)
__device__ __forceinline__ int wave_scan(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

// sum over the threads in front; total: over all of the block's
__device__ __forceinline__ int block_scan(int x, int *scratch, int &total)
{
    const int s = wave_scan(x);
    __syncthreads();   // the scratch may still be read
    if ((threadIdx.x & 63) == 63) scratch[threadIdx.x >> 6] = s;
    __syncthreads();
    // a wavefront's sum to each of 16 lanes
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, sums = wave_scan(lane < SORT_THREADS / 64 ? scratch[lane] : 0);
    total = __builtin_amdgcn_readlane(sums, 63);
    return (wave > 0 ? __builtin_amdgcn_readlane(sums, wave - 1) : 0) + s - x;
}

// A thread has tokens 2 thread and 2 thread + 1 of each of the SORT_LOADS runs of a tile: whole lines to a wavefront's load (eight tokens in a row to a
// thread are a line to each lane: 27 us for 16384 tokens in place of 13).  Ids outside the table, and those behind the last token, as -1.
template <int LOADS> struct Ids {
    typedef int64_t i64x2 __attribute__((ext_vector_type(2), aligned(8)));
    i64x2 v[LOADS];
    __device__ __forceinline__ void load(const SortArgs &s, int64_t tile)
    {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int64_t t = tile + (int64_t)j * 2 * SORT_THREADS + threadIdx.x * 2;
            v[j] = (i64x2){-1, -1};
            if (t + 1 < s.tokens)
                v[j] = *reinterpret_cast<const i64x2 *>(s.ids + t);
            else if (t < s.tokens)
                v[j][0] = s.ids[t];
        }
    }
    __device__ __forceinline__ void in_table(const SortArgs &s, int (&id)[LOADS][2]) const
    {
#pragma unroll
        for (int j = 0; j < LOADS; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) id[j][e] = v[j][e] >= 0 && v[j][e] < s.vocab ? (int)v[j][e] : -1;
    }
};

// Clears the table's gradient: 256 threads of each of CLEARING blocks, from one end to the other, so that all stores of a moment lie near each other (a
// plain fill of 671 MB: 106 us so, by 1024 threads of each 119, by pieces of 64 KB to a block 128).  The first block clears what lies off 16 bytes at
// either end too (whole values: two bytes at least).
constexpr int CLEARING = 256, CLEARING_THREADS = 256;
__device__ __forceinline__ void clear(const SortArgs &s)
{
    if (threadIdx.x >= CLEARING_THREADS) return;
    char *const end = s.clear + s.clear_bytes;
    char *const first = min(end, s.clear + (-reinterpret_cast<uintptr_t>(s.clear) & 15)), *const last = first + (end - first) / 16 * 16;
    const u32x4 zero = {0, 0, 0, 0};
    for (char *p = first + ((int64_t)blockIdx.x * CLEARING_THREADS + threadIdx.x) * 16; p < last; p += (int64_t)CLEARING * CLEARING_THREADS * 16)
        *reinterpret_cast<u32x4 *>(p) = zero;
    if (blockIdx.x == 0 && threadIdx.x < 16) {
        uint16_t *const front = reinterpret_cast<uint16_t *>(s.clear) + threadIdx.x, *const back = reinterpret_cast<uint16_t *>(last) + threadIdx.x;
        if (reinterpret_cast<char *>(front) < first) *front = 0;
        if (reinterpret_cast<char *>(back) < end) *back = 0;
    }
}

__global__ void __launch_bounds__(CLEARING_THREADS) clear_kernel(const SortArgs s) { clear(s); }

// The last 2^shift blocks sort; CLEARING in front of them (where there is something to clear) clear the table's gradient meanwhile, all of it: the rows that
// have one are written again by the next kernel.
template <int LOADS> __global__ void __launch_bounds__(SORT_THREADS) sort_kernel(const SortArgs s)
{
    if (s.clear && blockIdx.x < CLEARING) {
        clear(s);
        return;
    }
    constexpr int WAVES = SORT_THREADS / 64, TILE = SORT_THREADS * LOADS * 2;
    extern __shared__ int next[];                // [own]: counts, then where the next token of an id goes
    __shared__ int scratch[WAVES];
    __shared__ int counts[LOADS * WAVES];   // of the block's tokens, in the tile's order
    __shared__ uint32_t found[TILE];        // which of the block's ids << SORT_BITS | token of the tile, in the order of the tokens
    const int block = blockIdx.x - (s.clear ? CLEARING : 0), lane = threadIdx.x & 63, mask = (1 << s.shift) - 1;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int k = threadIdx.x; k < s.own; k += SORT_THREADS) next[k] = 0;
    __syncthreads();
    int lower = 0;
    int id[LOADS][2];
    Ids<LOADS> ahead;   // of the tile that comes next
    const int64_t last_tile = (s.tokens - 1) / TILE * TILE;
    ahead.load(s, last_tile);
    for (int64_t tile = last_tile; tile >= 0; tile -= TILE) {   // the first tile last: its ids are at hand below
        ahead.in_table(s, id);
        if (tile > 0) ahead.load(s, tile - TILE);
#pragma unroll
        for (int j = 0; j < LOADS; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int b = id[j][e] & mask;
                lower += id[j][e] >= 0 && b < block;
                if (id[j][e] >= 0 && b == block) atomicAdd(&next[id[j][e] >> s.shift], 1);   // whole numbers: in any order
            }
    }
    int at;
    block_scan(lower, scratch, at);
    // from counts to beginnings: each thread a run of ids
    const int run = (s.own + SORT_THREADS - 1) / SORT_THREADS;
    const int k0 = min(s.own, (int)threadIdx.x * run), k1 = min(s.own, k0 + run);
    int count_here = 0, all;
    for (int k = k0; k < k1; ++k) count_here += next[k];
    int begin = at + block_scan(count_here, scratch, all);
    for (int k = k0; k < k1; ++k) {
        const int count = next[k];
        next[k] = begin;
        s.begin[(int64_t)block * s.own + k] = begin;
        begin += count;
    }
    if (block == mask && threadIdx.x == 0) s.begin[(int64_t)s.own << s.shift] = at + all;
    if (!all) return;
    const uint64_t in_front = (1ull << lane) - 1;
    const int bits = 32 - __builtin_clz(s.own);
    for (int64_t tile = 0; tile < s.tokens; tile += TILE) {
        // the tile's tokens of this block, side by side and in their order
        if (tile > 0) ahead.in_table(s, id);
        if (tile + TILE < s.tokens) ahead.load(s, tile + TILE);
        int place[LOADS][2];
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            uint64_t has[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                id[j][e] = id[j][e] >= 0 && (id[j][e] & mask) == block ? id[j][e] >> s.shift : -1;
                has[e] = __ballot(id[j][e] >= 0);
            }
            place[j][0] = __popcll(has[0] & in_front) + __popcll(has[1] & in_front);
            place[j][1] = place[j][0] + (int)(has[0] >> lane & 1);
            if (lane == 0) counts[j * WAVES + wave] = __popcll(has[0]) + __popcll(has[1]);
        }
        __syncthreads();
        static_assert(LOADS * WAVES <= 128, "two counts to a lane");
        const bool counted = 2 * lane < LOADS * WAVES;
        const int c0 = counted ? counts[2 * lane] : 0, c1 = counted ? counts[2 * lane + 1] : 0, upto = wave_scan(c0 + c1);
        const int total = __builtin_amdgcn_readlane(upto, 63);
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int k = j * WAVES + wave;
            const int before = __builtin_amdgcn_readlane(upto, k / 2) - __builtin_amdgcn_readlane(k & 1 ? c1 : c0 + c1, k / 2);
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (id[j][e] >= 0) found[before + place[j][e]] = (uint32_t)id[j][e] << SORT_BITS | (j * 2 * SORT_THREADS + threadIdx.x * 2 + e);
        }
        __syncthreads();
        // Each wavefront has 64 of them and counts, of every token, those of its id among the lanes in front (lanes whose ids agree in every bit).  Then
        // the wavefronts take their places in turn.
        for (int first = 0; first < total; first += SORT_THREADS) {
            const int i = first + threadIdx.x;
            const bool live = i < total;
            const uint32_t f = live ? found[i] : 0, of = f >> SORT_BITS;
            uint64_t same = __ballot(live);
            for (int b = 0; b < bits; ++b) {
                const uint64_t set = __ballot(of >> b & 1);
                same &= of >> b & 1 ? set : ~set;
            }
            const int nearer = __popcll(same & in_front);
            const bool last = nearer == __popcll(same) - 1;
            int to = 0;
            for (int w = 0; first + w * 64 < total && w < WAVES; ++w) {
                if (w == wave && live) {
                    to = next[of] + nearer;
                    if (last) next[of] = to + 1;   // (behind the reads of all lanes: a wavefront's accesses to LDS are done in their order)
                }
                __syncthreads();
            }
            if (live) {
                s.order[to] = (int)(tile + (f & ((1 << SORT_BITS) - 1)));
                s.order_ids[to] = (int)(of << s.shift) + block;
            }
        }
        __syncthreads();
    }
}

struct SumArgs {
    const void *dY;
    void *dE;
    const int *begin, *order, *order_ids;
    float *partials;     // [pieces][2][d]: of the id that the piece begins with, of the one that it ends with
    int64_t d, items;    // items: pieces times tiles
    int tokens, own, shift, accumulate, pieces, tiles, join_pieces;   // tiles: of 64 units of a row
    float scale;
    __device__ __forceinline__ const int *begin_of(int64_t id) const { return begin + (id & ((1 << shift) - 1)) * own + (id >> shift); }
    __device__ __forceinline__ int total() const { return begin[(int64_t)own << shift]; }   // tokens whose id is in the table
};

template <sbn_dtype TABLE> __device__ __forceinline__ void *row_of(const SumArgs &s, int id)
{
    return static_cast<typename Row<TABLE>::value *>(s.dE) + (int64_t)id * s.d;
}

// whether an id's tokens, from place `begin` of the order on, all go with the piece that they begin in: they end in it or in the next
__device__ __forceinline__ bool of_one_piece(int begin, int end) { return end <= (begin / PIECE + 2) * PIECE; }

// what a piece has to do; the same for a whole wavefront
struct Piece {
    int token, id;          // of its places, and of those around it, one to a lane: place k at lane PIECE + 1 + k
    int first_k, end_k;     // its places
    bool begun, goes_on;    // the first id's tokens begin in an earlier piece; the last id's go on in a later one
    __device__ __forceinline__ int token_at(int k) const { return __builtin_amdgcn_readlane(token, PIECE + 1 + k); }
    __device__ __forceinline__ int id_at(int k) const { return __builtin_amdgcn_readlane(id, PIECE + 1 + k); }
    __device__ __forceinline__ bool last_of_id(int k) const { return k + 1 == end_k || id_at(k) != id_at(k + 1); }
    // how many places an id has that has place k, and no more than PIECE from there on
    __device__ __forceinline__ int places_of(int which, int k) const
    {
        return __popcll(__ballot(id == which) >> (PIECE + 1 + k) & ((1ull << PIECE) - 1));
    }
};

// All rows are asked for before the first is added, those of places that are not the piece's too: nothing branches between the loads (in which case each
// waited for the one before: 22 us in place of 14 for 2125 tokens of 2120 values).
template <sbn_dtype TABLE, sbn_dtype OUT, bool ACCUMULATE> __device__ __forceinline__ void sum_piece(const SumArgs &s, const Piece &piece, int number, int64_t u)
{
    constexpr int U = unit_of(TABLE, OUT);
    const int64_t c = columns<U>(u, s.d);
    float sum[U] = {}, sum_begun[U] = {};
    bool first = piece.begun;   // the present id is the piece's first, and begins in an earlier one
#pragma unroll 1
    for (int k0 = 0; k0 < piece.end_k; k0 += PIECE) {
        Raw<OUT, U> rows[PIECE];
        Raw<TABLE, U> old[ACCUMULATE ? PIECE : 1];
#pragma unroll
        for (int k = 0; k < PIECE; ++k) {
            rows[k].template load<true>(static_cast<const typename Row<OUT>::value *>(s.dY) + (int64_t)piece.token_at(k0 + k) * s.d, c);
            if (ACCUMULATE) old[k].template load<false>(row_of<TABLE>(s, max(piece.id_at(k0 + k), 0)), c);
        }
#pragma unroll
        for (int k = 0; k < PIECE; ++k)
            if (k0 + k >= piece.first_k && k0 + k < piece.end_k) {
                rows[k].add_to(sum);
                if (!piece.last_of_id(k0 + k) || (k0 + k + 1 == piece.end_k && (first || piece.goes_on))) continue;
                if (first) {
#pragma unroll
                    for (int i = 0; i < U; ++i) sum_begun[i] = sum[i];
                } else {
#pragma unroll
                    for (int i = 0; i < U; ++i) sum[i] *= s.scale;
                    if (ACCUMULATE) old[k].add_to(sum);
                    const Raw<TABLE, U> done = Raw<TABLE, U>::of(sum);
                    void *row = row_of<TABLE>(s, piece.id_at(k0 + k));
                    ACCUMULATE ? done.store_own(row, c, u * U) : done.store(row, c);   // (what is added to must not be written twice)
                }
                first = false;
#pragma unroll
                for (int i = 0; i < U; ++i) sum[i] = 0.0f;
            }
    }
    // partial sums: of the first id where it is not the last too, and of the last
    float *share = s.partials + (int64_t)number * 2 * s.d;
    if (piece.begun && !first) Raw<SBN_F32, U>::of(sum_begun).store(share, c);
    if (first)
        Raw<SBN_F32, U>::of(sum).store(share, c);
    else if (piece.goes_on)
        Raw<SBN_F32, U>::of(sum).store(share + s.d, c);
}

// the same for rows of less than U values, one to a lane
template <sbn_dtype TABLE, sbn_dtype OUT> __device__ __forceinline__ void sum_piece_few(const SumArgs &s, const Piece &piece, int number, int lane)
{
    float *share = s.partials + (int64_t)number * 2 * s.d;
    const int c = min(lane, (int)s.d - 1);
    float sum = 0.0f;
    bool first = piece.begun;
#pragma unroll 1
    for (int k = piece.first_k; k < piece.end_k; ++k) {
        sum += value_at<OUT>(static_cast<const typename Row<OUT>::value *>(s.dY) + (int64_t)piece.token_at(k) * s.d, c);
        if (!piece.last_of_id(k)) continue;
        void *row = row_of<TABLE>(s, piece.id_at(k));
        if (lane < s.d) {
            if (first)
                share[c] = sum;
            else if (k + 1 == piece.end_k && piece.goes_on)
                share[s.d + c] = sum;
            else
                set_value<TABLE>(row, c, s.accumulate ? sum * s.scale + value_at<TABLE>(row, c) : sum * s.scale);
        }
        first = false;
        sum = 0.0f;
    }
}

// a wavefront has a piece and 64 units of its columns
template <sbn_dtype TABLE, sbn_dtype OUT, bool ACCUMULATE> __global__ void __launch_bounds__(256) sum_kernel(const SumArgs s)
{
    constexpr int U = unit_of(TABLE, OUT);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * 4 + wave;
    if (item >= s.items) return;
    const int number = (int)(item / s.tiles), p0 = number * PIECE;
    const int64_t u = (item - (int64_t)number * s.tiles) * 64 + lane;
    // the places from the one in front of the piece before on, to the first behind the piece after: one to a lane
    constexpr int HERE = PIECE + 1;
    const int place = p0 + lane - HERE, at = min(max(place, 0), s.tokens - 1);
    const int total = s.total(), token = s.order[at], id = s.order_ids[at];
    if (p0 >= total) return;
    const bool there = place >= 0 && place < total;   // (behind the last there is anything)
    Piece piece;
    piece.token = there ? token : __builtin_amdgcn_readlane(token, HERE);
    piece.id = there ? id : -1;
    const int p1 = min(total, p0 + PIECE), front = piece.id_at(-1), behind = piece.id_at(PIECE);
    piece.first_k = 0;
    piece.end_k = p1 - p0;
    // an id that begins in a piece and ends in the next is the former's: no partial sums of ids of few tokens
    piece.begun = piece.id_at(0) == front;
    if (piece.begun && front != piece.id_at(-HERE) && front != behind) {
        piece.first_k = piece.places_of(front, 0);
        piece.begun = false;
    }
    piece.goes_on = behind >= 0 && piece.id_at(PIECE - 1) == behind;
    if (piece.goes_on && behind != front && behind != piece.id_at(2 * PIECE)) {
        piece.end_k = PIECE + piece.places_of(behind, PIECE);
        piece.goes_on = false;
    }
    if (s.d < U)
        sum_piece_few<TABLE, OUT>(s, piece, number, lane);
    else   // lanes behind the row's end too, for the places that they hold: they read and write its last columns, which others do alike
        sum_piece<TABLE, OUT, ACCUMULATE>(s, piece, number, u);
}

template <sbn_dtype TABLE, int U, int WAVES, int AT_ONCE>
__device__ __forceinline__ void join(const SumArgs &s, int piece, int id, int end, int lane, int wave, float (*sums)[64 * U])
{
    const int64_t u = (int64_t)blockIdx.y * 64 + lane;
    const int count = (end - 1) / PIECE - piece + 1;   // pieces that the id has a share of: the last of the first one, the first of the others
    float sum[U] = {};
    const auto add = [&](auto load) {
        for (int q0 = wave; q0 < count; q0 += WAVES * AT_ONCE) {
            float f[AT_ONCE][U];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                const int q = min(q0 + WAVES * j, count - 1);
                load(s.partials + ((int64_t)(piece + q) * 2 + (q == 0)) * s.d, f[j]);
            }
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j)
                if (q0 + WAVES * j < count) {
#pragma unroll
                    for (int k = 0; k < U; ++k) sum[k] += f[j][k];
                }
        }
    };
    if ((u + 1) * U <= s.d)
        add([&](const float *share, float (&f)[U]) { load_floats<U>(share, u * U, u * U + U, 0.0f, f); });
    else
        add([&](const float *share, float (&f)[U]) { load_floats<U>(share, u * U, s.d, 0.0f, f); });
    __syncthreads();   // the sums may still be read
#pragma unroll
    for (int k = 0; k < U; ++k) sums[wave][k * 64 + lane] = sum[k];
    __syncthreads();
    if (wave > 0 || u * U >= s.d) return;
    for (int w = 1; w < min(WAVES, count); ++w) {
#pragma unroll
        for (int k = 0; k < U; ++k) sum[k] += sums[w][k * 64 + lane];
    }
    void *row = row_of<TABLE>(s, id);
    float old[U] = {};
    if (s.accumulate) load_unit<TABLE, U>(row, u, s.d, old);
#pragma unroll
    for (int k = 0; k < U; ++k) sum[k] = s.accumulate ? sum[k] * s.scale + old[k] : sum[k] * s.scale;
    store_unit<TABLE, U>(row, u, s.d, sum);
}

// A block to join_pieces pieces and 64 units of the columns.  For every piece in which an id begins that goes on behind the next, eight wavefronts add the
// partial sums in turn, eight asked for at a time, and their sums are added in order (sixteen wavefronts: 9.5 us in place of 8.3 for 16384 tokens of 2560
// values, four 9.4; one id of 65536 tokens: 187, 175 and 289, beside 255 of the sort, in which
// one block places all of them, and 74 of the sums).
constexpr int JOIN_THREADS = 512;
template <sbn_dtype TABLE> __global__ void __launch_bounds__(JOIN_THREADS) join_kernel(const SumArgs s)
{
    constexpr int U = Row<TABLE>::E, WAVES = JOIN_THREADS / 64, AT_ONCE = 8;
    __shared__ float sums[WAVES][64 * U];
    const int total = s.total();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // a piece to a lane
    const int64_t p0 = ((int64_t)blockIdx.x * s.join_pieces + lane) * PIECE, p1 = p0 + PIECE;
    int id = -1, end = 0;
    if (lane < s.join_pieces && p1 < total) {
        id = s.order_ids[p1];
        const bool begins = s.order_ids[p1 - 1] == id && (p0 == 0 || s.order_ids[p0 - 1] != id);
        if (begins) end = s.begin_of(id)[1];
        if (!begins || of_one_piece((int)p0, end)) id = -1;
    }
    for (uint64_t todo = __ballot(id >= 0); todo; todo &= todo - 1) {
        const int k = __builtin_ctzll(todo);
        join<TABLE, U, WAVES, AT_ONCE>(s, blockIdx.x * s.join_pieces + k, __builtin_amdgcn_readlane(id, k), __builtin_amdgcn_readlane(end, k), lane, wave, sums);
    }
}

struct FewArgs {
    const int64_t *ids;
    const void *dY;
    void *dE;
    int64_t vocab, d;
    int tokens, tiles;   // tiles: of 64 units of a row
    float scale;
};

// The gradient of few tokens in one launch: a block to a token looks through all ids and lists the tokens that share its own.  The columns of an id are dealt to
// the blocks of its first tokens, as many as there are tiles; the other blocks end.  Wavefronts take tiles of their own, or, where a block has fewer and the
// tokens are many, runs of the list, whose sums are added in order.  Every row is read once and each of its values written by one thread.
// Bound by launches and trips to memory: added to a bf16 table of 2560 columns, 32 tokens take 3.4 us where the three launches by sorted tokens take 10.5, 512
// 4.2 (12.2), 1024 7.0 (12.7), 1531 10.0 (13.4); tokens of one id 1024 16.9 (17.5), 1531 23.2 (21.7).  Four wavefronts to a block: 3.5, 4.3, 5.5 and 7.5, but 26.5 and
// 37.7 where the id is one.  At 2048 tokens it is 13.2 against 15.5, and 30.9 against 25.6 where the id is one, 33 against 26 in rows of 7536: the others go by sorted tokens.
constexpr int FEW_WAVES = 8, FEW_LOADS = 3, FEW_TOKENS = FEW_WAVES * FEW_LOADS * 64, FEW_ROWS = 8;
template <sbn_dtype TABLE, sbn_dtype OUT, bool ACCUMULATE> __global__ void __launch_bounds__(FEW_WAVES * 64) few_kernel(const FewArgs s)
{
    constexpr int U = unit_of(TABLE, OUT);
    __shared__ int counts[FEW_WAVES], ranks[FEW_WAVES];
    __shared__ uint16_t list[FEW_TOKENS];
    __shared__ float sums[FEW_WAVES][64 * U];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = blockIdx.x;
    const int per = (s.tokens + FEW_WAVES * 64 - 1) / (FEW_WAVES * 64), begin = wave * per * 64;   // a wavefront's run of tokens
    int64_t ids[FEW_LOADS];
#pragma unroll
    for (int c = 0; c < FEW_LOADS; ++c) ids[c] = s.ids[min(begin + c * 64 + lane, s.tokens - 1)];
    const int64_t id = s.ids[t];
    if (id < 0 || id >= s.vocab) return;
    uint64_t same[FEW_LOADS];
    int count = 0, rank = 0;
#pragma unroll
    for (int c = 0; c < FEW_LOADS; ++c) {
        const int first = begin + c * 64;
        same[c] = __ballot(c < per && first + lane < s.tokens && ids[c] == id);
        count += __popcll(same[c]);
        rank += __popcll(t >= first + 64 ? same[c] : t <= first ? 0 : same[c] & ((1ull << (t - first)) - 1));
    }
    if (lane == 0) {
        counts[wave] = count;
        ranks[wave] = rank;
    }
    __syncthreads();
    int in_front = 0, n = 0;
    rank = 0;
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w) {
        if (w == wave) in_front = n;
        n += counts[w];
        rank += ranks[w];
    }
    n = __builtin_amdgcn_readfirstlane(n);   // (the same in all threads)
    rank = __builtin_amdgcn_readfirstlane(rank);
    const int blocks = min(n, s.tiles);
    if (rank >= blocks) return;
#pragma unroll
    for (int c = 0; c < FEW_LOADS; ++c) {
        if (same[c] >> lane & 1) list[in_front + __popcll(same[c] & ((1ull << lane) - 1))] = (uint16_t)(begin + c * 64 + lane);
        in_front += __popcll(same[c]);
    }
    __syncthreads();
    const int mine = (s.tiles - rank + blocks - 1) / blocks;   // tiles rank, rank + blocks, ...
    void *const row = static_cast<typename Row<TABLE>::value *>(s.dE) + id * s.d;
    const auto row_at = [&](int token) { return static_cast<const typename Row<OUT>::value *>(s.dY) + (int64_t)token * s.d; };
    const auto unit_at = [&](int j) { return (int64_t)(rank + j * blocks) * 64 + lane; };
    const auto finish = [&](float (&sum)[U], const Raw<TABLE, U> &old, int64_t u) {
#pragma unroll
        for (int k = 0; k < U; ++k) sum[k] *= s.scale;
        if (ACCUMULATE) old.add_to(sum);
        Raw<TABLE, U>::of(sum).store_own(row, columns<U>(u, s.d), u * U);
    };
    // one or two tokens: several tiles of a wavefront at once
    if (n <= 2) {
        constexpr int TILES = 4 / Raw<OUT, U>::N;
        const void *one = row_at(__builtin_amdgcn_readfirstlane(list[0])), *two = row_at(__builtin_amdgcn_readfirstlane(list[n - 1]));
#pragma unroll 1
        for (int j = wave; j < mine; j += FEW_WAVES * TILES) {
            Raw<OUT, U> first[TILES], second[TILES];
            Raw<TABLE, U> old[TILES];
#pragma unroll
            for (int q = 0; q < TILES; ++q) {   // (tiles past the row's end: its last columns)
                const int64_t c = columns<U>(unit_at(j + q * FEW_WAVES), s.d);
                first[q].template load<true>(one, c);
                if (ACCUMULATE) old[q].template load<false>(row, c);
            }
            if (n == 2) {
#pragma unroll
                for (int q = 0; q < TILES; ++q) second[q].template load<true>(two, columns<U>(unit_at(j + q * FEW_WAVES), s.d));
            }
#pragma unroll
            for (int q = 0; q < TILES; ++q) {
                const int64_t u = unit_at(j + q * FEW_WAVES);
                if (j + q * FEW_WAVES >= mine || u * U >= s.d) break;
                float sum[U] = {};
                first[q].add_to(sum);
                if (n == 2) second[q].add_to(sum);
                finish(sum, old[q], u);
            }
        }
        return;
    }
    constexpr int ROWS = FEW_ROWS / Raw<OUT, U>::N;
    const int runs = mine >= FEW_WAVES ? 1 : min(FEW_WAVES / mine, (n + ROWS - 1) / ROWS), at_once = FEW_WAVES / runs;
    const int run = (n + runs - 1) / runs, part = wave % runs, r0 = part * run, r1 = min(n, r0 + run);
#pragma unroll 1
    for (int j = wave / runs; j - wave / runs < mine; j += at_once) {   // (more than once only where runs is 1)
        const int64_t u = unit_at(j), c = columns<U>(u, s.d);
        const bool live = wave / runs < at_once && j < mine;   // of a whole wavefront: all its lanes have tokens to name, those behind the row's end too
        float sum[U] = {};
        Raw<TABLE, U> old;
        if (live) {
            if (ACCUMULATE) old.template load<false>(row, c);
#pragma unroll 1
            for (int r = r0; r < r1; r += ROWS) {
                const int some = list[min(r + lane, r1 - 1)];
                Raw<OUT, U> rows[ROWS];
#pragma unroll
                for (int k = 0; k < ROWS; ++k) rows[k].template load<true>(row_at(__builtin_amdgcn_readlane(some, k)), c);
#pragma unroll
                for (int k = 0; k < ROWS; ++k)
                    if (r + k < r1) rows[k].add_to(sum);
            }
        }
        if (runs > 1) {
#pragma unroll
            for (int k = 0; k < U; ++k) sums[wave][k * 64 + lane] = sum[k];
            __syncthreads();
            if (part == 0) {
                for (int w = 1; w < runs; ++w) {
#pragma unroll
                    for (int k = 0; k < U; ++k) sum[k] += sums[min(wave + w, FEW_WAVES - 1)][k * 64 + lane];
                }
            }
        }
        if (live && part == 0 && u * U < s.d) finish(sum, old, u);
    }
}

struct Carved {
    size_t begin, order, order_ids, partials, total;
};
Carved carve(int64_t tokens, int64_t d, int64_t vocab)
{
    Carved c;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at = align_up(at + bytes, 256);
        return here;
    };
    const int shift = sort_shift(vocab);
    c.begin = take((size_t)((ceil_div(vocab, (int64_t)1 << shift) << shift) + 1) * sizeof(int));
    c.order = take((size_t)tokens * sizeof(int));
    c.order_ids = take((size_t)tokens * sizeof(int));
    c.partials = take((size_t)ceil_div(tokens, PIECE) * 2 * d * sizeof(float));
    c.total = at;
    return c;
}

template <int LOADS> sbn_status launch_sort(const SortArgs &s, hipStream_t stream)
{
    static thread_local int raised_on = -1;   // the device on which this thread has raised the kernel's LDS
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e == hipSuccess && device != raised_on)
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(sort_kernel<LOADS>), hipFuncAttributeMaxDynamicSharedMemorySize, SORT_OWN * sizeof(int));
    if (e != hipSuccess) {
        set_hip_error(e, "hipFuncSetAttribute(sort_kernel)");
        return SBN_EHIP;
    }
    raised_on = device;
    hipLaunchKernelGGL(sort_kernel<LOADS>, dim3((unsigned)((1 << s.shift) + (s.clear ? CLEARING : 0))), dim3(SORT_THREADS), (size_t)s.own * sizeof(int), stream, s);
    return check_launch("sort_kernel");
}

template <sbn_dtype TABLE, sbn_dtype OUT> void few_as(FewArgs f, bool accumulate, hipStream_t stream)
{
    f.tiles = (int)ceil_div(f.d, 64 * unit_of(TABLE, OUT));
    const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)f.tokens), dim3(FEW_WAVES * 64), 0, stream, f); };
    accumulate ? launch(few_kernel<TABLE, OUT, true>) : launch(few_kernel<TABLE, OUT, false>);
}

template <sbn_dtype TABLE, sbn_dtype OUT> sbn_status sum_as(SumArgs s, hipStream_t stream)
{
    s.tiles = (int)ceil_div(s.d, 64 * unit_of(TABLE, OUT));
    s.items = (int64_t)s.pieces * s.tiles;
    const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(s.items, 4)), dim3(256), 0, stream, s); };
    s.accumulate ? launch(sum_kernel<TABLE, OUT, true>) : launch(sum_kernel<TABLE, OUT, false>);
    if (s.pieces > 2) {   // (an id of two pieces is one piece's)
        // up to four pieces to a block: most only look, but ids of one block wait for each other (16384 tokens of 2560 values by one 14.9 us, two 11.4, four 8.3,
        // eight 8.2; 65536 of 50000 ids, the frequent ones more often: four 39, eight 45; 1531 tokens of 1001: one and two 4.8, four 6.2)
        const int64_t tiles = ceil_div(s.d, 64 * Row<TABLE>::E);
        s.join_pieces = (int)std::min<int64_t>(4, ceil_div((s.pieces - 2) * tiles, 1024));
        hipLaunchKernelGGL(join_kernel<TABLE>, dim3((unsigned)ceil_div(s.pieces - 2, s.join_pieces), (unsigned)tiles), dim3(JOIN_THREADS), 0, stream, s);
    }
    return check_launch("sum_kernel");
}

}  // namespace

size_t embedding_workspace_bytes(int64_t tokens, int64_t d, int64_t vocab) { return carve(tokens, d, vocab).total; }

sbn_status launch_embedding(const void *E, sbn_dtype table, int64_t vocab, int64_t d, const int64_t *ids, int64_t tokens, float scale, void *Y, sbn_dtype out,
                            hipStream_t stream)
{
    const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(tokens, 4)), dim3(256), 0, stream, E, ids, tokens, vocab, d, scale, Y); };
    if (table == SBN_BF16)
        out == SBN_BF16 ? launch(embedding_kernel<SBN_BF16, SBN_BF16>) : launch(embedding_kernel<SBN_BF16, SBN_F32>);
    else
        out == SBN_BF16 ? launch(embedding_kernel<SBN_F32, SBN_BF16>) : launch(embedding_kernel<SBN_F32, SBN_F32>);
    return check_launch("embedding_kernel");
}

sbn_status launch_embedding_backward(const void *dY, sbn_dtype out, const int64_t *ids, int64_t tokens, int64_t vocab, int64_t d, float scale, bool accumulate,
                                     void *dE, sbn_dtype table, void *workspace, hipStream_t stream)
{
    const Carved c = carve(tokens, d, vocab);
    char *ws = static_cast<char *>(workspace);
    SortArgs o{};
    o.ids = ids;
    o.tokens = tokens;
    o.vocab = vocab;
    o.begin = reinterpret_cast<int *>(ws + c.begin);
    o.order = reinterpret_cast<int *>(ws + c.order);
    o.order_ids = reinterpret_cast<int *>(ws + c.order_ids);
    o.shift = sort_shift(vocab);
    o.own = (int)ceil_div(vocab, (int64_t)1 << o.shift);
    if (!accumulate) {
        o.clear = static_cast<char *>(dE);
        o.clear_bytes = vocab * d * (table == SBN_BF16 ? 2 : 4);
    }
    if (tokens <= FEW_TOKENS && d >= 8) {   // (rows of a whole unit)
        if (o.clear) hipLaunchKernelGGL(clear_kernel, dim3(CLEARING), dim3(CLEARING_THREADS), 0, stream, o);
        FewArgs f{};
        f.ids = ids;
        f.dY = dY;
        f.dE = dE;
        f.vocab = vocab;
        f.d = d;
        f.tokens = (int)tokens;
        f.scale = scale;
        if (table == SBN_BF16)
            out == SBN_BF16 ? few_as<SBN_BF16, SBN_BF16>(f, accumulate, stream) : few_as<SBN_BF16, SBN_F32>(f, accumulate, stream);
        else
            out == SBN_BF16 ? few_as<SBN_F32, SBN_BF16>(f, accumulate, stream) : few_as<SBN_F32, SBN_F32>(f, accumulate, stream);
        return check_launch("few_kernel");
    }
    const sbn_status st = tokens <= SORT_THREADS * 2 ? launch_sort<1>(o, stream) : launch_sort<SORT_LOADS>(o, stream);
    if (st != SBN_OK) return st;
    SumArgs s{};
    s.dY = dY;
    s.dE = dE;
    s.begin = o.begin;
    s.order = o.order;
    s.order_ids = o.order_ids;
    s.partials = reinterpret_cast<float *>(ws + c.partials);
    s.d = d;
    s.tokens = (int)tokens;
    s.own = o.own;
    s.shift = o.shift;
    s.accumulate = accumulate;
    s.pieces = (int)ceil_div(tokens, PIECE);
    s.scale = scale;
    if (table == SBN_BF16) return out == SBN_BF16 ? sum_as<SBN_BF16, SBN_BF16>(s, stream) : sum_as<SBN_BF16, SBN_F32>(s, stream);
    return out == SBN_BF16 ? sum_as<SBN_F32, SBN_BF16>(s, stream) : sum_as<SBN_F32, SBN_F32>(s, stream);
}

}  // namespace sbn
