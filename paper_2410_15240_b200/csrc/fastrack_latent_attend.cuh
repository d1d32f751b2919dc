// fastrack_latent_attend.cuh -- attention in the latent space: the kernel for single tokens, drafts and trees of drafts.
#pragma once
#include "fastrack_latent_device.cuh"

// 64 rows of queries (token, head) against tiles of 64 tokens, of which a tile in shared memory serves as K and as V:
//     S = Q C^T         64 x 64, M = rows, N = tokens, over latent + rope channels
//     O^T += C^T P^T    latent x rows, M = 128 channels at a time, N = rows, over the tile's tokens
// The second product is taken the other way round: the accumulator of 64 rows x 512 channels then takes 4 x 64 columns of tensor memory with
// all 128 lanes, N follows the number of rows that there are, and S keeps its two buffers beside it.  (With rows as M, 512 columns would be
// full of O alone, half of their lanes idle.)  Warps 0-7 make the weights and write them to shared memory; warp 8 brings the
// tiles; warp 9 issues the products.  The scores of the next tile are made while this one's weights are.
//
// All work is one line: for each sequence, for each group of row tiles, the tiles of tokens that the group sees.  The line is cut into equal
// runs, one for each group of CTAs (a CTA per row tile of a group; the CTAs of a group read the same tokens at the same time, all but the first
// out of L2).  What a run cuts is joined by a kernel of its own; a run has at most two such pieces, its first and its last.
//
// Weights enter the second product in 16 bits, as the latents are held: the answer is off by some half of its own rounding more (error against 64 bits
// bf16 0.0021 beside the rounding's 0.0017, f16 0.00021 to 0.00029 beside 0.00021).  Scores, references, sums and answers are kept in 32 bits.
//
// What bounds it, per tile, 512 + 64 channels and 64 rows: the scores' 36 products take 33 cycles each and the answers' 16 take 48 (64 rows as M,
// or 64 as N: shared memory's 128 bytes a cycle are what the operands wait for), 1960 together; memory brings a tile in 2500 at its SM's share.  It takes
// 3300: what is used again comes back some 1900 cycles after its last use, Q and two tiles are all that shared memory holds, and a tile's chain (scores,
// weights, answers) is 4200 long.  61 sequences of up to 4096 tokens, 128 heads, bf16: 94 us with the join's 14; 4 of up to 131 072, 64 heads, f16: 120 to 138 us
// (3.7 to 4.3 TB/s); 15 trees of 25 over up to 5000 tokens in blocks of 16, 16 heads: 108 us.  What it came from: copies and products issued by one
// lane 228, 267 and 224 us; a barrier per 64 or 128 channels and redundant waits 119, 144 and 140.  Tried instead: a part of a tile per 128 channels
// (107, 160, 136 us), 5 or 9 warps for small blocks' copies (no change).
#define LT_ROWS 64
#define LT_TOKENS 64
#define LT_A_THREADS 384
#define LT_A_BRINGERS 3                 // warps that bring tiles of small blocks
#define LT_A_STAGES 4                   // at most
// PAIRS: of 64 channels of the latent
template <int PAIRS> struct LtTile {
    static constexpr int CHUNKS = 2 * PAIRS + 1, BYTES = CHUNKS * 64 * LT_CHUNK_ROW, STAGES = PAIRS > 2 ? 2 : 4;
    static constexpr int FIRST = PAIRS > 1 ? PAIRS / 2 : 1;                  // pairs of a tile's first part; the second has the rest and the shared key
    static constexpr int P = (1 + STAGES) * BYTES, MISC = P + 64 * LT_CHUNK_ROW, SMEM = MISC + 2048 + 1024;    // after Q and the stages; room to round the base up
};
#define LT_A_AHEAD 2                    // the tile that is brought to L2 in advance (4: 4 x 131072 tokens 130 us, none 125, 2: 122)
#define LT_PART 16384                   // bytes of 128 channels of a tile
#define LT_RAISE 8.f                    // a row's reference is raised when a score is 2^8 above it: weights stay below 2^8, and O seldom has to be multiplied

// Barriers, 8 bytes each.  IN and OUT: of a stage's two parts.  A part is filled again while the other is still used, and scores begin with the first.
// (While the tensor cores read their operands, an access to shared memory takes some 240 cycles, a barrier's that has long been there too, so
// that more parts cost more than they bring, and barriers are asked before the answer is needed.)
enum { LT_A_IN = 0, LT_A_OUT = 2 * LT_A_STAGES, LT_A_S = 2 * LT_A_OUT, LT_A_P = LT_A_S + 2, LT_A_O, LT_A_Q, LT_A_END, LT_A_BARS };
struct LtAttend {
    KvRows q, q_rope, out;
    float* lse;
    const int32_t* parents;             // NULL: a chain
    int groups;                         // of CTAs: runs that the line is cut into
    int group_tiles;                    // row tiles, CTAs, of a group
    int seq_groups;                     // groups of row tiles of a sequence, at most
    int least;                          // tiles of a run, at least (2: 700 tokens in 13.7 us, as with 1; 3: 16)
    float* part_o;                      // [groups][2][group_tiles][64][latent]: the first piece of a run (begun before it), the last
    float* part_ml;                     // [groups][2][group_tiles][64][2]
    int* cuts;                          // [groups][4]: of a run whose last item goes on: first packed row of the sequence, the item's first row, pieces, rows of the sequence
};

// Tiles of tokens that an item (a sequence's group of row tiles) takes; one at least if there are rows.  (Rows of a sequence: at most 2^30.)
__device__ __forceinline__ int lt_item_tiles(const LtShape& S, const LtAttend& A, const LtSeq& q, int group)
{
    const int rows_of = A.group_tiles * LT_ROWS, first = group * rows_of, rows = q.n * S.heads;
    if (first >= rows) return 0;
    const int last = (int)((uint32_t)(min(first + rows_of, rows) - 1) / (uint32_t)S.heads);
    const int end = A.parents ? q.len : q.len - q.n + last + 1;
    return max((end + LT_TOKENS - 1) / LT_TOKENS, 1);
}

// A walk along a run.  Every warp makes its own; whoever looked for the run's first item has left it in `q` and `tiles`.
struct LtWalk {
    int64_t item_at, at, end;           // in the line: where the item begins, where the walk is, where the run ends
    int seq, group, from, to, tiles;    // the piece: tiles from .. to - 1 of the item's
    LtSeq q;
    __device__ __forceinline__ bool next(const LtShape& S, const LtBatch& B, const LtAttend& A)
    {
        while (at < end) {
            if (at == item_at + tiles) {                 // nothing left of this item
                item_at = at;
                if (++group == A.seq_groups) {
                    group = 0;
                    if (++seq >= B.n_seqs) return false;
                    q = lt_seq(B, seq);
                }
                tiles = lt_item_tiles(S, A, q, group);
                continue;
            }
            from = (int)(at - item_at);
            to = (int)min((int64_t)tiles, end - item_at);
            at = item_at + to;
            return true;
        }
        return false;
    }
};

struct LtMisc {
    uint64_t bars[LT_A_BARS];
    float factor[LT_ROWS];              // of rows: O's when the reference is raised, and 1 / l at the end
    int64_t out_at[LT_ROWS];            // of rows: where the answer goes
    uint32_t bad[3][2];                 // tokens of a tile with a score that is not finite, see lt_guard
    uint32_t present[8];                // of the last tiles: which 16 tokens have a page
    int stop, halt[2];                  // halt: what the rows' warps go by, all the same way (they have barriers among themselves)
    uint32_t tmem;
    LtWalk walk;                        // at the run's begin
    float of_half[2][LT_ROWS];          // of rows over half of the tokens: a tile's largest scores, and at the end the sums of weights
    int64_t warp_sum[LT_A_THREADS / 32];
};
static_assert(sizeof(LtMisc) <= 2048, "");

// The tokens before `len`, of 64 from t0 on, whose pages are there
__device__ __forceinline__ uint64_t lt_there(uint32_t present, int t0, int len)
{
    uint64_t m = 0;
#pragma unroll
    for (int g = 0; g < 4; g++) m |= present >> g & 1 ? 0xffffull << (16 * g) : 0ull;
    const int left = len - t0;
    return left >= 64 ? m : left <= 0 ? 0ull : m & ((1ull << left) - 1);
}
// Of 64 tokens from t0 on, those that new token j of a sequence sees
__device__ __forceinline__ uint64_t lt_sees(const LtAttend& A, const LtSeq& q, int j, int t0)
{
    const int base = q.len - q.n;                        // the first new token's place
    const int upto = (A.parents ? base : base + j + 1) - t0;
    uint64_t m = upto >= 64 ? ~0ull : upto <= 0 ? 0ull : (1ull << upto) - 1;
    if (A.parents && t0 + 64 > base) {
        for (int a = j;;) {                              // a parent is less than its child, so this ends
            const int bit = base + a - t0;
            if (bit >= 0 && bit < 64) m |= 1ull << bit;
            const int p = A.parents[q.start + a];
            if (p < 0 || p >= a) break;
            a = p;
        }
    }
    return m;
}

// Warps 0-7: the weights of the rows, and their answers.  Warps w and w + 4 have the same 16 rows, 32 tokens of a tile each.
#define LT_A_ROW_THREADS 256
template <int PAIRS, bool BF>
__device__ __forceinline__ void lt_attend_rows(const LtShape& S, const LtBatch& B, const LtAttend& A, LtWalk walk, int64_t share, uint8_t* sm, uint32_t sm_at, LtMisc& M,
                                               uint32_t bars, uint32_t tmem)
{
    using T = LtTile<PAIRS>;
    constexpr int chunks = 2 * PAIRS, latent = 128 * PAIRS;
    const int warp = threadIdx.x >> 5 & 3, half = threadIdx.x >> 7, lane = threadIdx.x & 31, quad = lane & 3;
    const int g = blockIdx.x / A.group_tiles, r = blockIdx.x % A.group_tiles;
    uint8_t* const p_sm = sm + T::P;
    volatile int* const stop = &M.stop;
    const uint32_t lanes = (uint32_t)warp << 21, s_at = tmem + lanes + 256 + 32 * half, o_at = tmem + lanes;
    const float scale = S.scale_log2;
    const uint32_t heads = S.heads;
    bool fine = true, halted = false;                    // fine: of this warp; where it is not, answers are NaN
    int c = 0;                                           // tiles so far
    if (r == 0 && threadIdx.x == 0) A.cuts[4 * g + 2] = 0;
    while (!halted && walk.next(S, B, A)) {
        const LtSeq& q = walk.q;
        const int first = (walk.group * A.group_tiles + r) * LT_ROWS, rows = min(LT_ROWS, q.n * (int)heads - first);
        const bool whole = walk.from == 0 && walk.to == walk.tiles;
        if (r == 0 && threadIdx.x == 0 && walk.from == 0 && !whole) {
            A.cuts[4 * g] = q.start;
            A.cuts[4 * g + 1] = first;
            A.cuts[4 * g + 2] = (int)((walk.item_at + walk.tiles - 1) / share) - g + 1;
            A.cuts[4 * g + 3] = q.n * (int)heads;
        }
        if (rows <= 0) continue;
        {
            // Q: 8 threads take a row's chunk
            const int piece = threadIdx.x & 7;
#pragma unroll
            for (int k2 = 0; k2 < LT_ROWS * 8 / LT_A_ROW_THREADS; k2++) {
                const int row = (threadIdx.x >> 3) + LT_A_ROW_THREADS / 8 * k2;
                const bool there = row < rows;
                const uint32_t at = there ? first + row : 0, j = at / heads, head = at - j * heads;
                const int64_t token = q.start + (int64_t)j;
                const uint16_t* src = (const uint16_t*)A.q.data + token * A.q.token_stride + head * A.q.head_stride + 8 * piece;
                const uint16_t* key = (const uint16_t*)A.q_rope.data + token * A.q_rope.token_stride + head * A.q_rope.head_stride + 8 * piece;
#pragma unroll
                for (int k = 0; k < chunks; k++) lt_copy16(sm_at + k * LT_ROWS * LT_CHUNK_ROW + lt_at(row, piece), src + 64 * k, there);
                if (8 * piece < S.rope) lt_copy16(sm_at + chunks * LT_ROWS * LT_CHUNK_ROW + lt_at(row, piece), key, there);
                if (piece == 0) M.out_at[row] = token * A.out.token_stride + head * A.out.head_stride;
            }
            lt_copies_done();
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            kv_warp_arrive(bars + 8 * LT_A_Q);
        }
        const bool active = 16 * warp < rows;
        // rows of this lane: 16 warp + lane / 4 and 8 further on
        const int my_row = 16 * warp + (lane >> 2);
        int j[2];
#pragma unroll
        for (int h = 0; h < 2; h++) j[h] = my_row + 8 * h < rows ? (int)((uint32_t)(first + my_row + 8 * h) / heads) : -1;
        const int see_all = A.parents ? q.len - q.n : q.len - q.n + (int)((uint32_t)first / heads) + 1;
        float m[2] = {KV_M_NONE, KV_M_NONE}, l[2] = {0.f, 0.f};
        for (int i = walk.from; i < walk.to && !halted; i++, c++) {
            const int t0 = i * LT_TOKENS, set = c % 3;
            // what is known of the tile first, while its scores are made
            fine = kv_warp_wait(bars + 8 * (LT_A_IN + 2 * (c % T::STAGES) + 1), c / T::STAGES & 1, stop) && fine;
            const uint32_t present = ((volatile uint32_t*)M.present)[c & 7];
            fine = kv_warp_wait(bars + 8 * (LT_A_S + (c & 1)), c >> 1 & 1, stop) && fine;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            uint32_t x[16];
            const bool ragged = t0 + LT_TOKENS > see_all || present != 15u;
            float top[2] = {-KV_INF, -KV_INF};
            if (active) {
                lt_tmem_load_quads(x, s_at + 64 * (c & 1));
                if (ragged) {
                    const uint64_t there = lt_there(present, t0, q.len);
                    uint32_t bad = 0, sees[2];
#pragma unroll
                    for (int h = 0; h < 2; h++) sees[h] = j[h] < 0 ? 0u : (uint32_t)((lt_sees(A, q, j[h], t0) & there) >> (32 * half)) >> (2 * quad);
#pragma unroll
                    for (int k = 0; k < 16; k++) {
                        const int bit = 8 * (k >> 2) + (k & 1);              // and 2 quad on
                        if (!(fabsf(__uint_as_float(x[k])) < KV_INF)) bad |= 1u << bit;
                        x[k] = sees[k >> 1 & 1] >> bit & 1 ? x[k] : 0xff800000u;
                    }
                    bad = __reduce_or_sync(0xffffffffu, bad << (2 * quad));
                    if (lane == 0 && bad) atomicOr(&M.bad[set][half], bad);
                }
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    top[0] = fmaxf(top[0], fmaxf(__uint_as_float(x[4 * k]), __uint_as_float(x[4 * k + 1])));
                    top[1] = fmaxf(top[1], fmaxf(__uint_as_float(x[4 * k + 2]), __uint_as_float(x[4 * k + 3])));
                }
            }
            // the set after next's: what it held two tiles ago has been read by all, who have come to the barrier of the tile before this one since
            if (threadIdx.x == 0) {
                M.bad[(set + 1) % 3][0] = M.bad[(set + 1) % 3][1] = 0;
                M.halt[c & 1] = *stop;
            }
            const bool raise = lt_any(1, LT_A_ROW_THREADS, top[0] * scale > m[0] + LT_RAISE || top[1] * scale > m[1] + LT_RAISE);
            halted = ((volatile int*)M.halt)[c & 1];
            const uint32_t p_free = kv_ended(bars + 8 * LT_A_O, c + 1 & 1);  // asked early, needed late
            if (raise) {
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 1));
                    top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 2)) * scale;
                    if (quad == 0) M.of_half[half][my_row + 8 * h] = top[h];
                }
                lt_sync(2, LT_A_ROW_THREADS);
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const float to = fmaxf(fmaxf(m[h], top[h]), M.of_half[half ^ 1][my_row + 8 * h]), fall = kv_exp2(m[h] - to);
                    l[h] *= fall;
                    m[h] = to;
                    if (quad == 0 && half == 0) M.factor[my_row + 8 * h] = fall;
                }
            }
            if (active) {
#pragma unroll
                for (int k = 0; k < 4; k++)
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        const float a = kv_exp2(fmaf(__uint_as_float(x[4 * k + 2 * h]), scale, -m[h])), b = kv_exp2(fmaf(__uint_as_float(x[4 * k + 2 * h + 1]), scale, -m[h]));
                        l[h] += a + b;
                        x[2 * k + h] = kv_pack<BF>(a, b);
                    }
            }
            // the product before is done: P is free, and O rests
            if (c > 0 && !__all_sync(0xffffffffu, p_free)) fine = kv_warp_wait(bars + 8 * LT_A_O, c + 1 & 1, stop) && fine;
            if (active) {
#pragma unroll
                for (int k = 0; k < 4; k++)
#pragma unroll
                    for (int h = 0; h < 2; h++) *(uint32_t*)(p_sm + lt_at(my_row + 8 * h, 4 * half + k) + 4 * quad) = x[2 * k + h];
            }
            if (raise && i > walk.from) {
                lt_sync(2, LT_A_ROW_THREADS);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (int b = half; b < PAIRS; b += 2)
#pragma unroll 1
                    for (int n = 0; n < rows; n += 32) {
                        uint32_t y[32];
                        kv_tmem_load32(y, o_at + 64 * b + n);
#pragma unroll
                        for (int k = 0; k < 32; k++) y[k] = __float_as_uint(__uint_as_float(y[k]) * M.factor[n + k]);
                        kv_tmem_store32(y, o_at + 64 * b + n);
                    }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            }
            if (ragged) {
                // Tokens that are not there become zeros, and so does what is not finite in tokens that some rows do not see: a weight of 0
                // times it would not be 0.  Such a token shows by its scores, of which every one is not finite: its values all enter them.
                uint8_t* const tile = sm + (1 + c % T::STAGES) * T::BYTES;
                const uint64_t there = lt_there(present, t0, q.len);
                const uint64_t some = see_all - t0 >= 64 ? 0ull : see_all <= t0 ? ~0ull : ~((1ull << (see_all - t0)) - 1);
                uint64_t todo = ~there | (some & ((uint64_t)((volatile uint32_t*)M.bad[set])[1] << 32 | ((volatile uint32_t*)M.bad[set])[0]));
                for (int n = threadIdx.x & 63, turn = threadIdx.x >> 6; todo; todo &= todo - 1, turn--) {
                    const int t = __ffsll((long long)todo) - 1;
                    if (turn & 3 || n >= 8 * chunks) continue;               // 64 threads take every fourth token
                    uint4* const at = (uint4*)(tile + (n >> 3) * LT_TOKENS * LT_CHUNK_ROW + lt_at(t, n & 7));
                    uint4 w = make_uint4(0, 0, 0, 0);
                    if (there >> t & 1) {
                        w = *at;
                        w = make_uint4(lt_finite2<BF>(w.x), lt_finite2<BF>(w.y), lt_finite2<BF>(w.z), lt_finite2<BF>(w.w));
                    }
                    *at = w;
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            kv_warp_arrive(bars + 8 * LT_A_P);
        }
        // the piece's end: the halves' sums
        const int64_t slot = ((int64_t)2 * g + (walk.from == 0)) * A.group_tiles + r;
        lt_sync(2, LT_A_ROW_THREADS);                    // the last tile's largest scores have been read
#pragma unroll
        for (int h = 0; h < 2; h++) {
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
            if (quad == 0) M.of_half[half][my_row + 8 * h] = l[h];
        }
        fine = kv_warp_wait(bars + 8 * LT_A_O, c - 1 & 1, stop) && fine && !*stop;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        lt_sync(2, LT_A_ROW_THREADS);
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int row = my_row + 8 * h;
            l[h] += M.of_half[half ^ 1][row];
            if (!fine) l[h] = __int_as_float(0x7fffffff);
            if (quad == 0 && half == 0) {
                M.factor[row] = l[h] == 0.f ? 0.f : 1.f / l[h];
                if (row < rows) {
                    if (!whole) *(float2*)(A.part_ml + 2 * (slot * LT_ROWS + row)) = make_float2(m[h], l[h]);
                    else if (A.lse) A.lse[(q.start + (int64_t)j[h]) * S.heads + ((uint32_t)(first + row) - j[h] * heads)] = l[h] == 0.f ? -KV_INF : (m[h] + log2f(l[h])) * 0.6931471805599453f;
                }
            }
        }
        lt_sync(2, LT_A_ROW_THREADS);
        for (int b = half; b < PAIRS; b += 2) {
            const int ch = 128 * b + 32 * warp + lane;
#pragma unroll 1
            for (int n = 0; n < rows; n += 32) {
                uint32_t y[32];
                kv_tmem_load32(y, o_at + 64 * b + n);
                if (whole) {
                    const bool odd = lane & 1;
#pragma unroll
                    for (int k = 0; k < 32; k += 2) {
                        // two lanes, two rows: each lane gets a pair of channels of one row
                        const float u = __uint_as_float(y[k]) * M.factor[n + k], w = __uint_as_float(y[k + 1]) * M.factor[n + k + 1];
                        const float got = __shfl_xor_sync(0xffffffffu, odd ? u : w, 1);
                        const int row = n + k + odd;
                        if (row < rows) *(uint32_t*)((uint16_t*)A.out.data + M.out_at[row] + (ch & ~1)) = odd ? kv_pack<BF>(got, w) : kv_pack<BF>(u, got);
                    }
                } else {
                    float* const to = A.part_o + (slot * LT_ROWS + n) * latent + ch;
#pragma unroll
                    for (int k = 0; k < 32; k++)
                        if (n + k < rows) to[k * latent] = __uint_as_float(y[k]);
                }
            }
        }
        lt_sync(2, LT_A_ROW_THREADS);                    // factor, of_half and out_at have been read
    }
}

// Warp 8: the tiles.  It and warp 9 are one chain of instructions each, of which every one counts: no divisions, addresses known early.
// A copy takes some 120 cycles to issue.  Blocks of less than 64 tokens need one for every block and 64 channels; these warps 8, 10 and 11 share
// (`turn` 0, 1, 2), and each arrives for its own.
template <int PAIRS>
__device__ __forceinline__ void lt_attend_bring(const LtShape& S, const LtBatch& B, const LtAttend& A, const CUtensorMap* map, const CUtensorMap* pairs_map, LtWalk walk, int turn,
                                                uint32_t sm_at, LtMisc& M, uint32_t bars)
{
    using T = LtTile<PAIRS>;
    const int lane = threadIdx.x & 31, r = blockIdx.x % A.group_tiles;
    const int box_shift = min(S.block_shift, 6), box = 1 << box_shift;
    const uint32_t box_bits = (1u << (box / 16)) - 1;
    volatile int* const stop = &M.stop;
    bool fine = true;
    int c = 0;                                           // tiles so far
    while (fine && walk.next(S, B, A)) {
        if ((walk.group * A.group_tiles + r) * LT_ROWS >= walk.q.n * S.heads) continue;
        int known = -1, pages = -1;                      // lane: page of the block known + lane
        for (int i = walk.from; i < walk.to && fine; i++) {
            const uint32_t stage = c % T::STAGES, in = bars + 8 * (LT_A_IN + 2 * stage), out = bars + 8 * (LT_A_OUT + 2 * stage), phase = c / T::STAGES & 1, to = sm_at + (1 + stage) * T::BYTES;
            const int block = i * LT_TOKENS >> S.block_shift, y = i * LT_TOKENS & (S.block_tokens - 1);
            if (known < 0 || block + 4 + (LT_A_AHEAD * LT_TOKENS >> S.block_shift) > known + 32) {
                known = block;
                pages = (int64_t)(block + lane) << S.block_shift < walk.q.len ? lt_page(B, walk.seq, block + lane) : -1;
            }
            uint32_t present = 0;
            int page[4];
            if (box_shift == 6) {
                page[0] = lt_uniform(pages, block - known);
                present = page[0] >= 0 ? 15u : 0u;
            } else {
#pragma unroll
                for (int b = 0; b < 4; b++) {
                    page[b] = b << box_shift < LT_TOKENS ? lt_uniform(pages, block + b - known) : -1;
                    if (page[b] >= 0) present |= box_bits << (b << box_shift >> 4);
                }
            }
            const uint32_t bytes = __popc(present) * 16 * LT_CHUNK_ROW;
            // chunks from .. upto - 1 of the tile's small blocks that are this warp's, and their bytes
            auto small = [&](int from, int upto, uint32_t bar) {
                lt_expect(bar, bytes * ((upto - from + LT_A_BRINGERS - 1 - turn) / LT_A_BRINGERS));
                for (int k = from + turn; k < upto; k += LT_A_BRINGERS)
#pragma unroll
                    for (int b = 0; b < 4; b++)
                        if (page[b] >= 0) lt_tma(to + (k * LT_TOKENS + (b << box_shift)) * LT_CHUNK_ROW, map, 64 * k, 0, page[b], bar);
            };
            fine = kv_warp_wait(out, phase ^ 1, stop);
            if (!fine) break;
            const uint32_t second_out = kv_ended(out + 8, phase ^ 1);
            if (box_shift == 6) {
                lt_expect(in, bytes * 2 * T::FIRST);
                if (present)
#pragma unroll
                    for (int p = 0; p < T::FIRST; p++) lt_tma(to + p * LT_PART, pairs_map, 0, y, 2 * p, page[0], in);
            } else {
                small(0, 2 * T::FIRST, in);
            }
            if (!__all_sync(0xffffffffu, second_out)) fine = kv_warp_wait(out + 8, phase ^ 1, stop);
            if (!fine) break;
            if (lane == 0 && turn == 0) ((volatile uint32_t*)M.present)[c & 7] = present;
            __syncwarp();
            if (box_shift == 6) {
                lt_expect(in + 8, bytes * (T::CHUNKS - 2 * T::FIRST));
                if (present) {
#pragma unroll
                    for (int p = T::FIRST; p < PAIRS; p++) lt_tma(to + p * LT_PART, pairs_map, 0, y, 2 * p, page[0], in + 8);
                    lt_tma(to + PAIRS * LT_PART, map, 128 * PAIRS, y, page[0], in + 8);
                }
            } else {
                small(2 * T::FIRST, T::CHUNKS, in + 8);
            }
            // Two stages do not hold what has to be on its way from memory: tiles further on are brought to L2.
            if (const int j = i + LT_A_AHEAD; turn == 0 && i > walk.from && j < walk.to)
#pragma unroll 1
                for (int b = 0; b << box_shift < LT_TOKENS; b++) {
                    const int far = lt_uniform(pages, ((j * LT_TOKENS + (b << box_shift)) >> S.block_shift) - known);
                    if (far >= 0)
                        lt_prefetch(B.pool + ((int64_t)far * S.block_tokens + (j * LT_TOKENS + (b << box_shift) & (S.block_tokens - 1))) * S.row, (uint32_t)(2 * S.row) << box_shift);
                }
            c++;
        }
    }
    // what is on its way arrives before the CTA ends
    for (int back = fine ? 1 : 0; back <= T::STAGES && back <= c; back++) {
        const int tile = c - back;
        // of a tile that was not finished, parts may have been asked for; if not, the wait runs out, bounded
        for (int part = 0; part < 2; part++) (void)kv_wait(bars + 8 * (LT_A_IN + 2 * (tile % T::STAGES) + part), tile / T::STAGES & 1);
    }
}

// Warp 9: the products
template <int PAIRS, bool BF>
__device__ __forceinline__ void lt_attend_products(const LtShape& S, const LtBatch& B, const LtAttend& A, LtWalk walk, uint32_t sm_at, LtMisc& M, uint32_t bars, uint32_t tmem)
{
    using T = LtTile<PAIRS>;
    const int r = blockIdx.x % A.group_tiles;
    constexpr uint32_t kind = 1u << 4 | (BF ? 1u << 7 | 1u << 10 : 0u);                      // f32 += bf16 * bf16 or f16 * f16
    constexpr uint32_t s_what = kind | (LT_ROWS / 16) << 24 | (LT_TOKENS / 8) << 17;
    constexpr uint32_t CHUNK = 64 * LT_CHUNK_ROW >> 4;   // in descriptors
    volatile int* const stop = &M.stop;
    const uint64_t q_desc = kv_desc(sm_at, 16, 1024), k_desc = kv_desc(sm_at + T::BYTES, 16, 1024), v_desc = kv_desc(sm_at + T::BYTES, LT_TOKENS * LT_CHUNK_ROW, 1024),
                   p_desc = kv_desc(sm_at + T::P, 16, 1024);
    bool fine = true;
    auto scores = [&](int c, bool there) {               // there: the first part is known to be
        const uint32_t stage = c % T::STAGES, s_at = tmem + 256 + 64 * (c & 1);
        const uint64_t k = k_desc + stage * (T::BYTES >> 4);
        const uint32_t in = bars + 8 * (LT_A_IN + 2 * stage), phase = c / T::STAGES & 1;
        if (!there) fine = kv_warp_wait(in, phase, stop);
        if (!fine) return;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t second = kv_ended(in + 8, phase);
#pragma unroll
        for (int n = 0; n < 2 * T::FIRST; n++) lt_mma_ss<4, 2, 2>(s_at, q_desc + n * CHUNK, k + n * CHUNK, s_what, n > 0);
        if (!__all_sync(0xffffffffu, second)) fine = kv_warp_wait(in + 8, phase, stop);
        if (!fine) return;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
        for (int n = 2 * T::FIRST; n < 2 * PAIRS; n++) lt_mma_ss<4, 2, 2>(s_at, q_desc + n * CHUNK, k + n * CHUNK, s_what, n > 0);
        lt_mma_ss<2, 2, 2>(s_at, q_desc + 2 * PAIRS * CHUNK, k + 2 * PAIRS * CHUNK, s_what, true);
        if (S.rope == 64) lt_mma_ss<2, 2, 2>(s_at, q_desc + 2 * PAIRS * CHUNK + 4, k + 2 * PAIRS * CHUNK + 4, s_what, true);
        kv_commit(bars + 8 * (LT_A_S + (c & 1)));
    };
    int c = 0, piece = 0;
    while (fine && walk.next(S, B, A)) {
        const int left = walk.q.n * S.heads - (walk.group * A.group_tiles + r) * LT_ROWS;
        if (left <= 0) continue;
        const uint32_t n = (uint32_t)(min(left, LT_ROWS) + 15) / 16 * 16;
        const uint32_t o_what = kind | 8u << 24 | n / 8 << 17 | 1u << 15;                    // A's M runs along the row
        fine = kv_warp_wait(bars + 8 * LT_A_Q, piece & 1, stop);
        if (fine) scores(c, false);
        for (int i = walk.from; i < walk.to && fine; i++, c++) {
            // The next tile's scores first, if it is there before this one's weights are: where memory is the bound it is not, and this one's
            // answers must not wait for it (they free the place that the tile after it comes to).
            bool next = i + 1 < walk.to, made = false;
            const uint32_t next_in = bars + 8 * (LT_A_IN + 2 * ((c + 1) % T::STAGES));
            for (int turn = 0; next && fine && turn < 1 << 18; turn++) {
                const uint32_t data = kv_ended(next_in, (c + 1) / T::STAGES & 1), weights = kv_ended(bars + 8 * LT_A_P, c & 1), end = *stop;
                made = __all_sync(0xffffffffu, weights);
                if (made || __any_sync(0xffffffffu, end)) break;
                if (__all_sync(0xffffffffu, data)) {
                    scores(c + 1, true);
                    next = false;
                }
            }
            if (fine && !made) fine = kv_warp_wait(bars + 8 * LT_A_P, c & 1, stop);
            if (!fine) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t stage = c % T::STAGES;
            const uint64_t v = v_desc + stage * (T::BYTES >> 4);
            const bool add = i > walk.from;
#pragma unroll
            for (int p = 0; p < PAIRS; p++) {
                lt_mma_ss<4, 2048 / 16, 2>(tmem + 64 * p, v + p * (LT_PART >> 4), p_desc, o_what, add);
                if (p + 1 == T::FIRST && PAIRS > 1) kv_commit(bars + 8 * (LT_A_OUT + 2 * stage));
            }
            if (PAIRS == 1) kv_commit(bars + 8 * (LT_A_OUT + 2 * stage));
            kv_commit(bars + 8 * (LT_A_OUT + 2 * stage + 1));
            kv_commit(bars + 8 * LT_A_O);
            if (next) scores(c + 1, false);
        }
        piece++;
    }
}

template <int PAIRS, bool BF>
__global__ void __launch_bounds__(LT_A_THREADS, 1) lt_attend_kernel(const LtShape S, const LtBatch B, const LtAttend A, const __grid_constant__ CUtensorMap map,
                                                                    const __grid_constant__ CUtensorMap pairs_map)
{
    extern __shared__ uint8_t lt_raw[];
    uint8_t* const sm = lt_raw + (-(uint32_t)__cvta_generic_to_shared(lt_raw) & 1023u);
    const uint32_t sm_at = (uint32_t)__cvta_generic_to_shared(sm);
    const int warp = threadIdx.x >> 5;
    LtMisc& M = *(LtMisc*)(sm + LtTile<PAIRS>::MISC);
    const uint32_t bars = (uint32_t)__cvta_generic_to_shared(M.bars);
    asm volatile("griddepcontrol.launch_dependents;");
    if (threadIdx.x == 0) {
        for (int i = 0; i < LT_A_BARS; i++) lt_init(bars + 8 * i, i == LT_A_P || i == LT_A_Q ? LT_A_ROW_THREADS / 32 : i < LT_A_OUT && S.block_tokens < LT_TOKENS ? LT_A_BRINGERS : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        M.stop = 0;
        for (int i = 0; i < 3; i++) M.bad[i][0] = M.bad[i][1] = 0;
    }
    if (warp == 9) asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"((uint32_t)__cvta_generic_to_shared(&M.tmem)) : "memory");

    asm volatile("griddepcontrol.wait;" ::: "memory");
    // the line's length, and where this run begins
    // (the last item that a thread has looked at is remembered: with no more items than threads, whoever has the first one need not read again)
    LtWalk w;
    int64_t known = -1;
    auto tiles_of = [&](int64_t item) {
        if (item != known) {
            w.seq = A.seq_groups == 1 ? (int)item : (int)(item / A.seq_groups);
            w.group = (int)(item - (int64_t)w.seq * A.seq_groups);
            w.q = lt_seq(B, w.seq);
            w.tiles = lt_item_tiles(S, A, w.q, w.group);
            known = item;
        }
        return w.tiles;
    };
    LtStretch mine = lt_stretch<LT_A_THREADS>((int64_t)B.n_seqs * A.seq_groups, tiles_of, M.warp_sum);
    const int64_t share = max((mine.total + A.groups - 1) / A.groups, (int64_t)A.least);
    const int64_t begin = blockIdx.x / A.group_tiles * share;
    if (mine.holds(begin)) {
        mine.find(begin, tiles_of);                      // which leaves the item in w
        w.item_at = mine.before;
        w.at = begin;
        w.end = min(begin + share, mine.total);
        M.walk = w;
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    LtWalk walk = M.walk;
    if (begin >= mine.total) walk.at = walk.end = 0;     // nothing to do
    const uint32_t tmem = *(volatile uint32_t*)&M.tmem;  // O: 64 columns per 128 channels; S: 2 x 64 from 256 on
    if (warp < 8) {
        lt_attend_rows<PAIRS, BF>(S, B, A, walk, share, sm, sm_at, M, bars, tmem);
    } else if (warp != 9) {
        if (warp == 8 || S.block_tokens < LT_TOKENS) lt_attend_bring<PAIRS>(S, B, A, &map, &pairs_map, walk, warp == 8 ? 0 : warp - 9, sm_at, M, bars);
    } else {
        lt_attend_products<PAIRS, BF>(S, B, A, walk, sm_at, M, bars, tmem);
        __syncwarp();
        kv_commit(bars + 8 * LT_A_END);                  // nothing is on its way any more when the memory is given back
        kv_wait(bars + 8 * LT_A_END, 0);
        __syncwarp();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 9) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

// Joins the pieces of items that runs cut.  A warp takes 128 channels of a row, 4 channels a lane, and asks for some pieces at a time; the pieces'
// references and sums it has in its lanes, 32 at a time.
#define LT_JOIN_THREADS 128
#define LT_JOIN_PIECES 4                // asked for at a time: most items are cut into two or three, and fewer registers leave more warps
#define LT_JOIN_CUTS 512                // most groups of CTAs
template <bool BF> __global__ void __launch_bounds__(LT_JOIN_THREADS) lt_join_kernel(const LtShape S, const LtBatch B, const LtAttend A)
{
    __shared__ int4 cuts[LT_JOIN_CUTS];
    __shared__ int cut_runs[LT_JOIN_CUTS], cut_count;
    const int lane = threadIdx.x & 31, pairs = S.latent / 128, rows_of = A.group_tiles * LT_ROWS;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (threadIdx.x < 32) {
        // the runs whose last item goes on, in order: every CTA has the same list
        int n = 0;
        for (int g0 = 0; g0 < A.groups; g0 += 5 * 32) {
            int4 cut[5];
#pragma unroll
            for (int k = 0; k < 5; k++) cut[k] = g0 + 32 * k + lane < A.groups ? *(const int4*)(A.cuts + 4 * (g0 + 32 * k + lane)) : make_int4(0, 0, 0, 0);
#pragma unroll
            for (int k = 0; k < 5; k++) {
                const uint32_t some = __ballot_sync(0xffffffffu, cut[k].z > 1);
                if (cut[k].z > 1) {
                    cut_runs[n + __popc(some & ((1u << lane) - 1))] = g0 + 32 * k + lane;
                    cuts[n + __popc(some & ((1u << lane) - 1))] = cut[k];
                }
                n += __popc(some);
            }
        }
        if (lane == 0) cut_count = n;
    }
    __syncthreads();
    const int of_cut = rows_of * pairs, work = cut_count * of_cut, step = gridDim.x * (LT_JOIN_THREADS / 32);
    for (int w = blockIdx.x * (LT_JOIN_THREADS / 32) + (threadIdx.x >> 5); w < work; w += step) {
        const int nth = w / of_cut, g = cut_runs[nth], at = w % of_cut, i = at / pairs, ch = at % pairs * 128 + 4 * lane;
        const int4 cut = cuts[nth];
        const int row = cut.y + i;
        const int64_t first_slot = (((int64_t)2 * g + 1) * A.group_tiles + i / LT_ROWS) * LT_ROWS + i % LT_ROWS, next_slot = first_slot + A.group_tiles * LT_ROWS,
                      slot_step = (int64_t)2 * A.group_tiles * LT_ROWS;      // pieces: the last of this run, the first of the next runs
        auto slot = [&](int s) { return s == 0 ? first_slot : next_slot + (s - 1) * slot_step; };
        if (row >= cut.w) continue;
        float m = KV_M_NONE, l = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s0 = 0; s0 < cut.z; s0 += 32) {
            const float2 ml = s0 + lane < cut.z ? *(const float2*)(A.part_ml + 2 * slot(s0 + lane)) : make_float2(KV_M_NONE, 0.f);
            float weight = 0.f;
            for (int s = 0; s < 32 && s0 + s < cut.z; s += LT_JOIN_PIECES) {
                float4 o[LT_JOIN_PIECES];
#pragma unroll
                for (int k = 0; k < LT_JOIN_PIECES; k++) o[k] = s0 + s + k < cut.z ? *(const float4*)(A.part_o + slot(s0 + s + k) * S.latent + ch) : make_float4(0.f, 0.f, 0.f, 0.f);
                if (s == 0) {
                    float top = ml.x;
#pragma unroll
                    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                    top = fmaxf(top, m);
                    const float fall = kv_exp2(m - top);
                    m = top;
                    weight = kv_exp2(ml.x - top);
                    float part = ml.y * weight;
#pragma unroll
                    for (int d = 16; d; d >>= 1) part += __shfl_xor_sync(0xffffffffu, part, d);
                    l = l * fall + part;
                    sum = make_float4(sum.x * fall, sum.y * fall, sum.z * fall, sum.w * fall);
                }
#pragma unroll
                for (int k = 0; k < LT_JOIN_PIECES; k++) {
                    const float by = __shfl_sync(0xffffffffu, weight, s + k);
                    if (s0 + s + k < cut.z) sum = make_float4(fmaf(by, o[k].x, sum.x), fmaf(by, o[k].y, sum.y), fmaf(by, o[k].z, sum.z), fmaf(by, o[k].w, sum.w));
                }
            }
        }
        const float by = l == 0.f ? 0.f : 1.f / l;
        const int j = (int)((uint32_t)row / (uint32_t)S.heads), head = row - j * S.heads;
        const int64_t token = cut.x + (int64_t)j;
        *(uint2*)((uint16_t*)A.out.data + token * A.out.token_stride + head * A.out.head_stride + ch) = make_uint2(kv_pack<BF>(sum.x * by, sum.y * by), kv_pack<BF>(sum.z * by, sum.w * by));
        if (ch == 0 && A.lse) A.lse[token * S.heads + head] = l == 0.f ? -KV_INF : (m + log2f(l)) * 0.6931471805599453f;
    }
}
