// fastrack_latent_expand.cuh -- keys and values of every head from the cached latents: a matrix product whose rows lie in pages.
#pragma once
#include "fastrack_latent_device.cuh"

// 256 tokens of a sequence, 128 for each CTA of a pair, times the weights of one head's keys and values (a unit: 128, 192 or 256 columns).  The
// tokens' latents stay in shared memory for as many units as the pair has of them; the weights come 64 channels at a time, half of the rows to each
// CTA.  All units form one line, which is cut into equal runs, one for each pair.  Warps 0-7 write the answers, 32 columns at a time, while the next
// unit's are made (two accumulators); warp 8 brings, warp 9 of the first CTA issues the products of both.
//
// What bounds it: the products (tensor pipe 75 % active) at the clock that the power leaves.  12 278 tokens of 64 heads, 512 channels, bf16: 192 us in a short
// run (1250 TFLOP/s), 232 in a long one (1030 of the 1416 that a long matrix product makes here).  What it came from: one SM per tile and
// 128 columns at a time 302 us (of shared memory's 128 bytes a cycle a product of 128 rows and 128 columns wants all; one of 256 columns
// shared by two SMs wants half); the answers by 8 instead of 4 warps 288 to 271.
#define LT_E_TOKENS 128
#define LT_E_THREADS 320
#define LT_E_STAGES 8                                    // of weights, at most; what latents of 512 channels leave room for are 5.  (A weight's way in takes some
                                                         // 2500 cycles from the stage's end of use on, a chunk's products 512: with 4 stages, 232 us instead of 200.)
#define LT_E_CHUNK (LT_E_TOKENS * LT_CHUNK_ROW)          // bytes of 64 channels of the tokens, or of up to 128 rows of weights

enum { LT_E_A_IN = 0, LT_E_A_OUT, LT_E_B_IN, LT_E_B_OUT = LT_E_B_IN + LT_E_STAGES, LT_E_D_IN = LT_E_B_OUT + LT_E_STAGES, LT_E_D_OUT = LT_E_D_IN + 2, LT_E_END = LT_E_D_OUT + 2, LT_E_BARS };
struct LtExpandMisc {
    uint64_t bars[LT_E_BARS];
    int stop;
    uint32_t tmem;
    int64_t item, item_at;
    int64_t warp_sum[LT_E_THREADS / 32];
};
#define LT_E_OUT_ROW 64                                  // bytes of 32 columns of a row, on the way out
// latents, weights, 2 KB per writing warp, the rest, room to round the base up
__host__ __device__ static inline int lt_expand_stages(int latent) { return latent == 512 ? 5 : latent == 384 ? 7 : LT_E_STAGES; }
static inline int lt_expand_smem(int latent) { return (latent / 64 + lt_expand_stages(latent)) * LT_E_CHUNK + 8 * 32 * LT_E_OUT_ROW + 2048 + 1024; }
static_assert(sizeof(LtExpandMisc) <= 2048, "");

struct LtExpand { KvRows k, v; const int32_t* key_starts; int total_keys, units; };          // units: of 256 tokens, the heads

// A walk along a run of units; tile: 256 tokens of a sequence
struct LtExpandWalk {
    int seq, tile, len;                 // of the piece: units from .. to - 1
    int from, to;
    int64_t at, end;                    // in the line
    bool fresh;
    __device__ __forceinline__ bool next(const LtBatch& B, const LtExpand& A)
    {
        if (at >= end) return false;
        if (!fresh) tile++;
        fresh = false;
        while (true) {
            if (seq >= B.n_seqs) return false;
            len = lt_len(B, seq);
            if (tile < (len + 2 * LT_E_TOKENS - 1) / (2 * LT_E_TOKENS)) break;
            tile = 0;
            seq++;
        }
        from = (int)(at % A.units);
        to = (int)min((int64_t)A.units, from + end - at);
        at += to - from;
        return true;
    }
};

template <bool BF>
__device__ __forceinline__ void lt_expand_write(const LtShape& S, const LtBatch& B, const LtExpand& A, LtExpandWalk walk, uint8_t* stage, uint32_t bars, volatile int* stop,
                                                uint32_t tmem)
{
    const int warp = threadIdx.x >> 5 & 3, half = threadIdx.x >> 7, lane = threadIdx.x & 31, rank = lt_rank();
    const uint32_t first_bars = lt_of_first(bars);
    uint8_t* const mine = stage + (threadIdx.x >> 5) * 32 * LT_E_OUT_ROW;
    // a piece of 16 bytes of a row: rows in pairs fill 128 bytes, swizzled by the pair
    auto at = [](int row, int piece) { return row * LT_E_OUT_ROW + ((piece ^ (row >> 1 & 3)) << 4); };
    int c = 0;
    bool fine = true;
    while (walk.next(B, A)) {                            // where a wait runs out, the answers from there on are NaN
        const int t0 = (2 * walk.tile + rank) * LT_E_TOKENS + 32 * warp, t = t0 + lane;
        const uint32_t there = __ballot_sync(0xffffffffu, t < walk.len && lt_page(B, walk.seq, t >> S.block_shift) >= 0);
        const int64_t first = (int64_t)A.key_starts[walk.seq] + t0;
        for (int u = walk.from; u < walk.to; u++, c++) {
            fine = fine && lt_pair_wait(bars + 8 * (LT_E_D_IN + (c & 1)), c >> 1 & 1, stop);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            for (int b = 32 * half; b < S.key + S.value; b += 64) {
                const KvRows& dst = b < S.key ? A.k : A.v;
                uint16_t* const to_head = (uint16_t*)dst.data + u * dst.head_stride + (b < S.key ? b : b - S.key) + 8 * (lane & 3);
                uint32_t x[32];
                kv_tmem_load32(x, tmem + ((uint32_t)warp << 21) + 256 * (c & 1) + b);
                if (b + 64 >= S.key + S.value) {         // the accumulator has been read
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    lt_pair_arrive(first_bars + 8 * (LT_E_D_OUT + (c & 1)));
                }
#pragma unroll
                for (int p = 0; p < 4; p++) {
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 8; e++) y[e] = !fine ? __int_as_float(0x7fffffff) : there >> lane & 1 ? __uint_as_float(x[8 * p + e]) : 0.f;
                    *(uint4*)(mine + at(lane, p)) = kv_narrow8<BF>(y);
                }
                __syncwarp();
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const int row = 8 * k + (lane >> 2);
                    const int64_t to = first + row;
                    if (t0 + row < walk.len && to >= 0 && to < A.total_keys) *(uint4*)(to_head + to * dst.token_stride) = *(const uint4*)(mine + at(row, lane & 3));
                }
                __syncwarp();
            }
        }
    }
}

__device__ __forceinline__ void lt_expand_bring(const LtShape& S, const LtBatch& B, const LtExpand& A, const CUtensorMap* pool, const CUtensorMap* weights,
                                                LtExpandWalk walk, uint32_t sm_at, uint32_t bars, volatile int* stop)
{
    const int lane = threadIdx.x & 31, rank = lt_rank(), chunks = S.latent / 64, box = min(S.block_tokens, 64), stages = lt_expand_stages(S.latent);
    const uint32_t weights_at = sm_at + chunks * LT_E_CHUNK, first_bars = lt_of_first(bars);
    int c = 0, pieces = 0, s = 0;                        // chunks of weights, pieces of latents; the next chunk's stage
    uint32_t phase = 0;
    bool fine = true;
    while (fine && walk.next(B, A)) {
        // lane: a box of both CTAs' tokens
        const int t = walk.tile * 2 * LT_E_TOKENS + lane * box;
        const int page = lane * box < 2 * LT_E_TOKENS && t < walk.len ? lt_page(B, walk.seq, t >> S.block_shift) : -1;
        const int boxes = __popc(__ballot_sync(0xffffffffu, page >= 0));
        fine = lt_pair_wait(bars + 8 * LT_E_A_OUT, (pieces & 1) ^ 1, stop);
        if (!fine) break;
        if (rank == 0) lt_expect(bars + 8 * LT_E_A_IN, boxes * box * LT_CHUNK_ROW * chunks);
        for (int b = 0; b < LT_E_TOKENS / box; b++) {
            const int from = lt_uniform(page, rank * (LT_E_TOKENS / box) + b);
            if (from >= 0)
                for (int k = 0; k < chunks; k++)
                    lt_pair_tma(sm_at + k * LT_E_CHUNK + b * box * LT_CHUNK_ROW, pool, 64 * k, ((2 * walk.tile + rank) * LT_E_TOKENS + b * box) & (S.block_tokens - 1), from,
                                first_bars + 8 * LT_E_A_IN);
        }
        pieces++;
        for (int u = walk.from; u < walk.to && fine; u++) {
            for (int k = 0; k < chunks; k++, c++) {
                fine = lt_pair_wait(bars + 8 * (LT_E_B_OUT + s), phase ^ 1, stop);
                if (!fine) break;
                if (rank == 0) lt_expect(bars + 8 * (LT_E_B_IN + s), (S.key + S.value) * LT_CHUNK_ROW);
                lt_pair_tma(weights_at + s * LT_E_CHUNK, weights, 64 * k, rank * ((S.key + S.value) / 2), u, first_bars + 8 * (LT_E_B_IN + s));
                s = s == stages - 1 ? 0 : s + 1;
                phase ^= s == 0;
            }
        }
    }
    // what is on its way, to both CTAs, arrives before they end
    if (rank == 0) {
        for (int back = 1; back <= stages && back <= c; back++) (void)kv_wait(bars + 8 * (LT_E_B_IN + (c - back) % stages), (c - back) / stages & 1);
        if (pieces) (void)kv_wait(bars + 8 * LT_E_A_IN, pieces - 1 & 1);
    }
}

template <bool BF>
__device__ __forceinline__ void lt_expand_products(const LtShape& S, const LtBatch& B, const LtExpand& A, LtExpandWalk walk, uint32_t sm_at, uint32_t bars, volatile int* stop,
                                                   uint32_t tmem)
{
    const int chunks = S.latent / 64, stages = lt_expand_stages(S.latent);
    constexpr uint32_t kind = 1u << 4 | (BF ? 1u << 7 | 1u << 10 : 0u) | (uint32_t)(2 * LT_E_TOKENS / 16) << 24;
    // A barrier's answer takes some 270 cycles while the tensor cores read: it is asked two stages ahead.
    int s = 0, units = 0, pieces = 0;                    // s: the stage
    uint32_t phase = 0, there = 0, next_there = 0;       // there: whether this stage's weights, and the next one's, are known to be
    const uint32_t what = kind | (uint32_t)(S.key + S.value) / 8 << 17;
    const uint64_t a0 = kv_desc(sm_at, 16, 1024), b0 = kv_desc(sm_at + chunks * LT_E_CHUNK, 16, 1024);
    while (walk.next(B, A)) {
        if (!lt_pair_wait(bars + 8 * LT_E_A_IN, pieces++ & 1, stop)) return;
        for (int u = walk.from; u < walk.to; u++, units++) {
            const uint32_t d = tmem + 256 * (units & 1);
            if (!lt_pair_wait(bars + 8 * (LT_E_D_OUT + (units & 1)), (units >> 1 & 1) ^ 1, stop)) return;
#pragma unroll 1
            for (int k = 0; k < chunks; k++) {
                if (!__all_sync(0xffffffffu, there) && !lt_pair_wait(bars + 8 * (LT_E_B_IN + s), phase, stop)) return;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint64_t a = a0 + k * (LT_E_CHUNK >> 4), b = b0 + s * (LT_E_CHUNK >> 4);
                const uint32_t out = bars + 8 * (LT_E_B_OUT + s);
                there = next_there;
                const int ahead = s + 2 < stages ? s + 2 : s + 2 - stages;
                next_there = lt_pair_ended(bars + 8 * (LT_E_B_IN + ahead), phase ^ (s + 2 >= stages));
                lt_pair_mma_ss<4, 2, 2>(d, a, b, what, k > 0);
                lt_pair_commit(out);
                s = s == stages - 1 ? 0 : s + 1;
                phase ^= s == 0;
            }
            lt_pair_commit(bars + 8 * (LT_E_D_IN + (units & 1)));
        }
        lt_pair_commit(bars + 8 * LT_E_A_OUT);
    }
}

template <bool BF>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(LT_E_THREADS, 1) lt_expand_kernel(const LtShape S, const LtBatch B, const LtExpand A, const __grid_constant__ CUtensorMap pool,
                                                                    const __grid_constant__ CUtensorMap weights)
{
    extern __shared__ uint8_t lt_raw[];
    uint8_t* const sm = lt_raw + (-(uint32_t)__cvta_generic_to_shared(lt_raw) & 1023u);
    const uint32_t sm_at = (uint32_t)__cvta_generic_to_shared(sm);
    const int warp = threadIdx.x >> 5;
    uint8_t* const stage = sm + (S.latent / 64 + lt_expand_stages(S.latent)) * LT_E_CHUNK;
    LtExpandMisc& M = *(LtExpandMisc*)(stage + 8 * 32 * LT_E_OUT_ROW);
    const uint32_t bars = (uint32_t)__cvta_generic_to_shared(M.bars);
    volatile int* const stop = &M.stop;
    if (threadIdx.x == 0) {
        for (int i = 0; i < LT_E_BARS; i++) lt_init(bars + 8 * i, i == LT_E_D_OUT || i == LT_E_D_OUT + 1 ? 16 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        M.stop = 0;
    }
    if (warp == 9) asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"((uint32_t)__cvta_generic_to_shared(&M.tmem)) : "memory");
    asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
    auto units_of = [&](int64_t seq) { return (int64_t)((lt_len(B, (int)seq) + 2 * LT_E_TOKENS - 1) / (2 * LT_E_TOKENS)) * A.units; };
    LtStretch mine = lt_stretch<LT_E_THREADS>(B.n_seqs, units_of, M.warp_sum);
    const int pairs = gridDim.x / 2;
    const int64_t share = (mine.total + pairs - 1) / pairs;
    LtExpandWalk walk;
    walk.at = blockIdx.x / 2 * share;
    walk.end = min(walk.at + share, mine.total);
    if (mine.holds(walk.at)) {
        mine.find(walk.at, units_of);
        M.item = mine.item;
        M.item_at = mine.before;
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    kv_cluster_sync();                                   // the other CTA's barriers are there, too
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    walk.seq = walk.at < walk.end ? (int)M.item : 0;
    walk.tile = walk.at < walk.end ? (int)((walk.at - M.item_at) / A.units) : 0;
    walk.fresh = true;
    const uint32_t tmem = *(volatile uint32_t*)&M.tmem;
    if (warp < 8) {
        lt_expand_write<BF>(S, B, A, walk, stage, bars, stop, tmem);
    } else if (warp == 8) {
        lt_expand_bring(S, B, A, &pool, &weights, walk, sm_at, bars, stop);
    } else if (lt_rank() == 0) {
        lt_expand_products<BF>(S, B, A, walk, sm_at, bars, stop, tmem);
        __syncwarp();
        lt_pair_commit(bars + 8 * LT_E_END);             // nothing is on its way any more when the memory is given back
        kv_wait(bars + 8 * LT_E_END, 0);
        __syncwarp();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    kv_cluster_sync();                                   // neither ends while the other's products or arrivals may reach it
    if (warp == 9) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}
