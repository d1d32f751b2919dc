// fastrack_latent_prompt.cuh -- attention of many new tokens over expanded keys and values.
#pragma once
#include <type_traits>
#include "fastrack_latent_device.cuh"

// A pair of CTAs takes 512 queries of one head, two tiles of 256 rows of which each CTA has 128, against 128 tokens at a time:
//     S_m = Q_m K^T  (tensor memory)  ->  P_m = weights as 16 bits (tensor memory, over S_m)  ->  O_m += P_m V.
// Each CTA brings half of K's tokens and half of V's channels; the tensor cores of both read both halves.  (One CTA for 256 queries took 955 us for
// 2 x 8000 tokens of 16 heads: K and V for it alone left no room for a second V, and of shared memory's 128 bytes a cycle a product of
// 128 x 128 wants all.)  Warps 0-3 and 4-7 make P_0 and P_1, a thread per row; warp 8 brings K, the shared keys and V; warp 9 of the first CTA
// issues the products of both, of which one row tile's run while the other's weights are made; warps 10 and 11 look after V where some rows do
// not see some tokens.
//
// Weights are rounded to the values' 16 bits (error against 64 bits bf16 0.0023, f16 0.00026 beside the answer's own rounding's 0.0017 and 0.0002).
// What bounds it, per 128 tokens and pair: the products 2560 cycles, the exponentials 2048; it takes 3800, a row tile's chain: scores seen 350 cycles
// after their end, largest 430, exponentials 1330, weights written and seen 380, products 1280.  3 x 1000 tokens over up to 6100, 32 heads, bf16: 280 us
// (840 TFLOP/s of the visible pairs); 2 x 8000, 16 heads, f16: 740 (890; in a short run 660).  Tried and dropped: weights in two halves with an
// arrival each (no change), two threads a row (655 against 664), 1/8 to 1/2 of the exponentials as polynomials (650 to 758).
#define LT_P_ROWS 128                                    // of a CTA's part of a row tile
#define LT_P_TOKENS 128
#define LT_P_THREADS 384
#define LT_P_STAGES 3
#define LT_P_CHUNK (128 * LT_CHUNK_ROW)                  // bytes of 64 channels of 128 rows: queries, V's tokens
#define LT_P_KEYS (LT_P_CHUNK / 2)                       // of 64 channels of K's 64 tokens
#define LT_P_APART 6                                     // tiles at most, in which some rows see tokens that others do not
#define LT_P_NOTES 8                                     // tiles whose pages are known at a time: more than the stages and what is in work

// K_IN, V_OK, P_IN and Q_IN are the first CTA's, which issues; V_IN and NOTE are each CTA's own; what the products free or finish both are told.
enum { LT_P_K_IN = 0, LT_P_K_OUT = LT_P_K_IN + LT_P_STAGES, LT_P_V_IN = LT_P_K_OUT + LT_P_STAGES, LT_P_V_OK = LT_P_V_IN + LT_P_STAGES, LT_P_V_OUT = LT_P_V_OK + LT_P_STAGES,
       LT_P_S_IN = LT_P_V_OUT + LT_P_STAGES, LT_P_P_IN = LT_P_S_IN + 2, LT_P_NOTE = LT_P_P_IN + 2, LT_P_Q_IN = LT_P_NOTE + LT_P_NOTES, LT_P_END, LT_P_BARS };
struct LtPromptMisc {
    uint64_t bars[LT_P_BARS];
    uint32_t present[LT_P_NOTES];                        // which 16 tokens have a page
    uint32_t apart[LT_P_APART][4];                       // tokens with values in this CTA's half of V that are not finite, from the first tile on that some rows see in part
    uint32_t some_apart;
    int stop;
    uint32_t tmem;
};
struct LtPrompt {
    KvRows q, q_rope, out;
    const uint16_t* v;                                   // values again, for the tokens that are taken apart
    int64_t v_token_stride, v_head_stride;
    float* lse;
    const int32_t* key_starts;
    int total_keys, tiles;                               // tiles: of 512 queries, at most
    bool k_heads, v_heads;                               // whether heads differ
    int splits;                                          // pairs that share a job's tokens between them, equal runs of its steps
    float* part_o;                                       // [splits][total_new][heads][value], if there are several
    float* part_ml;                                      // [splits][total_new][heads][2]
};
__host__ __device__ __forceinline__ int lt_prompt_k_chunks(const LtShape& S) { return S.key / 64 + 1; }
// Q; the stages, of K and then V each; the rest; room to round the base up
static inline int lt_prompt_smem(const LtShape& S) { return 2 * lt_prompt_k_chunks(S) * LT_P_CHUNK + LT_P_STAGES * (lt_prompt_k_chunks(S) * LT_P_KEYS + LT_P_CHUNK) + 1024 + 1024; }
static_assert(sizeof(LtPromptMisc) <= 1024, "");

// What a CTA works on
struct LtPromptJob {
    LtSeq q;
    int seq, head, row, rows, first_step, steps0, steps1;  // row: the pair's first query; rows: that there are; steps: of 128 tokens, for each row tile, from first_step on
    int lo, hi;                                          // tokens whose keys lie in the buffers
    int see_all;                                         // tokens before this one are seen by all rows
    int64_t key_start;
};

// The value's row of a token may hold what is not finite, the token's weight may be 0 for some rows, and 0 times it is not 0: see lt_prompt_guard.
__device__ __forceinline__ bool lt_prompt_ragged(const LtPromptJob& J, int t0, uint32_t present)
{
    return t0 < J.lo || t0 + LT_P_TOKENS > min(J.see_all, J.hi) || present != 0xffu;
}
__device__ __forceinline__ uint32_t lt_bits(int from, int upto)              // bits from .. upto - 1 of 32, of any numbers
{
    const uint32_t below = upto >= 32 ? 0xffffffffu : upto <= 0 ? 0u : (1u << upto) - 1, skip = from >= 32 ? 0xffffffffu : from <= 0 ? 0u : (1u << from) - 1;
    return below & ~skip;
}
// Of 32 tokens from t0 + 32 b on, those that are there
__device__ __forceinline__ uint32_t lt_prompt_there(const LtPromptJob& J, int t0, int b, uint32_t present)
{
    const uint32_t pages = (present >> 2 * b & 1 ? 0xffffu : 0u) | (present >> 2 * b & 2 ? 0xffff0000u : 0u);
    return pages & lt_bits(J.lo - t0 - 32 * b, J.hi - t0 - 32 * b);
}

template <bool BF>
__device__ __forceinline__ void lt_prompt_rows(const LtShape& S, const LtPrompt& A, int total_new, const LtPromptJob& J, int m_tile, uint32_t sm_at, LtPromptMisc& M, uint32_t bars,
                                               uint32_t tmem)
{
    const int warp = threadIdx.x >> 5, r = threadIdx.x & 127, first_row = J.row + LT_P_ROWS * (2 * m_tile + (int)lt_rank()), row = first_row + r,
              steps = m_tile ? J.steps1 : J.steps0;
    const bool valid = row < J.q.n;
    const int place = valid ? J.q.len - J.q.n + row : -1;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21, s_at = tmem + lanes + 128 * m_tile, o_at = tmem + lanes + 256 + 128 * m_tile;
    const int k_chunks = lt_prompt_k_chunks(S);
    volatile int* const stop = &M.stop;
    {
        // Q: 8 threads take a row's chunk
        const uint32_t to = sm_at + m_tile * k_chunks * LT_P_CHUNK;
        const int piece = r & 7;
        for (int i = r >> 3; i < LT_P_ROWS; i += 16) {
            const int at = first_row + i;
            const bool there = at < J.q.n;
            const int64_t token = J.q.start + (there ? at : 0);
            const uint16_t* src = (const uint16_t*)A.q.data + token * A.q.token_stride + J.head * A.q.head_stride;
            const uint16_t* key = (const uint16_t*)A.q_rope.data + token * A.q_rope.token_stride + J.head * A.q_rope.head_stride;
            for (int k = 0; k < k_chunks - 1; k++) lt_copy16(to + k * LT_P_CHUNK + lt_at(i, piece), src + 64 * k + 8 * piece, there);
            if (8 * piece < S.rope) lt_copy16(to + (k_chunks - 1) * LT_P_CHUNK + lt_at(i, piece), key + 8 * piece, there);
        }
        lt_copies_done();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        lt_pair_release(lt_of_first(bars) + 8 * LT_P_Q_IN);
    }
    const int first_place = J.q.len - J.q.n + first_row + 32 * (warp & 3);                   // of this warp's rows
    const uint32_t p_in = lt_of_first(bars) + 8 * (LT_P_P_IN + m_tile);
    const float scale = S.scale_log2;
    float m = KV_M_NONE, l = 0.f;
    bool fine = true;
    for (int s = 0; s < steps && fine; s++) {
        const int t0 = LT_P_TOKENS * (J.first_step + s);
        // what is known of the tile first, while its scores are made
        fine = kv_warp_wait(bars + 8 * (LT_P_NOTE + s % LT_P_NOTES), s / LT_P_NOTES & 1, stop);
        const uint32_t present = ((volatile uint32_t*)M.present)[s % LT_P_NOTES];
        fine = fine && lt_pair_wait(bars + 8 * (LT_P_S_IN + m_tile), s & 1, stop);
        if (!fine) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const bool ragged = t0 < J.lo || t0 + LT_P_TOKENS > min(first_place + 1, J.hi) || present != 0xffu;
        uint32_t x[64], z[64];
        kv_tmem_load64(x, s_at);
        kv_tmem_load64(z, s_at + 64);
        if (ragged) {
#pragma unroll
            for (int b = 0; b < 4; b++) {
                const uint32_t sees = lt_prompt_there(J, t0, b, present) & lt_bits(0, place + 1 - t0 - 32 * b);
#pragma unroll
                for (int i = 0; i < 32; i++) {
                    uint32_t& y = b < 2 ? x[32 * (b & 1) + i] : z[32 * (b & 1) + i];
                    y = sees >> i & 1 ? y : 0xff800000u;
                }
            }
        }
        float top = -KV_INF;
#pragma unroll
        for (int i = 0; i < 64; i += 2) {
            top = fmaxf(fmaxf(top, __uint_as_float(x[i])), __uint_as_float(x[i + 1]));
            top = fmaxf(fmaxf(top, __uint_as_float(z[i])), __uint_as_float(z[i + 1]));
        }
        top *= scale;
        const bool higher = top > m + 8.f;               // weights stay below 2^8, and O seldom has to be multiplied
        const float fall = higher ? kv_exp2(m - top) : 1.f;
        m = higher ? top : m;
        l *= fall;
        uint32_t p[32];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 32; i++) {
            const float a = kv_exp2(fmaf(__uint_as_float(x[2 * i]), scale, -m)), b = kv_exp2(fmaf(__uint_as_float(x[2 * i + 1]), scale, -m));
            sum += a + b;
            p[i] = kv_pack<BF>(a, b);
        }
        kv_tmem_store32(p, s_at);
#pragma unroll
        for (int i = 0; i < 32; i++) {
            const float a = kv_exp2(fmaf(__uint_as_float(z[2 * i]), scale, -m)), b = kv_exp2(fmaf(__uint_as_float(z[2 * i + 1]), scale, -m));
            sum += a + b;
            p[i] = kv_pack<BF>(a, b);
        }
        kv_tmem_store32(p, s_at + 32);
        l += sum;
        // The row tile's last product was issued before these scores were: it is done, and O rests.
        if (s > 0 && __any_sync(0xffffffffu, higher)) {
#pragma unroll 1
            for (int b = 0; b < S.value; b += 32) {
                uint32_t y[32];
                kv_tmem_load32(y, o_at + b);
#pragma unroll
                for (int i = 0; i < 32; i++) y[i] = __float_as_uint(__uint_as_float(y[i]) * fall);
                kv_tmem_store32(y, o_at + b);
            }
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        lt_pair_arrive(p_in);
    }
    fine = lt_pair_wait(bars + 8 * LT_P_END, 0, stop) && fine && !*stop;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const bool whole = A.splits == 1;
    const float by = !fine ? __int_as_float(0x7fffffff) : !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
    const int64_t token = J.q.start + (int64_t)row;
    if (!fine) l = by;
    if (valid && !whole) *(float2*)(A.part_ml + 2 * (((int64_t)blockIdx.y * total_new + token) * S.heads + J.head)) = make_float2(m, l);
    if (valid && whole && A.lse) A.lse[token * S.heads + J.head] = l == 0.f ? -KV_INF : (m + log2f(l)) * 0.6931471805599453f;
    const int apart_tile = min(J.see_all, J.hi) / LT_P_TOKENS;
    // the other CTA has looked after the other half of V
    uint32_t others, other_at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(other_at) : "r"((uint32_t)__cvta_generic_to_shared(&M.some_apart)), "r"(lt_rank() ^ 1u));
    asm volatile("ld.relaxed.cluster.shared::cluster.u32 %0, [%1];" : "=r"(others) : "r"(other_at) : "memory");
    const bool some_apart = others | *(volatile uint32_t*)&M.some_apart;
#pragma unroll 1
    for (int b = 0; b < S.value; b += 32) {
        uint32_t x[32];
        __syncwarp();
        if (steps > 0) {
            kv_tmem_load32(x, o_at + b);
        } else {
#pragma unroll
            for (int i = 0; i < 32; i++) x[i] = 0u;
        }
        if (!valid) continue;
        float y[32];
#pragma unroll
        for (int i = 0; i < 32; i++) y[i] = l == 0.f ? 0.f : __uint_as_float(x[i]) * by;
        // what the guard took out of V, for rows that see the token
#pragma unroll 1
        for (int w = 0; some_apart && w < 4 * LT_P_APART; w++) {
            uint32_t bits;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(other_at) : "r"((uint32_t)__cvta_generic_to_shared(&M.apart[0][w])), "r"(lt_rank() ^ 1u));
            asm volatile("ld.relaxed.cluster.shared::cluster.u32 %0, [%1];" : "=r"(bits) : "r"(other_at) : "memory");
            for (bits |= ((volatile uint32_t*)M.apart)[w]; bits; bits &= bits - 1) {
                const int t = apart_tile * LT_P_TOKENS + 32 * w + __ffs(bits) - 1;
                if (t > place) continue;
                const uint16_t* v = A.v + (J.key_start + t) * A.v_token_stride + J.head * A.v_head_stride + b;
#pragma unroll
                for (int i = 0; i < 32; i += 8) {
                    float e[8];
                    kv_widen8<BF>(*(const uint4*)(v + i), e);
#pragma unroll
                    for (int k = 0; k < 8; k++)
                        if (!(fabsf(e[k]) < KV_INF)) y[i + k] += e[k];
                }
            }
        }
        if (!whole) {
            float* dst = A.part_o + (((int64_t)blockIdx.y * total_new + token) * S.heads + J.head) * S.value + b;
#pragma unroll
            for (int i = 0; i < 8; i++) *(float4*)(dst + 4 * i) = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
            continue;
        }
        uint16_t* dst = (uint16_t*)A.out.data + token * A.out.token_stride + J.head * A.out.head_stride + b;
#pragma unroll
        for (int i = 0; i < 4; i++) *(uint4*)(dst + 8 * i) = kv_narrow8<BF>(y + 8 * i);
    }
}

// Warp 8
__device__ __forceinline__ void lt_prompt_bring(const LtShape& S, const LtBatch& B, const LtPrompt& A, const LtPromptJob& J, int steps, const CUtensorMap* pool,
                                                const CUtensorMap* k_map, const CUtensorMap* v_map, uint32_t sm_at, LtPromptMisc& M, uint32_t bars)
{
    const int lane = threadIdx.x & 31, rank = lt_rank(), k_chunks = lt_prompt_k_chunks(S), box = min(S.block_tokens, 64), boxes = LT_P_TOKENS / box;
    const uint32_t ring = sm_at + 2 * k_chunks * LT_P_CHUNK, stage_bytes = k_chunks * LT_P_KEYS + LT_P_CHUNK, k_in = lt_of_first(bars) + 8 * LT_P_K_IN;
    volatile int* const stop = &M.stop;
    int s = 0, k_brought = 0, stage = 0;
    uint32_t phase = 0;
    for (; s < steps; s++) {
        // lane: a box of the tile's shared keys, of both halves of the tokens
        const int t0 = LT_P_TOKENS * (J.first_step + s), t = t0 + lane * box;
        const int page = lane < boxes && t < J.hi ? lt_page(B, J.seq, t >> S.block_shift) : -1;
        const uint32_t some = __ballot_sync(0xffffffffu, page >= 0);
        uint32_t present = 0;
        for (int b = 0; b < boxes; b++)
            if (some >> b & 1) present |= ((1u << (box / 16)) - 1) << (b * (box / 16));
        if (!lt_pair_wait(bars + 8 * (LT_P_K_OUT + stage), phase ^ 1, stop)) break;
        if (lane == 0) ((volatile uint32_t*)M.present)[s % LT_P_NOTES] = present;
        kv_warp_arrive(bars + 8 * (LT_P_NOTE + s % LT_P_NOTES));
        const uint32_t to = ring + stage * stage_bytes, bar = k_in + 8 * stage, v_bar = bars + 8 * (LT_P_V_IN + stage);
        if (rank == 0) lt_expect(bars + 8 * (LT_P_K_IN + stage), 2 * (k_chunks - 1) * LT_P_KEYS + __popc(some) * box * LT_CHUNK_ROW);
        for (int k = 0; k < k_chunks - 1; k++) lt_pair_tma(to + k * LT_P_KEYS, k_map, 64 * k, (int)J.key_start + t0 + 64 * rank, A.k_heads ? J.head : 0, bar);
        for (int b = 0; b < boxes / 2; b++) {
            const int from = lt_uniform(page, rank * (boxes / 2) + b);
            if (from >= 0) lt_pair_tma(to + (k_chunks - 1) * LT_P_KEYS + b * box * LT_CHUNK_ROW, pool, S.latent, (t0 + 64 * rank + b * box) & (S.block_tokens - 1), from, bar);
        }
        k_brought++;
        if (!lt_pair_wait(bars + 8 * (LT_P_V_OUT + stage), phase ^ 1, stop)) break;
        lt_expect(v_bar, LT_P_CHUNK);
        // 64 channels from this CTA's half on; of values of 64 channels the products take the first 32
        lt_tma(to + k_chunks * LT_P_KEYS, v_map, rank * (S.value / 2), (int)J.key_start + t0, A.v_heads ? J.head : 0, v_bar);
        stage = stage == LT_P_STAGES - 1 ? 0 : stage + 1;
        phase ^= stage == 0;
    }
    // what is on its way, to both CTAs, arrives before they end
    for (int back = 1; rank == 0 && back <= LT_P_STAGES && back <= k_brought; back++)
        (void)kv_wait(bars + 8 * (LT_P_K_IN + (k_brought - back) % LT_P_STAGES), (k_brought - back) / LT_P_STAGES & 1);
    for (int back = 1; back <= LT_P_STAGES && back <= s; back++) (void)kv_wait(bars + 8 * (LT_P_V_IN + (s - back) % LT_P_STAGES), (s - back) / LT_P_STAGES & 1);
}

// Warp 9 of the first CTA.  A barrier's answer takes some 270 cycles while the tensor cores read: where the time does not matter it is asked early.
template <bool BF>
__device__ __forceinline__ void lt_prompt_products(const LtShape& S, const LtPromptJob& J, int steps, int parts, uint32_t sm_at, LtPromptMisc& M, uint32_t bars, uint32_t tmem)
{
    const int k_chunks = lt_prompt_k_chunks(S);
    constexpr uint32_t kind = 1u << 4 | (BF ? 1u << 7 | 1u << 10 : 0u) | (2 * LT_P_ROWS / 16) << 24;
    constexpr uint32_t s_what = kind | (LT_P_TOKENS / 8) << 17;
    const uint32_t o_what = kind | (uint32_t)S.value / 8 << 17 | 1u << 16;                   // V is the operand whose N runs along the row
    const uint32_t ring = sm_at + 2 * k_chunks * LT_P_CHUNK, stage_bytes = k_chunks * LT_P_KEYS + LT_P_CHUNK;
    const uint64_t q_desc = kv_desc(sm_at, 16, 1024), k_desc = kv_desc(ring, 16, 1024), v_desc = kv_desc(ring + k_chunks * LT_P_KEYS, LT_P_CHUNK, 1024);
    volatile int* const stop = &M.stop;
    auto scores = [&](int m, int stage) {
        const uint64_t a = q_desc + m * k_chunks * (LT_P_CHUNK >> 4), b = k_desc + stage * (stage_bytes >> 4);
        const uint32_t d = tmem + 128 * m;
        lt_pair_mma_ss<4, 2, 2>(d, a, b, s_what, false);
        if (k_chunks == 3) lt_pair_mma_ss<4, 2, 2>(d, a + (LT_P_CHUNK >> 4), b + (LT_P_KEYS >> 4), s_what, true);
        const uint64_t ar = a + (k_chunks - 1) * (LT_P_CHUNK >> 4), br = b + (k_chunks - 1) * (LT_P_KEYS >> 4);
        lt_pair_mma_ss<2, 2, 2>(d, ar, br, s_what, true);
        if (S.rope == 64) lt_pair_mma_ss<2, 2, 2>(d, ar + 4, br + 4, s_what, true);
        lt_pair_commit(bars + 8 * (LT_P_S_IN + m));
    };
    auto answers = [&](int m, int stage, bool add) { lt_pair_mma_ts<8, 2048 / 16>(tmem + 256 + 128 * m, tmem + 128 * m, v_desc + stage * (stage_bytes >> 4), o_what, add); };
    if (!lt_pair_wait(bars + 8 * LT_P_Q_IN, 0, stop)) return;
    // step s of a row tile: its answers when its weights are made, and then the scores of step s + 1 in the weights' place
    int stage = 0, next = 0;                             // of step s and of step s + 1
    uint32_t phase = 0, next_phase = 0, keys = 0;        // keys: whether the next step's are known to be there
    for (int s = -1; s < steps; s++) {
        const uint32_t k_in = bars + 8 * (LT_P_K_IN + next), v_ok = bars + 8 * (LT_P_V_OK + stage);
        const bool more = s + 1 < steps;
        if (s >= 0) {
            const uint32_t values = lt_pair_ended(v_ok, phase);
            keys = more ? lt_pair_ended(k_in, next_phase) : 1u;
            if (!__all_sync(0xffffffffu, values) && !lt_pair_wait(v_ok, phase, stop)) return;
        }
        for (int m = 0; m < parts; m++) {
            const int steps_m = m ? J.steps1 : J.steps0;
            if (s >= 0 && s < steps_m) {
                if (!lt_pair_wait(bars + 8 * (LT_P_P_IN + m), s & 1, stop)) return;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                answers(m, stage, s > 0);
            }
            if (m == parts - 1 && s >= 0) lt_pair_commit(bars + 8 * (LT_P_V_OUT + stage));
            if (m == 0 && more && !__all_sync(0xffffffffu, keys) && !lt_pair_wait(k_in, next_phase, stop)) return;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            if (s + 1 < steps_m) scores(m, next);
        }
        if (more) lt_pair_commit(bars + 8 * (LT_P_K_OUT + next));
        stage = next;
        phase = next_phase;
        next = next == LT_P_STAGES - 1 ? 0 : next + 1;
        next_phase ^= next == 0;
    }
}

// Warps 10 and 11: V of tokens that are not there becomes zeros.  Where some rows do not see a token, what is not finite in its V becomes 0
// too (a weight of 0 times it would not be 0), and is noted down: rows that see it add it at the end.
template <bool BF>
__device__ __forceinline__ void lt_prompt_guard(const LtShape& S, const LtPromptJob& J, int steps, uint8_t* sm, LtPromptMisc& M, uint32_t bars)
{
    const int n = threadIdx.x - 320, k_chunks = lt_prompt_k_chunks(S);
    uint8_t* const ring = sm + 2 * k_chunks * LT_P_CHUNK + k_chunks * LT_P_KEYS;
    const uint32_t v_ok = lt_of_first(bars) + 8 * LT_P_V_OK;
    volatile int* const stop = &M.stop;
    const int see_all = min(J.see_all, J.hi), apart_tile = see_all / LT_P_TOKENS;
    int stage = 0;
    uint32_t phase = 0;
    for (int s = 0; s < steps; s++) {
        if (!kv_warp_wait(bars + 8 * (LT_P_NOTE + s % LT_P_NOTES), s / LT_P_NOTES & 1, stop)) return;
        if (!kv_warp_wait(bars + 8 * (LT_P_V_IN + stage), phase, stop)) return;
        const int t0 = LT_P_TOKENS * (J.first_step + s), nth_apart = J.first_step + s - apart_tile;
        const uint32_t present = ((volatile uint32_t*)M.present)[s % LT_P_NOTES];
        if (lt_prompt_ragged(J, t0, present)) {
            uint8_t* const v_sm = ring + stage * (k_chunks * LT_P_KEYS + LT_P_CHUNK);
            for (int i = n; i < LT_P_TOKENS * 8; i += 64) {
                const int t = i & 127, piece = i >> 7;
                uint4* const at = (uint4*)(v_sm + lt_at(t, piece));
                const bool there = lt_prompt_there(J, t0, t >> 5, present) >> (t & 31) & 1;
                if (there && t0 + t < see_all) continue;
                const uint4 w = *at;
                uint4 f = make_uint4(0, 0, 0, 0);
                if (there) f = make_uint4(lt_finite2<BF>(w.x), lt_finite2<BF>(w.y), lt_finite2<BF>(w.z), lt_finite2<BF>(w.w));
                if (f.x != w.x || f.y != w.y || f.z != w.z || f.w != w.w) {
                    *at = f;
                    if (there && nth_apart < LT_P_APART) {
                        atomicOr(&M.apart[nth_apart][t >> 5], 1u << (t & 31));
                        M.some_apart = 1;
                    }
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            lt_pair_release(v_ok + 8 * stage);
        } else {
            lt_pair_arrive(v_ok + 8 * stage);
        }
        stage = stage == LT_P_STAGES - 1 ? 0 : stage + 1;
        phase ^= stage == 0;
    }
}

template <bool BF>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(LT_P_THREADS, 1)
    lt_prompt_kernel(const LtShape S, const LtBatch B, const LtPrompt A, const __grid_constant__ CUtensorMap pool, const __grid_constant__ CUtensorMap k_map,
                     const __grid_constant__ CUtensorMap v_map)
{
    extern __shared__ uint8_t lt_raw[];
    uint8_t* const sm = lt_raw + (-(uint32_t)__cvta_generic_to_shared(lt_raw) & 1023u);
    const uint32_t sm_at = (uint32_t)__cvta_generic_to_shared(sm);
    const int warp = threadIdx.x >> 5, k_chunks = lt_prompt_k_chunks(S);
    LtPromptMisc& M = *(LtPromptMisc*)(sm + 2 * k_chunks * LT_P_CHUNK + LT_P_STAGES * (k_chunks * LT_P_KEYS + LT_P_CHUNK));
    const uint32_t bars = (uint32_t)__cvta_generic_to_shared(M.bars);
    asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
    LtPromptJob J;
    const int job = blockIdx.x >> 1;
    J.seq = blockIdx.z;
    J.head = job / A.tiles;
    J.row = (A.tiles - 1 - job % A.tiles) * 4 * LT_P_ROWS;                   // those that see most first
    J.q = lt_seq(B, J.seq);
    if (J.row >= J.q.n) return;                          // both CTAs of the pair
    J.rows = min(J.q.n - J.row, 4 * LT_P_ROWS);
    const int parts = J.rows > 2 * LT_P_ROWS ? 2 : 1;
    J.key_start = A.key_starts[J.seq];
    J.lo = (int)min(max(-J.key_start, (int64_t)0), (int64_t)J.q.len);
    J.hi = (int)min(max((int64_t)A.total_keys - J.key_start, (int64_t)0), (int64_t)J.q.len);
    J.see_all = max(J.q.len - J.q.n + J.row + 1, 0);
    auto steps_to = [&](int rows) {
        const int end = min(J.q.len - J.q.n + J.row + rows, J.hi);
        return end > J.lo ? (end + LT_P_TOKENS - 1) / LT_P_TOKENS : 0;
    };
    J.steps0 = steps_to(min(J.rows, 2 * LT_P_ROWS));
    J.steps1 = parts == 2 ? steps_to(J.rows) : 0;
    const int share = (max(J.steps0, J.steps1) + A.splits - 1) / A.splits;   // this pair's run of them
    J.first_step = share * blockIdx.y;
    J.steps0 = min(max(J.steps0 - J.first_step, 0), share);
    J.steps1 = min(max(J.steps1 - J.first_step, 0), share);
    const int steps = max(J.steps0, J.steps1);
    if (threadIdx.x == 0) {
        for (int i = 0; i < LT_P_BARS; i++)
            lt_init(bars + 8 * i, i >= LT_P_V_OK && i < LT_P_V_OUT ? 4 : i == LT_P_P_IN || i == LT_P_P_IN + 1 ? 8 : i == LT_P_Q_IN ? 8 * parts : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        M.stop = 0;
        M.some_apart = 0;
        for (int i = 0; i < 4 * LT_P_APART; i++) M.apart[0][i] = 0;
    }
    if (warp == 9) asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"((uint32_t)__cvta_generic_to_shared(&M.tmem)) : "memory");
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    kv_cluster_sync();                                   // the other CTA's barriers are there, too
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *(volatile uint32_t*)&M.tmem;  // S_0, S_1, O_0, O_1: 128 columns each
    if (warp < 8) {
        if (warp < 4 * parts) lt_prompt_rows<BF>(S, A, B.total_new, J, warp >> 2, sm_at, M, bars, tmem);
    } else if (warp == 8) {
        lt_prompt_bring(S, B, A, J, steps, &pool, &k_map, &v_map, sm_at, M, bars);
    } else if (warp == 9) {
        if (lt_rank() == 0) {
            lt_prompt_products<BF>(S, J, steps, parts, sm_at, M, bars, tmem);
            __syncwarp();
            lt_pair_commit(bars + 8 * LT_P_END);         // the answers are there, and nothing is on its way any more when the memory is given back
            kv_wait(bars + 8 * LT_P_END, 0);
            __syncwarp();
        }
    } else {
        lt_prompt_guard<BF>(S, J, steps, sm, M, bars);
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    kv_cluster_sync();                                   // neither ends while the other may reach it
    if (warp == 9) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

// Joins the answers of pairs that shared a job's tokens, each with its own largest score m and sum l, in the shares' order: a warp takes a row,
// 128 / 32 or 64 / 32 channels a lane.  Answers wait in 32 bits, so that the only further rounding is the answer's own.
#define LT_P_JOIN_THREADS 128
template <bool BF> __global__ void __launch_bounds__(LT_P_JOIN_THREADS) lt_prompt_join_kernel(const LtShape S, const LtBatch B, const LtPrompt A)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, w = blockIdx.x * (LT_P_JOIN_THREADS / 32) + (threadIdx.x >> 5), j = w / S.heads, head = w - j * S.heads;
    const LtSeq q = lt_seq(B, blockIdx.y);
    if (j >= q.n) return;
    const int64_t token = q.start + (int64_t)j, row = token * S.heads + head, step = (int64_t)B.total_new * S.heads;
    float m = KV_M_NONE, l = 0.f, sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < A.splits; s++) m = fmaxf(m, A.part_ml[2 * (s * step + row)]);
#pragma unroll 4
    for (int s = 0; s < A.splits; s++) {
        const float2 ml = *(const float2*)(A.part_ml + 2 * (s * step + row));
        const float by = kv_exp2(ml.x - m), *o = A.part_o + (s * step + row) * S.value;
        l += ml.y * by;
        if (S.value == 128) {
            const float4 x = *(const float4*)(o + 4 * lane);
            sum[0] = fmaf(x.x, by, sum[0]);
            sum[1] = fmaf(x.y, by, sum[1]);
            sum[2] = fmaf(x.z, by, sum[2]);
            sum[3] = fmaf(x.w, by, sum[3]);
        } else {
            const float2 x = *(const float2*)(o + 2 * lane);
            sum[0] = fmaf(x.x, by, sum[0]);
            sum[1] = fmaf(x.y, by, sum[1]);
        }
    }
    const float by = l == 0.f ? 0.f : 1.f / l;
    uint16_t* const out = (uint16_t*)A.out.data + token * A.out.token_stride + head * A.out.head_stride;
    if (S.value == 128) *(uint2*)(out + 4 * lane) = make_uint2(kv_pack<BF>(sum[0] * by, sum[1] * by), kv_pack<BF>(sum[2] * by, sum[3] * by));
    else *(uint32_t*)(out + 2 * lane) = kv_pack<BF>(sum[0] * by, sum[1] * by);
    if (lane == 0 && A.lse) A.lse[row] = l == 0.f ? -KV_INF : (m + log2f(l)) * 0.6931471805599453f;
}
