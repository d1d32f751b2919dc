// fastrack_kv_prompt.cuh -- attention of many query rows over the 8-bit cache, on the 5th-generation tensor cores.
#pragma once
#include <type_traits>
#include "fastrack_kv_attend.cuh"

// One CTA takes 256 rows (two tiles of 128) of one kv head of one sequence against a chunk of the tokens, 128 at a time:
//     S_m = Q_m K^T  (tensor memory)  ->  P_m = weights as f16 (tensor memory, over S_m)  ->  O_m += P_m V.
// Warps 0-3 and 4-7 make P_0 and P_1 (a thread per row: no exchange between lanes), warps 8-11 bring the codes and widen them to f16
// in shared memory, where the tensor cores read them, and warp 12 issues the products.  S is made in two halves of 64 tokens, one
// while the other's weights are: both row tiles and both halves keep the tensor cores and the exponentials going at once, and the two
// row tiles share the widened K and V.
//
// What bounds it, per 128 tokens and SM: the products 4 x 512 cycles; shared memory 2560 (Q twice and K for S, V for O, the widened
// codes' way in: 320 KB at 128 B a cycle); the exponentials 2 x 128 x 128 at 16 a cycle, 2048.  It takes some 5000: a step of a row
// tile is a chain (scores from tensor memory, largest, exponentials, weights back) of some 2300 cycles, half of them exponentials,
// in which every access to shared memory, a barrier's too, waits for the tensor cores' reads (150 to 300 cycles).
// 3 x 1024 new tokens over up to 6100, 32 heads of 128, bf16: 315 us = 610 TFLOP/s of the visible pairs, tensor cores active 35 %.
// What it came from: one m16n8k16 row tile per pass 2231 us; this division of work, codes unrolled and generic addressing 843; packed
// arithmetic and less code 369; two halves and products issued by a converged warp 348.  Two threads per row took 375.
//
// What f16 operands or these steps would not hold right is taken apart at the end, token by token in 32 bits by the rows that see it: 16 tokens
// of the unfinished block with a value that is not finite or with sizes 2^8 apart, and 64 tokens whose scores may pass KV_P_LARGE, where
// y - m (see KV_P_MOST) would be rounded to steps of a quarter or more.  Both are rare; a third kind of step for them cost all others 3 to 20 %
// in registers.
#define KV_P_LARGE 0x1p22f
#define KV_P_ROWS 128                   // of a row tile
#define KV_P_TOKENS 128
#define KV_P_THREADS 416
#define KV_P_GROUPS (KV_P_TOKENS / KV_HALF)
#define KV_P_AHEAD 4                    // pairs of values between an exponential and the use of its result

template <int D> struct KvPrompt {
    static constexpr int HALVES = (D + 63) / 64;                             // runs of 64 channels: 128-byte rows, swizzled by the row's number
    static constexpr int TILE = HALVES * KV_P_TOKENS * 128;                  // bytes of a tile of 128 rows as f16
    static constexpr int Q = 0, K = 2 * TILE, V = 4 * TILE, SCALES = 6 * TILE, POWERS = SCALES + 4 * (KV_P_GROUPS + 1) * 16,
                         BARS = POWERS + KV_P_GROUPS * 8, END = BARS + 256;
    static constexpr int SMEM = END + 1024;                                  // the base is rounded up to 1024
    // byte of the 16-byte piece that holds channels ch .. ch + 7 of a row
    __device__ static int at(int row, int ch) { return (ch >> 6) * KV_P_TOKENS * 128 + row * 128 + (((ch >> 3 & 7) ^ (row & 7)) << 4); }
};

__device__ __forceinline__ uint64_t kv_desc(uint32_t smem, uint32_t lbo, uint32_t sbo)   // swizzle of 128 bytes
{
    return (uint64_t)((smem >> 4) & 0x3fff) | (uint64_t)((lbo >> 4) & 0x3fff) << 16 | (uint64_t)((sbo >> 4) & 0x3fff) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// One thread of the warp issues; the warp as a whole comes here, so that the compiler keeps addresses and descriptors in uniform
// registers, where the instruction wants them (moved there one by one they held up each instruction by 60 cycles).
__device__ __forceinline__ void kv_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add)
{
    asm volatile("{\n\t.reg .pred p, e;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(what), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void kv_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add)
{
    asm volatile("{\n\t.reg .pred p, e;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(what), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void kv_commit(uint32_t bar)
{
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}
// For a whole warp, when all its lanes have come
__device__ __forceinline__ void kv_warp_arrive(uint32_t bar)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

#define KV_R8(x, i) "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3]), "=r"(x[i + 4]), "=r"(x[i + 5]), "=r"(x[i + 6]), "=r"(x[i + 7])
#define KV_W8(x, i) "r"(x[i]), "r"(x[i + 1]), "r"(x[i + 2]), "r"(x[i + 3]), "r"(x[i + 4]), "r"(x[i + 5]), "r"(x[i + 6]), "r"(x[i + 7])
// Loads with their wait: between the two the registers are not there yet, but the compiler, which does not know, might move them.
__device__ __forceinline__ void kv_tmem_load32(uint32_t (&x)[32], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : KV_R8(x, 0), KV_R8(x, 8), KV_R8(x, 16), KV_R8(x, 24) : "r"(at) : "memory");
}
__device__ __forceinline__ void kv_tmem_load64(uint32_t (&x)[64], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%64];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : KV_R8(x, 0), KV_R8(x, 8), KV_R8(x, 16), KV_R8(x, 24), KV_R8(x, 32), KV_R8(x, 40), KV_R8(x, 48), KV_R8(x, 56) : "r"(at) : "memory");
}
__device__ __forceinline__ void kv_tmem_store32(const uint32_t (&x)[32], uint32_t at)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
                 ::KV_W8(x, 0), KV_W8(x, 8), KV_W8(x, 16), KV_W8(x, 24), "r"(at) : "memory");
}
// Two 32-bit floats in one instruction
__device__ __forceinline__ uint64_t kv_pair(float a, float b)
{
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float2 kv_unpair(uint64_t d)
{
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(d));
    return f;
}
__device__ __forceinline__ uint64_t kv_fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

// Bounded wait that also ends when another warp has given up.
__device__ __forceinline__ bool kv_wait_or_stop(uint32_t bar, uint32_t parity, volatile int* stop)
{
#pragma unroll 1
    for (int i = 0; i < 1 << 14; i++) {
#pragma unroll 1
        for (int k = 0; k < 16; k++) {
            uint32_t done;
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                         : "=r"(done) : "r"(bar), "r"(parity) : "memory");
            if (done) return true;
        }
        if (*stop) return false;
    }
    *stop = 1;
    return false;
}

// Whether the phase has ended: one question, whose answer may be used much later.  (While the tensor cores read their operands, an
// access to shared memory, a barrier's too, takes 150 to 300 cycles.)
__device__ __forceinline__ uint32_t kv_ended(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done;
}
// The same answer for a whole warp.  All lanes ask: where one lane does, the compiler carries on with that lane apart from the others.
__device__ __forceinline__ bool kv_warp_wait(uint32_t bar, uint32_t parity, volatile int* stop)
{
    return __all_sync(0xffffffffu, kv_wait_or_stop(bar, parity, stop));
}

// 16 codes as 16 f16
template <bool E4M3> __device__ __forceinline__ void kv_widen16(const uint4& w, uint4& lo, uint4& hi)
{
    kv_widen4<E4M3>(w.x, lo.x, lo.y);
    kv_widen4<E4M3>(w.y, lo.z, lo.w);
    kv_widen4<E4M3>(w.z, hi.x, hi.y);
    kv_widen4<E4M3>(w.w, hi.z, hi.w);
}

// Barriers, 8 bytes each from T::BARS on.  K_IN has four phases in turn because the scales beside K stay until the weights are made; by
// the time that a tile's K comes in, the weights of the fourth tile before it are done.
// S_IN and P_IN: [row tile][half of the tile's tokens]; O_IN: an answer product of the row tile is done.  TAIL: the unfinished block's powers are there.
// What the places that are used again rest on (step s: half s & 1 of tile s >> 1):
//   Slot j & 3 of the scales is written for tile j + 4 behind K_OUT of tile j + 2, whose scores were issued behind P_IN of both halves of tile
//   j + 1: every row is past tile j.  A row may read a slot from K_IN of its tile on (before, it holds the fourth tile before), and not
//   after P_IN of its second half.
//   A half of S is written by scores(s + 2) behind answers(s), in the order of issue, and answers(s) behind P_IN(s): the rows have
//   read their scores and written their weights.
//   O_IN has a phase for every step, of which a row asks for s - 1, and only where O has to be multiplied: it may never have asked for
//   others.  The parity tells phase s - 1 from s - 2 because s - 2 is over: answers(s - 2) and its commit were issued before scores(s) and its
//   commit, whose end, S_IN(s), the row has seen.  And O rests meanwhile: answers(s) wait for the row's P_IN(s).
enum { KV_K_IN = 0, KV_K_OUT = 4, KV_V_IN = 6, KV_V_OUT = 8, KV_S_IN = 10, KV_P_IN = 14, KV_O_IN = 18, KV_Q_IN = 20, KV_TAIL = 21, KV_END = 22, KV_BARS = 23 };

// What a tile's slot of T::SCALES holds: per 16 tokens {K's scale, y and z of V's (see KV_P_MOST), whether the tokens are there}; and of each half
// the largest scale of K, negative where some tokens are not there.
struct KvSlot { float4 group[KV_P_GROUPS]; float k_most[2], pad[2]; };

// 8 channels of K (which = 0) or V (1) of a kv head's token, from the sequence's tail (page -2) or a page, as 32-bit numbers
template <bool BF, bool E4M3>
__device__ __forceinline__ void kv_held8(const KvShape& S, const KvBatch& B, const uint16_t* tail, int kh, int which, int page, int at, int ch, float* x)
{
    if (page == -2) {
        kv_widen8<BF>(*(const uint4*)(tail + ((int64_t)which * S.block_tokens + at) * S.head_dim + ch), x);
    } else {
        const float scale = kv_finite(kv_scales(S, B, page)[2 * kh + which]);
        const uint2 codes = *(const uint2*)(B.pool + (uint64_t)page * S.page_bytes + (uint64_t)which * S.codes_bytes + ((uint64_t)kh * S.block_tokens + at) * S.head_dim + ch);
        kv_decode4<E4M3>(codes.x, scale, x);
        kv_decode4<E4M3>(codes.y, scale, x + 4);
    }
}

// Of up to 16 tokens of the unfinished block, from src on, the largest values' magnitudes: the largest of them and the least that is not zero.  For a warp.
template <int D, bool BF> __device__ __forceinline__ float2 kv_prompt_sizes(const uint16_t* src, int there)
{
    constexpr int LANES = D == 64 ? 8 : 16, ROWS = 32 / LANES, STEPS = KV_HALF / ROWS;       // lanes of a row (of 96 channels, 12 take part)
    const int lane = threadIdx.x & 31, ch = lane % LANES * 8;
    uint32_t amax[STEPS], most = 0, least = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < STEPS; i++) {
        const int row = i * ROWS + lane / LANES;
        amax[i] = row < there && ch < D ? kv_amax8<BF>(*(const uint4*)(src + row * D + ch)) : 0u;
    }
#pragma unroll
    for (int i = 0; i < STEPS; i++) {
#pragma unroll
        for (int d = 1; d < LANES; d <<= 1) amax[i] = max(amax[i], __shfl_xor_sync(0xffffffffu, amax[i], d));
        most = max(most, amax[i]);
        least = min(least, amax[i] - 1u);                // zero counts as the largest
    }
    most = __reduce_max_sync(0xffffffffu, most);
    least = __reduce_min_sync(0xffffffffu, least) + 1u;
    return BF ? make_float2(__uint_as_float(most), __uint_as_float(least))
              : make_float2(__half2float(__ushort_as_half((unsigned short)most)), __half2float(__ushort_as_half((unsigned short)least)));
}

// 128 (query, head) rows' weights, made tile by tile by 128 threads, a row each, and their answers; see the head of this file.
template <int D, bool BF, bool E4M3>
__device__ __forceinline__ void kv_prompt_rows(const KvShape& S, const KvBatch& B, const KvAttend& A, const KvSeq& q, int seq, int kh, int tile_row, int m_tile,
                                               int chunk, int begin, int end, int tiles, uint8_t* sm, uint32_t bars, volatile int* stop, uint32_t* apart,
                                               uint32_t tmem)
{
    using T = KvPrompt<D>;
    const int warp = threadIdx.x >> 5, r = threadIdx.x & 127, rows = q.n * S.group, row = tile_row + KV_P_ROWS * m_tile + r;
    const bool valid = row < rows;
    const int64_t token = q.start + row / S.group;
    const int head = kh * S.group + row % S.group, place = valid ? q.len - q.n + row / S.group : -1;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21, s_at = tmem + lanes + 128 * m_tile, o_at = tmem + lanes + 256 + 128 * m_tile;
    const KvSlot* const slots = (const KvSlot*)(sm + T::SCALES);
    const int warps = tile_row + KV_P_ROWS < rows ? 8 : 4;                   // that do this
    float factor = S.scale_log2, score_most;
    {
        // the row of Q, as f16 (bf16: over a power of two near its largest), to shared memory
        const uint16_t* src = (const uint16_t*)A.q.data + token * A.q.token_stride + head * A.q.head_stride;
        float inv = 1.f, size = 0.f;                     // size: of the row's values as f16, the sum of magnitudes
        if (BF) {
            uint32_t amax = 0;
#pragma unroll 4
            for (int i = 0; i < D / 8; i++) amax = max(amax, valid ? kv_amax8<true>(*(const uint4*)(src + 8 * i)) : 0u);
            const float p = kv_power_below(amax);
            factor *= p;
            inv = kv_power_inverse(p);
        }
#pragma unroll 4
        for (int i = 0; i < D / 8; i++) {
            uint4 w = valid ? *(const uint4*)(src + 8 * i) : make_uint4(0, 0, 0, 0);
            float x[8];
            kv_widen8<BF>(w, x);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                x[e] *= inv;
                size += fabsf(x[e]);
            }
            if (BF) w = kv_narrow8<false>(x);
            *(uint4*)(sm + T::Q + m_tile * T::TILE + T::at(r, 8 * i)) = w;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        kv_warp_arrive(bars + 8 * KV_Q_IN);
        // no score of the warp's rows is larger than this times K's scale (a row with infinities or NaN has no answers to be careful of)
        score_most = __uint_as_float(__reduce_max_sync(0xffffffffu, size < KV_INF ? __float_as_uint(factor * size) : 0u)) * (E4M3 ? 448.f : 127.f);
    }
    // Powers of two for the unfinished block, 16 tokens at a time, while the first codes come.  What one power would not hold (values that are not
    // finite, tokens whose largest values are 2^8 apart; f16 K needs none) stays out of the products: the rows take it apart at the end.
    const int tail_begin = q.full << S.block_shift, tail_tile = begin + (tail_begin - begin) / KV_P_TOKENS * KV_P_TOKENS;
    const uint16_t* const tail = (const uint16_t*)B.tail + (uint64_t)seq * S.tail_values + (uint64_t)kh * 2 * S.block_tokens * D;
    if (tail_begin < end) {
        for (int g = warp; g < KV_P_GROUPS; g += warps) {
            const int t = tail_tile + KV_HALF * g, there = min(KV_HALF, q.len - t);
            if (t < tail_begin || t >= end) continue;
            const float2 k = kv_prompt_sizes<D, BF>(tail + (int64_t)(t - tail_begin) * D, there), v = kv_prompt_sizes<D, BF>(tail + ((int64_t)S.block_tokens + t - tail_begin) * D, there);
            auto wide = [](float2 sizes) { return !(sizes.x < KV_INF) || sizes.x > 256.f * sizes.y; };
            if ((threadIdx.x & 31) == 0) {
                ((float2*)(sm + T::POWERS))[g] = make_float2(kv_power_below(__float_as_uint(k.x)), kv_v_power(v.x));
                if ((BF && wide(k)) || wide(v)) atomicOr(apart, 1u << g);
            }
        }
        kv_warp_arrive(bars + 8 * KV_TAIL);
    }
    // rows of this warp: tokens up to see_all are seen by all of them, tokens behind low_all are in every one's window
    const int first_row = tile_row + KV_P_ROWS * m_tile + 32 * (warp & 3), last_row = min(first_row + 31, rows - 1);
    const int see_all = first_row + 31 < rows ? q.len - q.n + first_row / S.group : -1;
    const int low_all = A.window > 0 ? q.len - q.n + last_row / S.group - A.window : -1;
    const int unit_stride = B.max_new * S.group;        // units of weights: 64 tokens, or smaller blocks
    float* const units = A.unit_l2 && valid ? A.unit_l2 + ((int64_t)seq * S.kv_heads + kh) * A.units * unit_stride + row : nullptr;
    const bool small_units = units && S.block_tokens < 64;
    float m = KV_M_NONE, l = 0.f;                        // see KV_P_MOST
    bool fine = true;
    // Steps of 64 tokens: while this one's weights are made, the next one's scores are (in the other half of S).
    uint32_t ended = 0;                                  // whether this step's scores are known to be there
    for (int s = 0; s < 2 * tiles && fine; s++) {
        const int j = s >> 1, half = s & 1, t0 = begin + 64 * s;
        const uint32_t at = s_at + 64 * half;
        const KvSlot& slot = slots[j & 3];
        if (!half) fine = kv_warp_wait(bars + 8 * (KV_K_IN + (j & 3)), j >> 2 & 1, stop);
        float4 sc[4];                                    // the scales of the 16-token groups
#pragma unroll
        for (int g = 0; g < 4; g++) sc[g] = slot.group[4 * half + g];
        if (!__all_sync(0xffffffffu, ended)) fine = kv_warp_wait(bars + 8 * (KV_S_IN + 2 * m_tile + half), j & 1, stop) && fine;
        if (!fine) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const float k_most = slot.k_most[half];
        const bool ragged = __float_as_int(k_most) < 0 || t0 + 63 > see_all || t0 <= low_all;
        float fall = 1.f, z[4];                          // fall: what l and O are multiplied by for a new m
        uint64_t sum[4] = {0, 0, 0, 0};                  // of 16 tokens' weights each
        // Scores may be so large that y - m would be rounded to steps of a quarter or more: these rows see nothing here, and take the tokens apart at
        // the end.
        const bool large = !(fabsf(k_most) * score_most < KV_P_LARGE);
        if (large && (threadIdx.x & 31) == 0) atomicOr(apart, 256u << warp);
        auto pass = [&](auto some_hidden) {
            constexpr bool RAGGED = decltype(some_hidden)::value;
            uint32_t seen[2] = {0xffffffffu, 0xffffffffu};                   // which of 32 tokens the row sees
            float f[4];
#pragma unroll
            for (int g = 0; g < 4; g++) f[g] = sc[g].x * factor;
            if (RAGGED)
#pragma unroll
                for (int b = 0; b < 2; b++) {
                    const int t = t0 + 32 * b, upto = large ? 0 : min(max(place - t + 1, 0), 32), from = A.window > 0 ? min(max(place - A.window + 1 - t, 0), 32) : 0;
                    seen[b] = (uint32_t)(((uint64_t)1 << upto) - 1) & ~(uint32_t)(((uint64_t)1 << from) - 1);
                    if (sc[2 * b].w == 0.f) seen[b] &= 0xffff0000u;
                    if (sc[2 * b + 1].w == 0.f) seen[b] &= 0x0000ffffu;
                }
            uint32_t x[64];
            kv_tmem_load64(x, at);
            // the largest s + y; a scale is not negative, so that of 16 tokens with one scale the largest product is the largest score
            float top = -KV_INF;
#pragma unroll
            for (int g = 0; g < 4; g++) {
                if (RAGGED)
#pragma unroll
                    for (int i = 16 * g; i < 16 * g + 16; i++) x[i] = seen[g >> 1] >> (i & 31) & 1 ? x[i] : 0xff800000u;
                const int o = 16 * g;
                float u = fmaxf(fmaxf(__uint_as_float(x[o]), __uint_as_float(x[o + 1])), __uint_as_float(x[o + 2]));
                float w = fmaxf(fmaxf(__uint_as_float(x[o + 3]), __uint_as_float(x[o + 4])), __uint_as_float(x[o + 5]));
                u = fmaxf(fmaxf(u, __uint_as_float(x[o + 6])), __uint_as_float(x[o + 7]));
                w = fmaxf(fmaxf(w, __uint_as_float(x[o + 8])), __uint_as_float(x[o + 9]));
                u = fmaxf(fmaxf(u, __uint_as_float(x[o + 10])), __uint_as_float(x[o + 11]));
                w = fmaxf(fmaxf(w, __uint_as_float(x[o + 12])), __uint_as_float(x[o + 13]));
                u = fmaxf(fmaxf(u, __uint_as_float(x[o + 14])), __uint_as_float(x[o + 15]));
                top = fmaxf(top, fmaf(fmaxf(u, w), f[g], sc[g].y));                  // a NaN (0 times -inf where 16 hidden tokens have a scale of 0) does not count
            }
            // without a branch, behind which the compiler might leave the rows apart: the tensor memory's instructions want the warp whole
            const bool higher = top > m + KV_P_MOST;
            top -= KV_P_BITS;
            fall = higher ? kv_exp2(m - top) : 1.f;
            l *= fall;
            m = higher ? top : m;
            // A pair of values takes three steps, some pairs apart: an exponential's result comes after some 40 cycles, and the unit takes one
            // of a warp every 8, between which there is room for the other steps.
            float up[4];
#pragma unroll
            for (int g = 0; g < 4; g++) {
                up[g] = sc[g].y - m;
                z[g] = sc[g].z;
            }
            // ask for the next step's scores now
            ended = kv_ended(bars + 8 * (KV_S_IN + 2 * m_tile + (half ^ 1)), (s + 1) >> 1 & 1);
            uint32_t p[32], rest[BF ? 1 : 32];           // f16 answers: what rounding leaves out, see kv_weights
#pragma unroll
            for (int i = 0; i < 32 + KV_P_AHEAD; i++) {
                if (i < 32) {
                    const float fg = f[i >> 3], ug = up[i >> 3];
                    uint32_t &u = x[2 * i], &w = x[2 * i + 1];
                    const float2 e = kv_unpair(kv_fma2(kv_pair(__uint_as_float(u), __uint_as_float(w)), kv_pair(fg, fg), kv_pair(ug, ug)));
                    u = __float_as_uint(e.x);
                    w = __float_as_uint(e.y);
                    asm volatile("ex2.approx.ftz.f32 %0, %0;" : "+r"(u));
                    asm volatile("ex2.approx.ftz.f32 %0, %0;" : "+r"(w));
                }
                if (i >= KV_P_AHEAD) {
                    const int k = i - KV_P_AHEAD;
                    uint32_t &u = x[2 * k], &w = x[2 * k + 1];
                    if (RAGGED) {
                        u = seen[k >> 4] >> (2 * k & 31) & 1 ? u : 0u;
                        w = seen[k >> 4] >> ((2 * k & 31) + 1) & 1 ? w : 0u;
                    }
                    asm volatile("{\n\t.reg .b64 t;\n\tmov.b64 t, {%1, %2};\n\tadd.rn.f32x2 %0, %0, t;\n\t}" : "+l"(sum[k >> 3]) : "r"(u), "r"(w));
                    asm volatile("cvt.rn.f16x2.f32 %0, %2, %1;" : "=r"(p[k]) : "r"(u), "r"(w));
                    if (!BF) {
                        const float2 e = kv_unpack<false>(p[k]);
                        rest[BF ? 0 : k] = kv_pack<false>(__uint_as_float(u) - e.x, __uint_as_float(w) - e.y);
                    }
                }
            }
            kv_tmem_store32(p, at);                      // over the scores of the first 32 tokens
            if constexpr (!BF) kv_tmem_store32(rest, at + 32);
        };
        if (ragged || large) pass(std::true_type());
        else pass(std::false_type());
        if (s > 0 && __any_sync(0xffffffffu, fall != 1.f)) {
            // behind the product of the step before, the last that has been issued
            fine = kv_warp_wait(bars + 8 * (KV_O_IN + m_tile), (s - 1) & 1, stop);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
            for (int b = 0; b < D / 32; b++) {
                uint32_t y[32];
                kv_tmem_load32(y, o_at + 32 * b);
#pragma unroll
                for (int i = 0; i < 32; i++) y[i] = __float_as_uint(__uint_as_float(y[i]) * fall);
                kv_tmem_store32(y, o_at + 32 * b);
            }
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        kv_warp_arrive(bars + 8 * (KV_P_IN + 2 * m_tile + half));
        // behind the arrival: the row's sum, and the units'
        float w[4];
#pragma unroll
        for (int g = 0; g < 4; g++) {
            const float2 e = kv_unpair(sum[g]);
            w[g] = e.x + e.y;
            w[g] = w[g] == 0.f ? 0.f : w[g] * z[g];                          // a hidden block's scale may be NaN
        }
        const float total = (w[0] + w[1]) + (w[2] + w[3]);
        l += total;
        if (units && !small_units) {
            if (t0 < end) units[(int64_t)(t0 >> 6) * unit_stride] = kv_unit_log2(total, m);
        } else if (units) {
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const int t = t0 + KV_HALF * g;
                if (t < end && (S.block_tokens == 16 || !(g & 1)))
                    units[(int64_t)(t >> S.block_shift) * unit_stride] = kv_unit_log2(S.block_tokens == 16 ? w[g] : w[g] + w[g | 1], m);
            }
        }
    }
    if (fine && tiles > 0) fine = kv_warp_wait(bars + 8 * (KV_S_IN + 2 * m_tile), tiles & 1, stop);     // all products
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    // Tokens that the products left out, 16 at a time in 32 bits: their scores from the staged Q, then every 32 channels of O through registers.
    // The warp stays together for the tensor memory's instructions; a row that does not see a token has a weight of 0 for it.
    __syncwarp();
    const uint32_t left_out = *(volatile uint32_t*)apart & 255u;
    const bool some_large = *(volatile uint32_t*)apart >> 8 >> warp & 1;
    for (int t0 = some_large ? begin : tail_tile; t0 < end && (left_out || some_large); t0 += 64) {
        float k_most = 0.f;                              // as in the slot
        for (int t = t0; t < min(t0 + 64, end) && some_large; t += KV_HALF) {
            const int page = t < tail_begin ? kv_page(B, seq, t >> S.block_shift) : -1, group = (t - tail_tile) / KV_HALF;
            const float ks = page >= 0 ? kv_finite(kv_scales(S, B, page)[2 * kh]) : t >= tail_begin && !(left_out >> group & 1) ? ((const float2*)(sm + T::POWERS))[group].x : 0.f;
            k_most = fmaxf(k_most, ks);
        }
        const bool large = !(k_most * score_most < KV_P_LARGE);
#pragma unroll 1
        for (int t = t0; t < min(t0 + 64, end); t += KV_HALF) {
            const bool in_tail = t >= tail_begin;
            const int page = in_tail ? -2 : kv_page(B, seq, t >> S.block_shift), at = in_tail ? t - tail_begin : t & (S.block_tokens - 1);
            if (page == -1 || !(large || (in_tail && left_out >> ((t - tail_tile) / KV_HALF) & 1))) continue;
            float w[KV_HALF], top = m, sum = 0.f;
            uint32_t sees = 0;
#pragma unroll 1
            for (int i = 0; i < KV_HALF; i++) {
                w[i] = -KV_INF;
                if (t + i > place || t + i >= end || (A.window > 0 && t + i <= place - A.window)) continue;
                float dot = 0.f;
#pragma unroll 2
                for (int ch = 0; ch < D; ch += 8) {
                    float a[8], b[8];
                    kv_widen8<false>(*(const uint4*)(sm + T::Q + m_tile * T::TILE + T::at(r, ch)), a);
                    kv_held8<BF, E4M3>(S, B, tail, kh, 0, page, at + i, ch, b);
#pragma unroll
                    for (int e = 0; e < 8; e++) dot = fmaf(a[e], b[e], dot);
                }
                w[i] = __fmul_rn(dot, factor);           // rounded, for the largest and for the weights alike
                top = fmaxf(top, w[i]);
                sees |= 1u << i;
            }
            __syncwarp();
            const float fall = kv_exp2(m - top);
            m = top;
#pragma unroll 1
            for (int i = 0; i < KV_HALF; i++) sum += w[i] = kv_exp2(w[i] - m);
            l = l * fall + sum * (1.f / 134217728);
            if (units && sees) {                         // the sum was made without them: -inf, or other tokens'
                float& unit = units[(int64_t)(t >> A.unit_shift) * unit_stride];
                const float of_these = m + kv_log2(sum), most = fmaxf(unit, of_these);
                unit = sum == 0.f ? unit : most + kv_log2(kv_exp2(unit - most) + kv_exp2(of_these - most));
            }
#pragma unroll 1
            for (int b = 0; b < D / 32; b++) {
                uint32_t x[32];
                __syncwarp();
                kv_tmem_load32(x, o_at + 32 * b);
#pragma unroll
                for (int e = 0; e < 32; e++) x[e] = __float_as_uint(__uint_as_float(x[e]) * fall);
#pragma unroll 1
                for (int i = 0; i < KV_HALF && t + i < end; i++) {
                    const float weight = w[i];
                    const bool seen = sees >> i & 1;
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        float v[8];
                        kv_held8<BF, E4M3>(S, B, tail, kh, 1, page, at + i, 32 * b + e, v);
#pragma unroll
                        for (int k = 0; k < 8; k++) {
                            const float y = __uint_as_float(x[e + k]);
                            x[e + k] = __float_as_uint(fabsf(v[k]) < KV_INF ? fmaf(weight, v[k], y) : seen ? y + v[k] : y);
                        }
                    }
                }
                __syncwarp();
                kv_tmem_store32(x, o_at + 32 * b);
            }
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        }
    }
    __syncwarp();
    const float out_factor = !fine ? __int_as_float(0x7fffffff) : A.splits == 1 ? kv_over_sum(l) : 1.f;
#pragma unroll
    for (int b = 0; b < D / 32; b++) {
        uint32_t x[32];
        __syncwarp();
        if (tiles > 0) {
            kv_tmem_load32(x, o_at + 32 * b);
        } else {
#pragma unroll
            for (int i = 0; i < 32; i++) x[i] = 0u;
        }
        if (!valid) continue;
        float y[32];
#pragma unroll
        for (int i = 0; i < 32; i++) y[i] = l == 0.f && fine ? 0.f : __uint_as_float(x[i]) * out_factor;
        if (A.splits == 1) {
            uint16_t* dst = (uint16_t*)A.out.data + token * A.out.token_stride + head * A.out.head_stride + 32 * b;
#pragma unroll
            for (int i = 0; i < 4; i++) *(uint4*)(dst + 8 * i) = kv_narrow8<BF>(y + 8 * i);
        } else {
            float* dst = A.part_o + (((int64_t)chunk * B.total_new + token) * S.q_heads + head) * D + 32 * b;
#pragma unroll
            for (int i = 0; i < 8; i++) *(float4*)(dst + 4 * i) = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
        }
    }
    if (!valid) return;
    if (A.splits == 1) {
        const float l2 = kv_sum_log2(l, m);
        if (A.lse) A.lse[token * S.q_heads + head] = l2 * 0.6931471805599453f;
        A.lse2[kv_lse2_at(S, q, kh, row)] = l2;
    } else {
        *(float2*)(A.part_ml + 2 * (((int64_t)chunk * B.total_new + token) * S.q_heads + head)) = make_float2(m, l);
    }
}

// K and V of the tiles, widened to f16: 128 threads, of which warp w has tokens 32 w .. 32 w + 31 of a tile.
template <int D, bool BF, bool E4M3>
__device__ __forceinline__ void kv_prompt_bring(const KvShape& S, const KvBatch& B, const KvSeq& q, int seq, int kh, int begin, int end, int tiles, uint8_t* sm,
                                                uint32_t bars, volatile int* stop, const volatile uint32_t* apart)
{
    using T = KvPrompt<D>;
    // A lane's share of 16 tokens, P pieces of 16 channels.  Eight rows by four pieces of 64 channels at a time: eight lanes then write
    // pieces of two neighbouring rows, which the swizzle keeps apart.  The last 32 of 96 channels go sixteen rows by two pieces.
    constexpr int P = D / 32;
    auto row_of = [](int lane, int i) { return D == 96 && i == 2 ? lane >> 1 : (lane >> 2) + 8 * (D == 128 ? i >> 1 : i); };
    auto channel_of = [](int lane, int i) { return D == 96 && i == 2 ? 64 + 16 * (lane & 1) : 16 * (lane & 3) + 64 * (D == 128 ? i & 1 : 0); };
    const int warp = threadIdx.x >> 5 & 3, lane = threadIdx.x & 31;
    const int tail_begin = q.full << S.block_shift;
    KvSlot* const slots = (KvSlot*)(sm + T::SCALES);
    const uint16_t* const tail = (const uint16_t*)B.tail + (uint64_t)seq * S.tail_values + (uint64_t)kh * 2 * S.block_tokens * D;
    // 16 tokens from t on: page >= 0, absent or behind the end -1, of the tail -2
    auto kind_of = [&](int t) { return t >= end ? -1 : t >= tail_begin ? -2 : kv_page(B, seq, t >> S.block_shift); };
    auto codes = [&](uint4 (&w)[2][P], int which, int t0, int2 kind) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int page = h ? kind.y : kind.x;
            const uint8_t* src = B.pool + (uint64_t)page * S.page_bytes + (uint64_t)which * S.codes_bytes +
                                 ((uint64_t)kh * S.block_tokens + ((t0 + KV_HALF * h) & (S.block_tokens - 1))) * D;
#pragma unroll
            for (int i = 0; i < P; i++) w[h][i] = page >= 0 ? __ldg((const uint4*)(src + row_of(lane, i) * D + channel_of(lane, i))) : make_uint4(0, 0, 0, 0);
        }
    };
    const volatile float2* const powers = (const volatile float2*)(sm + T::POWERS);
    auto store = [&](const uint4 (&w)[2][P], int which, int t0, int2 kind, uint8_t* dst) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            if ((h ? kind.y : kind.x) != -2) {
#pragma unroll
                for (int i = 0; i < P; i++) {
                    const int row = 32 * warp + KV_HALF * h + row_of(lane, i), ch = channel_of(lane, i);
                    uint4 lo, hi;
                    kv_widen16<E4M3>(w[h][i], lo, hi);   // an absent page's zero bytes are zeros
                    *(uint4*)(dst + T::at(row, ch)) = lo;
                    *(uint4*)(dst + T::at(row, ch + 8)) = hi;
                }
                continue;
            }
            const float inv = kv_power_inverse(which ? powers[2 * warp + h].y : powers[2 * warp + h].x);
#pragma unroll 1
            for (int i = 0; i < P; i++) {
                const int row = KV_HALF * h + row_of(lane, i), ch = channel_of(lane, i);
                uint4 v[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
                if (t0 + row < q.len) {
                    const uint4* src = (const uint4*)(tail + ((uint64_t)which * S.block_tokens + t0 + row - tail_begin) * D + ch);
                    v[0] = src[0];
                    v[1] = src[1];
                    if (BF || which)
#pragma unroll
                        for (int k = 0; k < 2; k++) {
                            float x[8];
                            kv_widen8<BF>(v[k], x);
#pragma unroll
                            for (int e = 0; e < 8; e++) x[e] *= inv;
                            v[k] = kv_narrow8<false>(x);
                        }
                }
                *(uint4*)(dst + T::at(32 * warp + row, ch)) = v[0];
                *(uint4*)(dst + T::at(32 * warp + row, ch + 8)) = v[1];
            }
        }
    };
    uint4 kw[2][P], vw[2][P];
    int t0 = begin + 32 * warp;
    int2 kind = make_int2(kind_of(t0), kind_of(t0 + KV_HALF));
    codes(kw, 0, t0, kind);
    codes(vw, 1, t0, kind);
    auto scale_of = [&](int page) { return page >= 0 ? __ldg((const float2*)(kv_scales(S, B, page) + 2 * kh)) : make_float2(0.f, 0.f); };
    int scale_page = kind_of(begin + KV_HALF * (lane & 7)), scale_next = kind_of(begin + KV_P_TOKENS + KV_HALF * (lane & 7));
    float2 scale = scale_of(scale_page);
    for (int j = 0; j < tiles; j++, t0 += KV_P_TOKENS) {
        const int2 next = make_int2(kind_of(t0 + KV_P_TOKENS), kind_of(t0 + KV_P_TOKENS + KV_HALF));
        KvSlot& slot = slots[j & 3];
        const int tile0 = begin + KV_P_TOKENS * j;
        if (!kv_warp_wait(bars + 8 * (KV_K_OUT + (j & 1)), (j >> 1 & 1) ^ 1, stop)) return;
        if (tile0 + KV_P_TOKENS > tail_begin && tail_begin < end) {
            // once: the tail lies in one tile
            if (!kv_warp_wait(bars + 8 * KV_TAIL, 0, stop)) return;
            if (*apart >> 2 * warp & 1) kind.x = -1;
            if (*apart >> 2 * warp & 2) kind.y = -1;
        }
        if (warp == 0) {
            // lane g < 8: 16 tokens' scales, asked for a tile ahead
            float ks = kv_finite(scale.x), vs = kv_finite(scale.y), k_most = ks;
            int page = scale_page;
            if (page == -2) {
                k_most = powers[lane & 7].x;
                vs = powers[lane & 7].y;
                ks = BF ? k_most : 1.f;
                if (*apart >> (lane & 7) & 1) {
                    page = -1;
                    k_most = 0.f;
                }
            }
            scale_page = scale_next;
            scale = scale_of(scale_page);
            scale_next = kind_of(tile0 + 2 * KV_P_TOKENS + KV_HALF * (lane & 7));
            const float2 share = kv_v_share(vs);
            const uint32_t absent = __ballot_sync(0xffffffffu, page == -1);
            k_most = fmaxf(k_most, __shfl_xor_sync(0xffffffffu, k_most, 1));
            k_most = fmaxf(k_most, __shfl_xor_sync(0xffffffffu, k_most, 2));
            if (lane < 8) slot.group[lane] = make_float4(ks, share.x, share.y, page == -1 ? 0.f : 1.f);
            if (lane < 8 && (lane & 3) == 0) slot.k_most[lane >> 2] = copysignf(k_most, absent >> lane & 15 ? -1.f : 1.f);
        }
        store(kw, 0, t0, kind, sm + T::K + (j & 1) * T::TILE);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        kv_warp_arrive(bars + 8 * (KV_K_IN + (j & 3)));
        codes(kw, 0, t0 + KV_P_TOKENS, next);
        if (!kv_warp_wait(bars + 8 * (KV_V_OUT + (j & 1)), (j >> 1 & 1) ^ 1, stop)) return;
        store(vw, 1, t0, kind, sm + T::V + (j & 1) * T::TILE);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        kv_warp_arrive(bars + 8 * (KV_V_IN + (j & 1)));
        codes(vw, 1, t0 + KV_P_TOKENS, next);
        kind = next;
    }
}

// The products, by one warp.  They run in the order in which they are issued: scores are written over weights after those have been
// used.
template <int D, bool BF>
__device__ __forceinline__ void kv_prompt_products(int tiles, int parts, uint32_t sm_at, uint32_t bars, volatile int* stop, uint32_t tmem)
{
    using T = KvPrompt<D>;
    // f32 += f16 * f16; M = 128, N in eights; V is the operand whose N runs along the row
    constexpr uint32_t shape = 1u << 4 | (uint32_t)(KV_P_ROWS / 16) << 24;
    constexpr uint32_t s_what = shape | (uint32_t)(64 / 8) << 17, o_what = shape | (uint32_t)(D / 8) << 17 | 1u << 16;
    auto scores = [&](int s, int m) {                    // of 64 tokens
        const int j = s >> 1, half = s & 1;
        const uint64_t a = kv_desc(sm_at + T::Q + m * T::TILE, 16, 1024), b = kv_desc(sm_at + T::K + (j & 1) * T::TILE + half * 64 * 128, 16, 1024);
#pragma unroll
        for (int k = 0; k < D / 16; k++) {
            const uint32_t off = ((k >> 2) * KV_P_TOKENS * 128 + (k & 3) * 32) >> 4;
            kv_mma_ss(tmem + 128 * m + 64 * half, a + off, b + off, s_what, k > 0);
        }
        kv_commit(bars + 8 * (KV_S_IN + 2 * m + half));
    };
    auto answers = [&](int s, int m) {
        const int j = s >> 1, half = s & 1;
        const uint64_t b = kv_desc(sm_at + T::V + (j & 1) * T::TILE + half * 64 * 128, KV_P_TOKENS * 128, 1024);
#pragma unroll
        for (int k = 0; k < 4; k++) kv_mma_ts(tmem + 256 + 128 * m, tmem + 128 * m + 64 * half + 8 * k, b + (k * 2048 >> 4), o_what, s > 0 || k > 0);
        if (!BF)
#pragma unroll
            for (int k = 0; k < 4; k++) kv_mma_ts(tmem + 256 + 128 * m, tmem + 128 * m + 64 * half + 32 + 8 * k, b + (k * 2048 >> 4), o_what, true);
        kv_commit(bars + 8 * (KV_O_IN + m));
    };
    kv_wait_or_stop(bars + 8 * KV_Q_IN, 0, stop);
    // step s of a row tile: its answers when its weights are made, and then the scores of step s + 2, in the place of those weights
    for (int s = -2; s < 2 * tiles; s++) {
        const int next = s + 2, j = next >> 1;
        if (next < 2 * tiles && !(next & 1)) kv_wait_or_stop(bars + 8 * (KV_K_IN + (j & 3)), j >> 2 & 1, stop);
        if (s >= 0 && !(s & 1)) kv_wait_or_stop(bars + 8 * (KV_V_IN + (s >> 1 & 1)), s >> 2 & 1, stop);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        for (int m = 0; m < parts; m++) {
            if (s >= 0) {
                kv_wait_or_stop(bars + 8 * (KV_P_IN + 2 * m + (s & 1)), s >> 1 & 1, stop);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                answers(s, m);
            }
            if (next < 2 * tiles) scores(next, m);
        }
        if (s == 2 * tiles - 1)
            for (int m = 0; m < parts; m++) kv_commit(bars + 8 * (KV_S_IN + 2 * m));         // the end
        if (s >= 0 && (s & 1)) kv_commit(bars + 8 * (KV_V_OUT + (s >> 1 & 1)));
        if (next < 2 * tiles && (next & 1)) kv_commit(bars + 8 * (KV_K_OUT + (j & 1)));
    }
}

template <int D, bool BF, bool E4M3>
__global__ void __launch_bounds__(KV_P_THREADS, 1) kv_prompt_kernel(const KvShape S, const KvBatch B, const KvAttend A)
{
    using T = KvPrompt<D>;
    extern __shared__ uint8_t kv_raw[];
    // rounded up by an offset, so that the compiler still knows it for shared memory
    uint8_t* const sm = kv_raw + (-(uint32_t)__cvta_generic_to_shared(kv_raw) & 1023u);
    const uint32_t sm_at = (uint32_t)__cvta_generic_to_shared(sm), bars = sm_at + T::BARS;
    const int warp = threadIdx.x >> 5;
    const int chunk = blockIdx.y, kh = blockIdx.x % S.kv_heads, tile_row = blockIdx.x / S.kv_heads * A.rows, seq = blockIdx.z;
    asm volatile("griddepcontrol.launch_dependents;");
    const KvSeq q = kv_seq(S, B, seq);
    const KvSpan span = kv_span(S, q, A.window, tile_row, A.rows);
    const int rows = q.n * S.group;
    if (tile_row >= rows) return;
    const int begin = span.begin + chunk * A.chunk, end = min(span.end, begin + A.chunk);
    if (begin >= end && chunk > 0) return;
    const int tiles = max((end - begin + KV_P_TOKENS - 1) / KV_P_TOKENS, 0), parts = tile_row + KV_P_ROWS < rows ? 2 : 1;

    volatile int* const stop = (volatile int*)(sm + T::BARS + 8 * KV_BARS);
    // apart: what the rows take apart at the end, the unfinished block's tile by 16 tokens in 8 bits, then a bit for each warp that left out 64
    uint32_t *const tmem_at = (uint32_t*)(sm + T::BARS + 8 * KV_BARS + 4), *const apart = tmem_at + 1;
    if (threadIdx.x == 0) {
        for (int i = 0; i < KV_BARS; i++) {
            const int count = i < KV_K_OUT || i == KV_V_IN || i == KV_V_IN + 1 || (i >= KV_P_IN && i < KV_O_IN) ? 4 : i == KV_Q_IN ? 4 * parts : i == KV_TAIL ? 4 * parts : 1;
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bars + 8 * i), "r"(count) : "memory");
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *stop = 0;
        *apart = 0;
    }
    if (warp == 12) asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"((uint32_t)__cvta_generic_to_shared(tmem_at)) : "memory");
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *(volatile uint32_t*)tmem_at;  // S_0, S_1, O_0, O_1: 128 columns each

    if (warp < 8) {
        if (warp < 4 * parts) kv_prompt_rows<D, BF, E4M3>(S, B, A, q, seq, kh, tile_row, warp >> 2, chunk, begin, end, tiles, sm, bars, stop, apart, tmem);
    } else if (warp < 12) {
        kv_prompt_bring<D, BF, E4M3>(S, B, q, seq, kh, begin, end, tiles, sm, bars, stop, apart);
    } else {
        kv_prompt_products<D, BF>(tiles, parts, sm_at, bars, stop, tmem);
        __syncwarp();
        kv_commit(bars + 8 * KV_END);                    // nothing is on its way any more when the memory is given back
        kv_wait(bars + 8 * KV_END, 0);
        __syncwarp();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 12) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}
