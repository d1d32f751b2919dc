// fastrack_kv.cu -- handle, launches and small kernels of the key-value cache operators (include/fastrack_kv.h).
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>
#include <atomic>
#include <new>
#include <type_traits>

#include "../../include/fastrack_kv.h"
#include "fastrack_kv_attend.cuh"
#include "fastrack_kv_device.cuh"
#include "fastrack_kv_prompt.cuh"

// ------------------------------------------------------------------------------------------------ rotary ----

#define KV_ROT_THREADS 256

template <bool BF> __device__ __forceinline__ void kv_turn_raw(const KvShape& S, const float* cs, const float* sn, uint4& a, uint4& b)
{
    float x[16];
    kv_widen8<BF>(a, x);
    kv_widen8<BF>(b, x + 8);
    kv_turn(S, x, cs, sn);
    a = kv_narrow8<BF>(x);
    b = kv_narrow8<BF>(x + 8);
}
template <bool BF> __device__ __forceinline__ void kv_turn16(const KvShape& S, int u, int64_t position, uint4& a, uint4& b)
{
    float cs[8], sn[8];
    kv_angles(S, u, position, false, cs, sn);
    kv_turn_raw<BF>(S, cs, sn, a, b);
}

// One thread turns one unit (16 channels) of a token in heads h0 .. h0 + per - 1: the unit's cosines and sines are made once for them, while
// the first heads' values are on their way.
template <bool BF, int AHEAD>
__device__ __forceinline__ void kv_turn_heads(const KvShape& S, const KvRows& in, const KvRows& out, const int64_t* positions, int64_t token, int u, int h0, int per,
                                              int heads, bool inverse)
{
    const KvUnit unit = kv_unit(S, u);
    if (!unit.turned && in.data == out.data) return;
    const uint16_t* src = (const uint16_t*)in.data + token * in.token_stride + h0 * in.head_stride;
    uint16_t* dst = (uint16_t*)out.data + token * out.token_stride + h0 * out.head_stride;
    const int n = min(per, heads - h0);
    float cs[8], sn[8];
    for (int h = 0; h < n; h += AHEAD) {
        uint4 a[AHEAD], b[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; k++)
            if (h + k < n) {
                a[k] = *(const uint4*)(src + (h + k) * in.head_stride + unit.a);
                b[k] = *(const uint4*)(src + (h + k) * in.head_stride + unit.b);
            }
        if (h == 0 && unit.turned) kv_angles(S, u, positions[token], inverse, cs, sn);
#pragma unroll
        for (int k = 0; k < AHEAD; k++)
            if (h + k < n) {
                if (unit.turned) kv_turn_raw<BF>(S, cs, sn, a[k], b[k]);
                *(uint4*)(dst + (h + k) * out.head_stride + unit.a) = a[k];
                *(uint4*)(dst + (h + k) * out.head_stride + unit.b) = b[k];
            }
    }
}

template <bool BF>
__global__ void __launch_bounds__(KV_ROT_THREADS) kv_rotary_kernel(const KvShape S, const KvRows in, const KvRows out, const int64_t* __restrict__ positions,
                                                                   const int64_t tokens, const int heads, const int per, const bool inverse)
{
    const int units = S.head_dim / 16, groups = (heads + per - 1) / per;
    const int64_t idx = (int64_t)blockIdx.x * KV_ROT_THREADS + threadIdx.x, token = idx / units / groups;
    if (token >= tokens) return;
    kv_turn_heads<BF, 4>(S, in, out, positions, token, (int)(idx % units), (int)(idx / units % groups) * per, per, heads, inverse);
}

// ------------------------------------------------------------------------------------------------ append ----

#define KV_APPEND_THREADS 256

struct KvAppend { KvRows k, v, q, q_out; int slots, quant_ctas, q_per; bool spread; };

// Raw values of unit u of a token: K (which = 0) or V of a new token, or what the tail has of one from before the call.
__device__ __forceinline__ const uint16_t* kv_unit_source(const KvShape& S, const KvBatch& B, const KvAppend& A, const KvSeq& q, int seq, int kh, int which, int token)
{
    const int j = token - (q.len - q.n);
    if (j < 0) return (const uint16_t*)B.tail + (uint64_t)seq * S.tail_values + ((uint64_t)(2 * kh + which) * S.block_tokens + (token & (S.block_tokens - 1))) * S.head_dim;
    const KvRows& r = which ? A.v : A.k;
    return (const uint16_t*)r.data + (q.start + j) * r.token_stride + kh * r.head_stride;
}

// The largest magnitude over the CTA, as bits (a NaN is larger than everything)
__device__ __forceinline__ uint32_t kv_cta_max(uint32_t amax, uint32_t* warp_max)
{
    amax = __reduce_max_sync(0xffffffffu, amax);
    if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < KV_APPEND_THREADS / 32; w++) amax = max(amax, warp_max[w]);
    return amax;
}

// One full block of one kv head: every value is read once and stays in registers between the search for the largest and the rounding.
// N: units per thread of K, and of V.  All loads go out before the first use.
template <bool BF, bool E4M3, int N>
__device__ __forceinline__ void kv_append_block(const KvShape& S, const KvBatch& B, const KvAppend& A, const KvSeq& q, int seq, int kh, int t0, int page,
                                                uint32_t (*warp_max)[KV_APPEND_THREADS / 32])
{
    constexpr float top = E4M3 ? 448.f : 127.f;
    const int units = S.head_dim / 16, items = S.block_tokens * units, tid = threadIdx.x;
    uint8_t* const dst = B.pool + (uint64_t)page * S.page_bytes;
    uint4 w[2][N][2];
#pragma unroll
    for (int which = 0; which < 2; which++)
#pragma unroll
        for (int k = 0; k < N; k++) {
            const int i = tid + k * KV_APPEND_THREADS;
            if (i < items) {
                const uint16_t* src = kv_unit_source(S, B, A, q, seq, kh, which, t0 + i / units);
                const KvUnit unit = kv_unit(S, i % units);
                w[which][k][0] = *(const uint4*)(src + unit.a);
                w[which][k][1] = *(const uint4*)(src + unit.b);
            } else {
                w[which][k][0] = w[which][k][1] = make_uint4(0, 0, 0, 0);
            }
        }
#pragma unroll
    for (int which = 0; which < 2; which++) {
        float x[N][16];
        float most = 0.f;
#pragma unroll
        for (int k = 0; k < N; k++) {
            const int i = tid + k * KV_APPEND_THREADS, u = i % units, j = t0 + i / units - (q.len - q.n);
            kv_widen8<BF>(w[which][k][0], x[k]);
            kv_widen8<BF>(w[which][k][1], x[k] + 8);
            if (which == 0 && i < items && j >= 0 && kv_unit(S, u).turned) {
                float cs[8], sn[8];
                kv_angles(S, u, B.positions[q.start + j], false, cs, sn);
                kv_turn(S, x[k], cs, sn);
            }
#pragma unroll
            for (int e = 0; e < 16; e++) most = kv_max_nan(most, x[k][e]);
        }
        const uint32_t amax = kv_cta_max(__float_as_uint(most) & 0x7fffffffu, warp_max[which]);
        const float peak = amax < __float_as_uint(0x1p-100f) ? 0.f : __uint_as_float(amax), factor = peak == 0.f ? 0.f : top / peak;
#pragma unroll
        for (int k = 0; k < N; k++) {
            const int i = tid + k * KV_APPEND_THREADS;
            if (i >= items) break;
#pragma unroll
            for (int e = 0; e < 16; e++) x[k][e] = __fmul_rn(x[k][e], factor);
            const KvUnit unit = kv_unit(S, i % units);
            uint8_t* row = dst + (uint64_t)which * S.codes_bytes + ((uint64_t)kh * S.block_tokens + i / units) * S.head_dim;
            *(uint2*)(row + unit.a) = make_uint2(kv_codes4<E4M3>(x[k]), kv_codes4<E4M3>(x[k] + 4));
            *(uint2*)(row + unit.b) = make_uint2(kv_codes4<E4M3>(x[k] + 8), kv_codes4<E4M3>(x[k] + 12));
        }
        if (tid == 0) ((float*)kv_scales(S, B, page))[2 * kh + which] = peak / top;
    }
}

// quant_ctas CTAs: one block that the call touches, of one kv head.  The CTA of a sequence's first block also writes the head's tail,
// after it has read what the tail held: no other CTA touches the head's tail row.  The others turn q.  Where the first kind fits on
// the device at once it comes first, since it takes longest (5 x 333 tokens and their reading back: 17.6 us, 19.5 with the kinds mixed).
// Where it doesn't, the two are spread evenly, since the others wait for memory where those compute (17478 tokens: 84 us, 89 in order).
template <bool BF, bool E4M3, int N>
__global__ void __launch_bounds__(KV_APPEND_THREADS, N < 4 ? 3 : 2) kv_append_kernel(const KvShape S, const KvBatch B, const KvAppend A)
{
    const int units = S.head_dim / 16, tid = threadIdx.x;
    auto first_kind = [&](unsigned cta) { return A.spread ? (int)((uint64_t)cta * A.quant_ctas / gridDim.x) : min((int)cta, A.quant_ctas); };   // of the CTAs before cta
    const int before = first_kind(blockIdx.x);
    if (first_kind(blockIdx.x + 1) == before) {
        const int groups = (S.q_heads + A.q_per - 1) / A.q_per;
        const int64_t idx = (int64_t)((int)blockIdx.x - before) * KV_APPEND_THREADS + tid;
        const int64_t token = idx / units / groups;
        if (token >= B.total_new) return;
        kv_turn_heads<BF, 2>(S, A.q, A.q_out, B.positions, token, (int)(idx % units), (int)(idx / units % groups) * A.q_per, A.q_per, S.q_heads, false);
        return;
    }
    const int kh = before % S.kv_heads, slot = before / S.kv_heads % A.slots, seq = before / S.kv_heads / A.slots;
    const KvSeq q = kv_seq(S, B, seq);
    if (q.n == 0) return;
    const int first = max(q.len - q.n, 0), block = (first >> S.block_shift) + slot;
    __shared__ uint32_t warp_max[2][KV_APPEND_THREADS / 32];
    if (block < q.full) {
        const int page = kv_page(B, seq, block);
        if (page >= 0) kv_append_block<BF, E4M3, N>(S, B, A, q, seq, kh, block << S.block_shift, page, warp_max);
    }
    if (slot == 0) {
        __syncthreads();                                // the old tail has been read
        const int from = max(q.full << S.block_shift, first);
        for (int i = tid; i < 2 * (q.len - from) * units; i += KV_APPEND_THREADS) {
            const int u = i % units, which = i / units & 1, token = from + i / units / 2;
            const KvUnit unit = kv_unit(S, u);
            const uint16_t* src = kv_unit_source(S, B, A, q, seq, kh, which, token);
            uint4 a = *(const uint4*)(src + unit.a), b = *(const uint4*)(src + unit.b);
            if (which == 0 && unit.turned) kv_turn16<BF>(S, u, B.positions[q.start + token - (q.len - q.n)], a, b);
            uint16_t* dst = (uint16_t*)B.tail + (uint64_t)seq * S.tail_values + ((uint64_t)(2 * kh + which) * S.block_tokens + (token & (S.block_tokens - 1))) * S.head_dim;
            *(uint4*)(dst + unit.a) = a;
            *(uint4*)(dst + unit.b) = b;
        }
    }
}

// ------------------------------------------------------------------------------------------------ read ----

template <bool BF, bool E4M3>
__global__ void __launch_bounds__(256) kv_read_kernel(const KvShape S, const KvBatch B, const KvRows ko, const KvRows vo)
{
    const int seq = blockIdx.z, which = blockIdx.y & 1, kh = blockIdx.y >> 1, pieces = S.head_dim / 8;
    // piece blockIdx.x * 256 + threadIdx.x of max_len * pieces: there may be 2^34, so the multiple of 256 * pieces is taken off first
    const int i = blockIdx.x % pieces * 256 + threadIdx.x, token = blockIdx.x / pieces * 256 + i / pieces, at = i % pieces * 8;
    if (token >= B.max_len) return;
    const KvSeq q = kv_seq(S, B, seq);
    const int block = token >> S.block_shift, in_block = token & (S.block_tokens - 1);
    uint4 w = make_uint4(0, 0, 0, 0);
    if (token < q.len) {
        if (block == q.full) {
            w = *(const uint4*)((const uint16_t*)B.tail + (uint64_t)seq * S.tail_values + ((uint64_t)(2 * kh + which) * S.block_tokens + in_block) * S.head_dim + at);
        } else {
            const int page = kv_page(B, seq, block);
            if (page >= 0) {
                const float scale = kv_scales(S, B, page)[2 * kh + which];
                const uint2 codes = *(const uint2*)(B.pool + (uint64_t)page * S.page_bytes + (uint64_t)which * S.codes_bytes +
                                                    ((uint64_t)kh * S.block_tokens + in_block) * S.head_dim + at);
                float x[8];
                kv_decode4<E4M3>(codes.x, scale, x);
                kv_decode4<E4M3>(codes.y, scale, x + 4);
                w = kv_narrow8<BF>(x);
            }
        }
    }
    const KvRows& r = which ? vo : ko;
    *(uint4*)((uint16_t*)r.data + ((int64_t)seq * B.max_len + token) * r.token_stride + kh * r.head_stride + at) = w;
}

// ------------------------------------------------------------------------------------------------ evict ----

#define KV_EVICT_THREADS 1024
#define KV_EVICT_KEYS 49152             // scores kept in shared memory; those of later blocks are added up again where they are needed

struct KvEvict {
    int table_stride, mass_stride, budget, keep_first, keep_last, keys;
    const int32_t *table, *lens;
    const float* mass;
    int32_t *table_out, *lens_out;
    float* mass_out;
    int32_t *evicted, *n_evicted;
};

// A float as an unsigned number of the same order; every NaN becomes the largest.
__device__ __forceinline__ uint32_t kv_order(float x)
{
    if (x != x) return 0xffffffffu;
    x += 0.f;                                           // -0 is 0
    const uint32_t b = __float_as_uint(x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Exclusive sum of `flag` over the CTA's threads in order, and the total; two barriers.
__device__ __forceinline__ int kv_rank(bool flag, int* warp_sums, int& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t votes = __ballot_sync(0xffffffffu, flag);
    if (lane == 0) warp_sums[warp] = __popc(votes);
    __syncthreads();
    const int sum = warp_sums[lane];
    int before = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) { const int o = __shfl_up_sync(0xffffffffu, before, d); if (lane >= d) before += o; }
    total = __shfl_sync(0xffffffffu, before, 31);
    __syncthreads();
    return __shfl_sync(0xffffffffu, before - sum, warp) + __popc(votes & ((1u << lane) - 1u));
}

#define KV_EVICT_COUNTS 8               // copies of the histogram: weights have few exponents, and one counter for all warps holds them up
#define KV_EVICT_HEADS 8                // heads whose weights a thread moves between two barriers

// Exclusive sums of CH flags per thread, in the order of b = c * THREADS + thread, and the total; two barriers.
template <int THREADS, int CH>
__device__ __forceinline__ void kv_ranks(const bool (&flag)[CH], int (&rank)[CH], int& total, int (*counts)[THREADS / 32])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t votes[CH];
#pragma unroll
    for (int c = 0; c < CH; c++) {
        votes[c] = __ballot_sync(0xffffffffu, flag[c]);
        if (lane == 0) counts[c][warp] = __popc(votes[c]);
    }
    __syncthreads();
    total = 0;
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const int mine = lane < THREADS / 32 ? counts[c][lane] : 0;
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) { const int o = __shfl_up_sync(0xffffffffu, upto, d); if (lane >= d) upto += o; }
        rank[c] = total + __shfl_sync(0xffffffffu, upto - mine, warp) + __popc(votes[c] & ((1u << lane) - 1u));
        total += __shfl_sync(0xffffffffu, upto, 31);
    }
    __syncthreads();
}

// Eviction of a sequence that one CTA holds in registers: up to CH * THREADS blocks with up to KV_EVICT_HEADS heads.  Everything is read
// once, before anything is written (in place is safe); the score of the last block to leave is found by radix selection, 8 bits at a
// time, and a block's new place is its place less the blocks before it that leave.
// Bound by the latency of its passes (one read, 4 x 3 barriers, 2, one write), not by its bytes.
template <int THREADS, int CH>
__global__ void __launch_bounds__(THREADS) kv_evict_resident_kernel(const KvShape S, const KvEvict A)
{
    __shared__ int hist[KV_EVICT_COUNTS][256], counts[CH][THREADS / 32], warp_sums[8], pick[3];
    const int seq = blockIdx.x, tid = threadIdx.x;
    const int len = max(A.lens[seq], 0), most = min(A.table_stride, A.mass_stride);
    const int full = min(len >> S.block_shift, most), held = min((len + S.block_tokens - 1) >> S.block_shift, most);
    const int lo = min(A.keep_first, full), hi = max(full - A.keep_last, lo);
    const int drop = min(max(full - A.budget, 0), hi - lo);
    const float* const mass = A.mass + (int64_t)seq * S.kv_heads * A.mass_stride;
    float* const mass_out = A.mass_out + (int64_t)seq * S.kv_heads * A.mass_stride;
    float w[CH][KV_EVICT_HEADS];
    int32_t page[CH];
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const int b = c * THREADS + tid;
        page[c] = b < held ? A.table[(int64_t)seq * A.table_stride + b] : -1;
#pragma unroll
        for (int h = 0; h < KV_EVICT_HEADS; h++) w[c][h] = b < held && h < S.kv_heads ? mass[(int64_t)h * A.mass_stride + b] : 0.f;
    }
    for (int i = tid; i < KV_EVICT_COUNTS * 256; i += THREADS) hist[i >> 8][i & 255] = 0;
    uint32_t key[CH];
    bool free[CH];
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const int b = c * THREADS + tid;
        free[c] = drop > 0 && b >= lo && b < hi;
        double x = 0.;
#pragma unroll
        for (int h = 0; h < KV_EVICT_HEADS; h++) x += w[c][h];
        key[c] = kv_order((float)x);
    }
    __syncthreads();
    uint32_t limit = 0;
    int ties = drop, equal = drop;                      // of the blocks with exactly the limit's score: those that leave, and all
    for (int shift = 24; shift >= 0 && drop > 0; shift -= 8) {
#pragma unroll
        for (int c = 0; c < CH; c++)
            if (free[c] && (shift == 24 || key[c] >> (shift + 8) == limit >> (shift + 8))) atomicAdd(&hist[tid >> 5 & (KV_EVICT_COUNTS - 1)][key[c] >> shift & 255], 1);
        __syncthreads();
        int mine = 0, upto = 0;
        if (tid < 256) {
#pragma unroll
            for (int k = 0; k < KV_EVICT_COUNTS; k++) { mine += hist[k][tid]; hist[k][tid] = 0; }
            upto = mine;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) { const int o = __shfl_up_sync(0xffffffffu, upto, d); if ((tid & 31) >= d) upto += o; }
            if ((tid & 31) == 31) warp_sums[tid >> 5] = upto;
        }
        __syncthreads();
        if (tid < 256) {
#pragma unroll
            for (int k = 0; k < 8; k++) upto += k < tid >> 5 ? warp_sums[k] : 0;
            if (upto - mine < ties && ties <= upto) { pick[0] = tid; pick[1] = ties - (upto - mine); pick[2] = mine; }
        }
        __syncthreads();
        limit |= (uint32_t)pick[0] << shift;
        ties = pick[1];
        equal = pick[2];
    }
    bool out[CH];
    int rank[CH], total;
    if (ties < equal) {                                 // of equals the lowest places leave
#pragma unroll
        for (int c = 0; c < CH; c++) out[c] = free[c] && key[c] == limit;
        kv_ranks<THREADS, CH>(out, rank, total, counts);
#pragma unroll
        for (int c = 0; c < CH; c++) out[c] = free[c] && (key[c] < limit || (out[c] && rank[c] < ties));
    } else {
#pragma unroll
        for (int c = 0; c < CH; c++) out[c] = free[c] && key[c] <= limit;
    }
    kv_ranks<THREADS, CH>(out, rank, total, counts);    // its barriers also stand between all reads and all writes
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const int b = c * THREADS + tid, to = b - rank[c];
        if (b >= held) continue;
        if (out[c]) {
            A.evicted[(int64_t)seq * A.table_stride + rank[c]] = page[c];
        } else {
            A.table_out[(int64_t)seq * A.table_stride + to] = page[c];
#pragma unroll
            for (int h = 0; h < KV_EVICT_HEADS; h++)
                if (h < S.kv_heads) mass_out[(int64_t)h * A.mass_stride + to] = w[c][h];
        }
    }
    for (int b = held - drop + tid; b < A.table_stride; b += THREADS) A.table_out[(int64_t)seq * A.table_stride + b] = -1;
    for (int b = drop + tid; b < A.table_stride; b += THREADS) A.evicted[(int64_t)seq * A.table_stride + b] = -1;
    for (int b = held - drop + tid; b < A.mass_stride; b += THREADS)
        for (int h = 0; h < S.kv_heads; h++) mass_out[(int64_t)h * A.mass_stride + b] = 0.f;
    if (tid == 0) {
        A.lens_out[seq] = len - (drop << S.block_shift);
        A.n_evicted[seq] = drop;
    }
}

// Any number of blocks and heads, by one CTA per sequence.  The score of the last block to leave is found by radix selection, 8 bits at a time; then one pass in block
// order moves what stays: a block's new place is its place less the blocks before it that leave.  What 1024 blocks have is read
// before a barrier that precedes every write at or above their places: in place is safe.
// Bound by the latency of these dependent passes (4 x 3 barriers, then 4 per 1024 blocks and 8 heads), not by its bytes.
__global__ void __launch_bounds__(KV_EVICT_THREADS) kv_evict_kernel(const KvShape S, const KvEvict A)
{
    extern __shared__ uint32_t keys[];
    __shared__ int hist[KV_EVICT_COUNTS][256], warp_sums[32], pick[3];
    const int seq = blockIdx.x, tid = threadIdx.x;
    const int len = max(A.lens[seq], 0), most = min(A.table_stride, A.mass_stride);
    const int full = min(len >> S.block_shift, most), held = min((len + S.block_tokens - 1) >> S.block_shift, most);
    const int lo = min(A.keep_first, full), hi = max(full - A.keep_last, lo);
    const int drop = min(max(full - A.budget, 0), hi - lo);
    const float* const mass = A.mass + (int64_t)seq * S.kv_heads * A.mass_stride;
    float* const mass_out = A.mass_out + (int64_t)seq * S.kv_heads * A.mass_stride;
    auto score = [&](int b) {
        double x = 0.;
#pragma unroll 8
        for (int h = 0; h < S.kv_heads; h++) x += mass[(int64_t)h * A.mass_stride + b];
        return kv_order((float)x);
    };
    auto key = [&](int b) { return b < A.keys ? keys[b] : score(b); };
    uint32_t limit = 0;
    int ties = 0, equal = 0;                            // of the blocks with exactly the limit's score: those that leave, and all
    if (drop > 0) {
        for (int i = tid; i < KV_EVICT_COUNTS * 256; i += KV_EVICT_THREADS) hist[i >> 8][i & 255] = 0;
        __syncthreads();
        ties = drop;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int b = lo + tid; b < hi; b += KV_EVICT_THREADS) {
                const uint32_t k = shift == 24 ? score(b) : key(b);
                if (shift == 24 && b < A.keys) keys[b] = k;
                if (shift == 24 || k >> (shift + 8) == limit >> (shift + 8)) atomicAdd(&hist[tid >> 5 & (KV_EVICT_COUNTS - 1)][k >> shift & 255], 1);
            }
            __syncthreads();
            int mine = 0, upto = 0;
            if (tid < 256) {
#pragma unroll
                for (int c = 0; c < KV_EVICT_COUNTS; c++) { mine += hist[c][tid]; hist[c][tid] = 0; }
                upto = mine;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) { const int o = __shfl_up_sync(0xffffffffu, upto, d); if ((tid & 31) >= d) upto += o; }
                if ((tid & 31) == 31) warp_sums[tid >> 5] = upto;
            }
            __syncthreads();
            if (tid < 256) {
#pragma unroll
                for (int w = 0; w < 8; w++) upto += w < tid >> 5 ? warp_sums[w] : 0;
                if (upto - mine < ties && ties <= upto) { pick[0] = tid; pick[1] = ties - (upto - mine); pick[2] = mine; }
            }
            __syncthreads();
            limit |= (uint32_t)pick[0] << shift;
            ties = pick[1];
            equal = pick[2];
        }
    }
    int out_at = 0, tie_at = 0;
    for (int b0 = 0; b0 < held; b0 += KV_EVICT_THREADS) {
        const int b = b0 + tid;
        const bool free = drop > 0 && b >= lo && b < hi;
        const uint32_t k = free ? key(b) : 0u;
        const bool tie = free && k == limit;
        bool out = free && (k < limit || tie);
        int total;
        if (ties < equal) {                             // of equals the lowest places leave
            const int rank = tie_at + kv_rank(tie, warp_sums, total);
            tie_at += total;
            if (tie && rank >= ties) out = false;
        }
        const int before = out_at + kv_rank(out, warp_sums, total);
        out_at += total;
        const bool stay = b < held && !out;
        const int to = b - before;
        const int32_t page = b < held ? A.table[(int64_t)seq * A.table_stride + b] : -1;
        for (int h0 = 0; h0 < S.kv_heads; h0 += KV_EVICT_HEADS) {
            float w[KV_EVICT_HEADS];
#pragma unroll
            for (int h = 0; h < KV_EVICT_HEADS; h++) w[h] = stay && h0 + h < S.kv_heads ? mass[(int64_t)(h0 + h) * A.mass_stride + b] : 0.f;
            __syncthreads();
            if (h0 == 0) {
                if (stay) A.table_out[(int64_t)seq * A.table_stride + to] = page;
                if (out) A.evicted[(int64_t)seq * A.table_stride + before] = page;
            }
            if (stay)
#pragma unroll
                for (int h = 0; h < KV_EVICT_HEADS; h++)
                    if (h0 + h < S.kv_heads) mass_out[(int64_t)(h0 + h) * A.mass_stride + to] = w[h];
        }
    }
    __syncthreads();
    for (int b = held - drop + tid; b < A.table_stride; b += KV_EVICT_THREADS) A.table_out[(int64_t)seq * A.table_stride + b] = -1;
    for (int b = drop + tid; b < A.table_stride; b += KV_EVICT_THREADS) A.evicted[(int64_t)seq * A.table_stride + b] = -1;
    for (int b = held - drop + tid; b < A.mass_stride; b += KV_EVICT_THREADS)
        for (int h = 0; h < S.kv_heads; h++) mass_out[(int64_t)h * A.mass_stride + b] = 0.f;
    if (tid == 0) {
        A.lens_out[seq] = len - (drop << S.block_shift);
        A.n_evicted[seq] = drop;
    }
}

// ------------------------------------------------------------------------------------------------ handle ----

struct fastrack_kv {
    fastrack_kv_config config;
    KvShape shape;
    int device, num_sms;
    uint64_t* d_turns;
    PFN_cuTensorMapEncodeTiled_v12000 encode;
    std::atomic<int> last_cuda_error;
    std::atomic<uint64_t> launches;
};

// Shared memory beyond the default has to be asked for, once per kernel and device.
template <int D> static cudaError_t kv_attend_prepare()
{
    cudaError_t e = cudaSuccess;
    auto ask = [&](const void* kernel, int rows) { if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kv_attend_smem<D>(rows) + 16 * KV_WARPS); };
    ask((const void*)kv_attend_kernel<D, true, true, 1>, 8);
    ask((const void*)kv_attend_kernel<D, true, false, 1>, 8);
    ask((const void*)kv_attend_kernel<D, false, true, 1>, 8);
    ask((const void*)kv_attend_kernel<D, false, false, 1>, 8);
    ask((const void*)kv_attend_kernel<D, true, true, 2>, 16);
    ask((const void*)kv_attend_kernel<D, true, false, 2>, 16);
    ask((const void*)kv_attend_kernel<D, false, true, 2>, 16);
    ask((const void*)kv_attend_kernel<D, false, false, 2>, 16);
    auto ask_prompt = [&](const void* kernel) { if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, KvPrompt<D>::SMEM); };
    ask_prompt((const void*)kv_prompt_kernel<D, true, true>);
    ask_prompt((const void*)kv_prompt_kernel<D, true, false>);
    ask_prompt((const void*)kv_prompt_kernel<D, false, true>);
    ask_prompt((const void*)kv_prompt_kernel<D, false, false>);
    return e;
}

static int kv_cuda(fastrack_kv* kv, cudaError_t e)
{
    if (e == cudaSuccess) return FASTRACK_OK;
    kv->last_cuda_error = (int)e;
    (void)cudaGetLastError();
    return FASTRACK_ERR_CUDA;
}
static int kv_launched(fastrack_kv* kv, int count = 1)
{
    kv->launches += (uint64_t)count;
    return kv_cuda(kv, cudaGetLastError());
}
static int kv_check_device(fastrack_kv* kv)
{
    int dev = -1;
    const int rc = kv_cuda(kv, cudaGetDevice(&dev));
    return rc != FASTRACK_OK ? rc : dev == kv->device ? FASTRACK_OK : FASTRACK_ERR_ARG;
}
static bool kv_misaligned(const void* p, size_t a) { return p == nullptr || ((uintptr_t)p & (a - 1)) != 0; }
static bool kv_bad_rows(const fastrack_kv_rows* r) { return !r || kv_misaligned(r->data, 16) || (r->token_stride & 7) || (r->head_stride & 7); }
static KvRows kv_rows(const fastrack_kv_rows* r) { return {r->data, r->token_stride, r->head_stride}; }
static int kv_log2i(int x) { int s = 0; while ((1 << s) < x) s++; return s; }

static bool kv_bad_batch(const fastrack_kv* kv, const fastrack_kv_batch* b)
{
    if (!b || b->n_seqs < 0 || b->total_new < 0 || b->max_new < 0 || b->max_len < 0 || b->max_len > 1 << 30 || b->pool_pages < 0 || b->table_stride < 0) return true;
    if (b->n_seqs > 65535 || b->max_new > b->total_new || b->max_len / kv->config.block_tokens > b->table_stride) return true;
    if ((int64_t)b->max_new * kv->config.q_heads > 1 << 30 || (int64_t)b->total_new * kv->config.q_heads > INT32_MAX) return true;
    if (b->n_seqs == 0) return false;
    if (b->pool_pages > 0 && kv_misaligned(b->d_pool, 16)) return true;
    return kv_misaligned(b->d_tail, 16) || kv_misaligned(b->d_lens, 4) || kv_misaligned(b->d_starts, 4) || (b->table_stride > 0 && kv_misaligned(b->d_table, 4));
}
static KvBatch kv_batch(const fastrack_kv_batch* b)
{
    return {b->n_seqs, b->total_new, b->max_new, b->max_len, b->pool_pages, b->table_stride, (uint8_t*)b->d_pool, b->d_tail, b->d_table, b->d_lens,
            b->d_starts, b->d_positions};
}

extern "C" int fastrack_kv_create(const fastrack_kv_config* c, fastrack_kv** out)
{
    if (out) *out = nullptr;
    if (!c || !out) return FASTRACK_ERR_ARG;
    if ((c->dtype != FASTRACK_KV_BF16 && c->dtype != FASTRACK_KV_F16) || (c->format != FASTRACK_KV_INT8 && c->format != FASTRACK_KV_E4M3)) return FASTRACK_ERR_ARG;
    if (c->kv_heads < 1 || c->q_heads < 1 || c->q_heads > 1024 || c->q_heads % c->kv_heads) return FASTRACK_ERR_ARG;
    if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128) return FASTRACK_ERR_ARG;
    if (c->block_tokens != 16 && c->block_tokens != 32 && c->block_tokens != 64 && c->block_tokens != 128) return FASTRACK_ERR_ARG;
    if (c->rotary < FASTRACK_ROTARY_NONE || c->rotary > FASTRACK_ROTARY_INTERLEAVED) return FASTRACK_ERR_ARG;
    if (c->rotary == FASTRACK_ROTARY_NONE ? c->rotary_dim != 0
                                          : c->rotary_dim < 16 || c->rotary_dim > c->head_dim || c->rotary_dim % 16 || !c->frequencies || !isfinite(c->rotary_gain))
        return FASTRACK_ERR_ARG;
    if (!isfinite(c->softmax_scale) || c->softmax_scale < 0.f) return FASTRACK_ERR_ARG;
    uint64_t turns[KV_MAX_PAIRS] = {0};
    for (int i = 0; i < c->rotary_dim / 2; i++) {
        if (!isfinite(c->frequencies[i])) return FASTRACK_ERR_ARG;
        const long double t = (long double)c->frequencies[i] / 6.283185307179586476925286766559L;
        const long double part = floorl((t - floorl(t)) * 18446744073709551616.0L);
        turns[i] = part < 18446744073709551616.0L ? (uint64_t)part : 0u;
    }
    fastrack_kv* kv = new (std::nothrow) fastrack_kv();
    if (!kv) return FASTRACK_ERR_NOMEM;
    kv->config = *c;
    kv->config.frequencies = nullptr;
    kv->last_cuda_error = 0;
    kv->launches = 0;
    KvShape& S = kv->shape;
    S.q_heads = c->q_heads;
    S.kv_heads = c->kv_heads;
    S.group = c->q_heads / c->kv_heads;
    S.head_dim = c->head_dim;
    S.block_tokens = c->block_tokens;
    S.block_shift = kv_log2i(c->block_tokens);
    S.rotary = c->rotary;
    S.rotary_dim = c->rotary_dim;
    S.rotary_gain = c->rotary_gain;
    S.scale_log2 = (c->softmax_scale == 0.f ? 1.f / sqrtf((float)c->head_dim) : c->softmax_scale) * 1.4426950408889634f;
    S.codes_bytes = (uint32_t)(c->kv_heads * c->block_tokens * c->head_dim);
    S.page_bytes = (2ull * S.codes_bytes + 8ull * (uint64_t)c->kv_heads + 127) / 128 * 128;
    S.tail_values = 2ull * S.codes_bytes;
    cudaError_t e = cudaGetDevice(&kv->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&kv->num_sms, cudaDevAttrMultiProcessorCount, kv->device);
    void* encode = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (e == cudaSuccess) e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &encode, 12000, cudaEnableDefault, &found);
    if (e == cudaSuccess && (found != cudaDriverEntryPointSuccess || !encode)) e = cudaErrorNotSupported;
    kv->encode = (PFN_cuTensorMapEncodeTiled_v12000)encode;
    if (e == cudaSuccess) e = cudaMalloc(&kv->d_turns, sizeof turns);
    if (e == cudaSuccess) e = cudaMemcpy(kv->d_turns, turns, sizeof turns, cudaMemcpyHostToDevice);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kv_evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, KV_EVICT_KEYS * 4);
    if (e == cudaSuccess) e = c->head_dim == 64 ? kv_attend_prepare<64>() : c->head_dim == 96 ? kv_attend_prepare<96>() : kv_attend_prepare<128>();
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        fastrack_kv_destroy(kv);
        return e == cudaErrorMemoryAllocation ? FASTRACK_ERR_NOMEM : FASTRACK_ERR_CUDA;
    }
    S.turns = kv->d_turns;
    *out = kv;
    return FASTRACK_OK;
}

extern "C" void fastrack_kv_destroy(fastrack_kv* kv)
{
    if (!kv) return;
    if (kv->d_turns) (void)cudaFree(kv->d_turns);
    delete kv;
}

extern "C" size_t fastrack_kv_page_bytes(const fastrack_kv* kv) { return kv ? (size_t)kv->shape.page_bytes : 0; }
extern "C" size_t fastrack_kv_tail_bytes(const fastrack_kv* kv) { return kv ? (size_t)kv->shape.tail_values * 2 : 0; }
extern "C" int fastrack_kv_last_cuda_error(const fastrack_kv* kv) { return kv ? kv->last_cuda_error.load() : 0; }
extern "C" uint64_t fastrack_kv_launch_count(const fastrack_kv* kv) { return kv ? kv->launches.load() : 0; }

extern "C" int fastrack_rotary_frequencies(int rotary_dim, double base, int scaling, double factor, double original_len, double* frequencies, float* gain)
{
    const double two_pi = 6.283185307179586476925286766559;
    if (rotary_dim < 2 || (rotary_dim & 1) || !frequencies || !(base > 1) || !isfinite(base) || !(factor >= 1) || !isfinite(factor)) return FASTRACK_ERR_ARG;
    if (scaling < FASTRACK_FREQ_PLAIN || scaling > FASTRACK_FREQ_RAMP) return FASTRACK_ERR_ARG;
    if (scaling == FASTRACK_FREQ_BASE && rotary_dim < 4) return FASTRACK_ERR_ARG;
    if (scaling == FASTRACK_FREQ_RAMP && (!(original_len > 0) || !isfinite(original_len))) return FASTRACK_ERR_ARG;
    // the slowest pair has the exponent (rotary_dim - 2) / rotary_dim
    if (scaling == FASTRACK_FREQ_BASE) base *= pow(factor, (double)rotary_dim / (rotary_dim - 2));
    for (int i = 0; i < rotary_dim / 2; i++) {
        double f = pow(base, -2.0 * i / rotary_dim);
        if (scaling == FASTRACK_FREQ_LINEAR) f /= factor;
        if (scaling == FASTRACK_FREQ_RAMP) {
            const double turns = original_len * f / two_pi, keep = fmin(1.0, fmax(0.0, (turns - 1) / (32.0 - 1)));
            f = f * keep + f / factor * (1 - keep);
        }
        frequencies[i] = f;
    }
    if (gain) *gain = scaling == FASTRACK_FREQ_RAMP ? (float)(0.1 * log(factor) + 1) : 1.f;
    return FASTRACK_OK;
}

// Heads that one thread turns: as many as still leave every SM two CTAs.
static int kv_heads_per_thread(const fastrack_kv* kv, int64_t tokens, int heads)
{
    int per = 8;
    while (per > 1 && tokens * (kv->shape.head_dim / 16) * ((heads + per - 1) / per) < (int64_t)2 * KV_ROT_THREADS * kv->num_sms) per /= 2;
    return per;
}

extern "C" int fastrack_rotary(fastrack_kv* kv, int64_t tokens, int heads, const fastrack_kv_rows* in, const fastrack_kv_rows* out,
                               const int64_t* d_positions, int inverse, void* stream)
{
    if (!kv || tokens < 0 || heads < 0 || heads > 65536 || tokens > (int64_t)1 << 40) return FASTRACK_ERR_ARG;
    if (tokens == 0 || heads == 0) return FASTRACK_OK;
    if (kv_bad_rows(in) || kv_bad_rows(out) || (kv->config.rotary && kv_misaligned(d_positions, 8))) return FASTRACK_ERR_ARG;
    if (in->data == out->data && (in->token_stride != out->token_stride || in->head_stride != out->head_stride)) return FASTRACK_ERR_ARG;
    if (int rc = kv_check_device(kv)) return rc;
    const int per = kv_heads_per_thread(kv, tokens, heads);
    const int64_t threads = tokens * (kv->shape.head_dim / 16) * ((heads + per - 1) / per), ctas = (threads + KV_ROT_THREADS - 1) / KV_ROT_THREADS;
    if (ctas > INT32_MAX) return FASTRACK_ERR_ARG;
    auto kernel = kv->config.dtype == FASTRACK_KV_BF16 ? kv_rotary_kernel<true> : kv_rotary_kernel<false>;
    kernel<<<(unsigned)ctas, KV_ROT_THREADS, 0, (cudaStream_t)stream>>>(kv->shape, kv_rows(in), kv_rows(out), d_positions, tokens, heads, per, inverse != 0);
    return kv_launched(kv);
}

extern "C" int fastrack_kv_append(fastrack_kv* kv, const fastrack_kv_batch* batch, const fastrack_kv_rows* k, const fastrack_kv_rows* v,
                                  const fastrack_kv_rows* q, const fastrack_kv_rows* q_out, void* stream)
{
    if (!kv || kv_bad_batch(kv, batch) || !q != !q_out) return FASTRACK_ERR_ARG;
    if (batch->n_seqs == 0 || batch->total_new == 0 || batch->max_new == 0) return FASTRACK_OK;
    if (kv_bad_rows(k) || kv_bad_rows(v) || (q && (kv_bad_rows(q) || kv_bad_rows(q_out))) || (kv->config.rotary && kv_misaligned(batch->d_positions, 8)))
        return FASTRACK_ERR_ARG;
    if (q && q->data == q_out->data && (q->token_stride != q_out->token_stride || q->head_stride != q_out->head_stride)) return FASTRACK_ERR_ARG;
    if (int rc = kv_check_device(kv)) return rc;
    const KvShape& S = kv->shape;
    KvAppend A;
    memset(&A, 0, sizeof A);
    A.k = kv_rows(k);
    A.v = kv_rows(v);
    A.slots = (batch->max_new + S.block_tokens - 2) / S.block_tokens + 1;       // blocks that max_new tokens can touch
    const int64_t quant = (int64_t)batch->n_seqs * A.slots * S.kv_heads;
    int64_t turn = 0;
    A.q_per = 1;
    if (q) {
        A.q = kv_rows(q);
        A.q_out = kv_rows(q_out);
        A.q_per = kv_heads_per_thread(kv, batch->total_new, S.q_heads);
        turn = ((int64_t)batch->total_new * (S.head_dim / 16) * ((S.q_heads + A.q_per - 1) / A.q_per) + KV_APPEND_THREADS - 1) / KV_APPEND_THREADS;
    }
    if (quant + turn > INT32_MAX) return FASTRACK_ERR_ARG;
    A.quant_ctas = (int)quant;
    const bool bf = kv->config.dtype == FASTRACK_KV_BF16, e4 = kv->config.format == FASTRACK_KV_E4M3;
    const int each = (S.block_tokens * (S.head_dim / 16) + KV_APPEND_THREADS - 1) / KV_APPEND_THREADS;     // units per thread: 1 .. 4
    auto pick = [&](auto n) {
        constexpr int N = decltype(n)::value;
        return bf ? (e4 ? kv_append_kernel<true, true, N> : kv_append_kernel<true, false, N>) : (e4 ? kv_append_kernel<false, true, N> : kv_append_kernel<false, false, N>);
    };
    auto kernel = each == 1 ? pick(std::integral_constant<int, 1>()) : each == 2 ? pick(std::integral_constant<int, 2>()) : pick(std::integral_constant<int, 4>());
    A.spread = quant > (int64_t)kv->num_sms * (each < 4 ? 3 : 2);
    kernel<<<(unsigned)(quant + turn), KV_APPEND_THREADS, 0, (cudaStream_t)stream>>>(S, kv_batch(batch), A);
    return kv_launched(kv);
}

extern "C" int fastrack_kv_read(fastrack_kv* kv, const fastrack_kv_batch* batch, const fastrack_kv_rows* k_out, const fastrack_kv_rows* v_out, void* stream)
{
    if (!kv || kv_bad_batch(kv, batch)) return FASTRACK_ERR_ARG;
    if (batch->n_seqs == 0 || batch->max_len == 0) return FASTRACK_OK;
    if (kv_bad_rows(k_out) || kv_bad_rows(v_out)) return FASTRACK_ERR_ARG;
    if (int rc = kv_check_device(kv)) return rc;
    const KvShape& S = kv->shape;
    const int64_t x = ((int64_t)batch->max_len * (S.head_dim / 8) + 255) / 256;
    const bool bf = kv->config.dtype == FASTRACK_KV_BF16, e4 = kv->config.format == FASTRACK_KV_E4M3;
    auto kernel = bf ? (e4 ? kv_read_kernel<true, true> : kv_read_kernel<true, false>) : (e4 ? kv_read_kernel<false, true> : kv_read_kernel<false, false>);
    kernel<<<dim3((unsigned)x, 2u * S.kv_heads, batch->n_seqs), 256, 0, (cudaStream_t)stream>>>(S, kv_batch(batch), kv_rows(k_out), kv_rows(v_out));
    return kv_launched(kv);
}

// ------------------------------------------------------------------------------------------------ attention ----

#define KV_WAVES 4                      // times that chunks fill the SMs, where there is so much (61 sequences of up to 4096 tokens with weights, 4 x 131072,
                                        // 16 x 20000, 16 x 3000 .. 30000: 67, 177, 117 and 104 us; 3 times 70, 175, 116 and 107)
#define KV_CHUNK_LEAST 1024             // tokens of a chunk, where chunks fill the SMs once with more
#define KV_CHUNK_CLUSTER 2048           // tokens of a chunk in a cluster: above, more chunks than a cluster has are worth the join (where a cluster
                                        // would have less than 4 chunks, 61 sequences of up to 4096 tokens took 75 us against 67)

struct KvPlan { int rows, splits, chunk, row_tiles, units, unit_shift; size_t ml, lse2, unit_l2, total; };   // byte offsets in the workspace, part_o at 0

// Whether chunks go through the workspace
static bool kv_parts(const KvPlan& p) { return p.splits > 1 && p.chunk > 0; }

// A plan for a window needs no more of the workspace than the plan without one.
static KvPlan kv_plan(const fastrack_kv* kv, const fastrack_kv_batch* b, bool mass, int window)
{
    const KvShape& S = kv->shape;
    KvPlan p;
    const int64_t rows = (int64_t)b->max_new * S.group;
    p.rows = rows <= 8 ? 8 : rows <= 16 ? 16 : 2 * KV_P_ROWS;
    p.row_tiles = (int)((rows + p.rows - 1) / p.rows);
    const bool prompt = p.rows > 16;
    const int64_t seen = (int64_t)window + b->max_new + S.block_tokens, span = window > 0 && seen < b->max_len ? seen : b->max_len;
    const int64_t spans = (int64_t)b->n_seqs * S.kv_heads * p.row_tiles > 0 ? (int64_t)b->n_seqs * S.kv_heads * p.row_tiles : 1;
    const int64_t step = prompt ? KV_P_TOKENS : KV_STEP, most = (span + step - 1) / step;
    const int64_t room = (prompt ? 1 : 4) * (int64_t)kv->num_sms, fill = (room + spans - 1) / spans;       // chunks of a span that fill the SMs
    // chunks of a span where there is much: rounded down, since some more than fill the SMs would be a wave of their own
    const int64_t waves = KV_WAVES * room / spans > fill ? KV_WAVES * room / spans : fill;
    int64_t splits = prompt ? fill : waves < span / KV_CHUNK_LEAST ? waves : span / KV_CHUNK_LEAST > fill ? span / KV_CHUNK_LEAST : fill;
    const bool cluster = !prompt && fill >= 4 && span <= KV_CHUNK_CLUSTER * (fill < KV_CLUSTER ? fill : KV_CLUSTER);
    if (cluster) splits = fill < KV_CLUSTER ? fill : KV_CLUSTER;
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    const size_t room_for = cluster || splits < 2 ? 0 : (size_t)splits;       // grows with the span, as the chunks, rounded to steps, need not
    p.chunk = cluster ? 0 : (int)(((span + splits - 1) / splits + step - 1) / step * step);
    p.splits = cluster || p.chunk == 0 ? (int)splits : (int)((span + p.chunk - 1) / p.chunk);
    p.unit_shift = prompt ? (S.block_shift < 6 ? S.block_shift : 6) : 4;   // blocks of up to 64 tokens, or 16 tokens
    p.units = (b->max_len + (1 << p.unit_shift) - 1) >> p.unit_shift;
    const size_t all = (size_t)b->total_new * S.q_heads;
    p.ml = room_for * all * S.head_dim * 4;
    p.lse2 = p.ml + room_for * all * 8;
    p.unit_l2 = (p.lse2 + all * 4 + 15) / 16 * 16;
    p.total = p.unit_l2 + (mass ? (size_t)b->n_seqs * S.kv_heads * p.units * (size_t)rows * 4 : 0);
    return p;
}

extern "C" size_t fastrack_kv_attention_workspace(const fastrack_kv* kv, const fastrack_kv_batch* batch, int with_mass)
{
    if (!kv || kv_bad_batch(kv, batch)) return 0;
    return kv_plan(kv, batch, with_mass != 0, 0).total + 16;
}

// A launch whose start may overlap the end of the kernel before it in the stream; the kernel waits (griddepcontrol.wait) before it
// reads anything that one wrote.
template <class... P, class... Q>
static void kv_launch_after(cudaStream_t stream, dim3 grid, int threads, void (*kernel)(P...), Q... args)
{
    cudaLaunchConfig_t c = {};
    cudaLaunchAttribute overlap;
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    c.gridDim = grid;
    c.blockDim = dim3(threads);
    c.stream = stream;
    c.attrs = &overlap;
    c.numAttrs = 1;
    (void)cudaLaunchKernelEx(&c, kernel, P(args)...);    // an error stays for cudaGetLastError
}

template <int D, bool BF>
static void kv_attend_launch(const fastrack_kv* kv, const KvBatch& B, const KvAttend& A, const CUtensorMap& pool, bool parts, int weigh_tiles, cudaStream_t stream)
{
    const KvShape& S = kv->shape;
    const bool e4 = kv->config.format == FASTRACK_KV_E4M3;
    const dim3 grid(S.kv_heads * A.row_tiles, A.splits, B.n_seqs);
    if (A.rows > 16) (e4 ? kv_prompt_kernel<D, BF, true> : kv_prompt_kernel<D, BF, false>)<<<grid, KV_P_THREADS, KvPrompt<D>::SMEM, stream>>>(S, B, A);
    auto kernel = A.rows == 8 ? (e4 ? kv_attend_kernel<D, BF, true, 1> : kv_attend_kernel<D, BF, false, 1>)
                              : (e4 ? kv_attend_kernel<D, BF, true, 2> : kv_attend_kernel<D, BF, false, 2>);
    if (A.rows <= 16) {
        cudaLaunchConfig_t c = {};
        cudaLaunchAttribute cluster;
        cluster.id = cudaLaunchAttributeClusterDimension;
        cluster.val.clusterDim.y = A.chunk == 0 ? A.splits : 1;
        cluster.val.clusterDim.x = cluster.val.clusterDim.z = 1;
        c.gridDim = grid;
        c.blockDim = dim3(32 * KV_WARPS);
        c.dynamicSmemBytes = kv_attend_smem<D>(A.rows) + 16 * KV_WARPS;
        c.stream = stream;
        c.attrs = &cluster;
        c.numAttrs = 1;
        (void)cudaLaunchKernelEx(&c, kernel, S, B, A, pool);                 // an error stays for cudaGetLastError
    }
    if (parts) kv_launch_after(stream, dim3((unsigned)(B.max_new * S.q_heads + weigh_tiles * S.kv_heads), B.n_seqs), 32 * KV_WARPS, kv_join_kernel<D, BF>, S, B, A);
}

// The pool as a tensor of bytes (head_dim, rows of a page: K of all heads, then V, pages); boxes of 16 rows of one page.
static int kv_pool_map(fastrack_kv* kv, const KvBatch& B, CUtensorMap* map)
{
    const KvShape& S = kv->shape;
    memset(map, 0, sizeof *map);
    if (B.pool_pages == 0) return FASTRACK_OK;           // every page is absent
    const cuuint64_t dims[3] = {(cuuint64_t)S.head_dim, 2ull * S.kv_heads * S.block_tokens, (cuuint64_t)B.pool_pages};
    const cuuint64_t strides[2] = {(cuuint64_t)S.head_dim, S.page_bytes};
    const cuuint32_t box[3] = {(cuuint32_t)S.head_dim, KV_HALF, 1}, steps[3] = {1, 1, 1};
    const CUtensorMapSwizzle swizzle = S.head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : S.head_dim == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE;
    auto encode = [&] {
        return kv->encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, B.pool, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    };
    CUresult r = encode();
    // a thread that has made no runtime call yet has no context, which the driver's function wants: setting the device, which is current
    // by number already, makes it so
    if (r == CUDA_ERROR_INVALID_CONTEXT && kv_cuda(kv, cudaSetDevice(kv->device)) == FASTRACK_OK) r = encode();
    if (r == CUDA_SUCCESS) return FASTRACK_OK;
    kv->last_cuda_error = (int)r;
    return FASTRACK_ERR_CUDA;
}

extern "C" int fastrack_kv_attention(fastrack_kv* kv, const fastrack_kv_batch* batch, const fastrack_kv_rows* q, const fastrack_kv_rows* out, float* d_lse,
                                     int window, const float* d_mass_in, float* d_mass_out, int mass_stride, void* d_workspace, size_t workspace_bytes,
                                     void* stream)
{
    if (!kv || kv_bad_batch(kv, batch) || window < 0 || !d_mass_in != !d_mass_out) return FASTRACK_ERR_ARG;
    if (batch->n_seqs == 0 || batch->max_len == 0 && batch->total_new == 0) return FASTRACK_OK;
    const KvShape& S = kv->shape;
    if (window >= batch->max_len) window = 0;            // hides nothing; and places plus a window stay below 2^31
    const bool mass = d_mass_out != nullptr;
    if (mass && (kv_misaligned(d_mass_in, 4) || kv_misaligned(d_mass_out, 4) || mass_stride < (batch->max_len + S.block_tokens - 1) / S.block_tokens)) return FASTRACK_ERR_ARG;
    if (batch->total_new > 0 && (kv_bad_rows(q) || kv_bad_rows(out) || (d_lse && kv_misaligned(d_lse, 4)))) return FASTRACK_ERR_ARG;
    const KvPlan p = kv_plan(kv, batch, mass, window);
    if (kv_misaligned(d_workspace, 16) || workspace_bytes < p.total) return FASTRACK_ERR_ARG;
    if (int rc = kv_check_device(kv)) return rc;
    const KvBatch B = kv_batch(batch);
    KvAttend A;
    memset(&A, 0, sizeof A);
    char* const ws = (char*)d_workspace;
    A.lse = d_lse;
    A.window = window;
    A.rows = p.rows;
    A.splits = p.splits;
    A.chunk = p.chunk;
    A.row_tiles = p.row_tiles;
    A.units = p.units;
    A.part_o = (float*)ws;
    A.part_ml = (float*)(ws + p.ml);
    A.lse2 = (float*)(ws + p.lse2);
    A.unit_l2 = mass ? (float*)(ws + p.unit_l2) : nullptr;
    A.mass_in = d_mass_in;
    A.mass_out = d_mass_out;
    A.mass_stride = mass_stride;
    A.unit_shift = p.unit_shift;
    const int blocks = mass ? (batch->max_len + S.block_tokens - 1) / S.block_tokens : 0;
    const bool few = (int64_t)batch->max_new * S.group <= KV_MASS_ROWS;
    const int weigh_tiles = few ? (blocks + 32 * KV_WARPS - 1) / (32 * KV_WARPS) : 0;                          // of kv_join_kernel
    int launches = 0;
    cudaStream_t st = (cudaStream_t)stream;
    if (batch->total_new > 0 && batch->max_new > 0) {
        A.q = kv_rows(q);
        A.out = kv_rows(out);
        const bool bf = kv->config.dtype == FASTRACK_KV_BF16;
        CUtensorMap pool;
        if (int rc = kv_pool_map(kv, B, &pool)) return rc;
        switch (S.head_dim) {
        case 64: bf ? kv_attend_launch<64, true>(kv, B, A, pool, kv_parts(p), weigh_tiles, st) : kv_attend_launch<64, false>(kv, B, A, pool, kv_parts(p), weigh_tiles, st); break;
        case 96: bf ? kv_attend_launch<96, true>(kv, B, A, pool, kv_parts(p), weigh_tiles, st) : kv_attend_launch<96, false>(kv, B, A, pool, kv_parts(p), weigh_tiles, st); break;
        default: bf ? kv_attend_launch<128, true>(kv, B, A, pool, kv_parts(p), weigh_tiles, st) : kv_attend_launch<128, false>(kv, B, A, pool, kv_parts(p), weigh_tiles, st); break;
        }
        launches += 1 + kv_parts(p);
    }
    if (blocks > 0 && !(launches && kv_parts(p) && few)) {
        auto kernel = few ? kv_mass_kernel<true> : kv_mass_kernel<false>;
        const dim3 grid(few ? (blocks + 255) / 256 : blocks, S.kv_heads, batch->n_seqs);
        // it reads lengths before it waits, which this call's own kernels do not write, but one of the caller's might
        if (launches) kv_launch_after(st, grid, 256, kernel, S, B, A);
        else kernel<<<grid, 256, 0, st>>>(S, B, A);
        launches++;
    }
    return kv_launched(kv, launches);
}

extern "C" int fastrack_kv_evict(fastrack_kv* kv, const fastrack_kv_eviction* e, void* stream)
{
    if (!kv || !e || e->n_seqs < 0 || e->table_stride < 0 || e->mass_stride < 0 || e->budget < 0 || e->keep_first < 0 || e->keep_last < 0) return FASTRACK_ERR_ARG;
    if (e->n_seqs == 0) return FASTRACK_OK;
    const void* need[] = {e->d_table, e->d_lens, e->d_mass, e->d_table_out, e->d_lens_out, e->d_mass_out, e->d_evicted, e->d_n_evicted};
    for (const void* p : need) if (kv_misaligned(p, 4)) return FASTRACK_ERR_ARG;
    if (int rc = kv_check_device(kv)) return rc;
    KvEvict A;
    A.table_stride = e->table_stride;
    A.mass_stride = e->mass_stride;
    A.budget = e->budget;
    A.keep_first = e->keep_first;
    A.keep_last = e->keep_last;
    const int most = e->table_stride < e->mass_stride ? e->table_stride : e->mass_stride;
    A.keys = most < KV_EVICT_KEYS ? most : KV_EVICT_KEYS;
    A.table = e->d_table;
    A.lens = e->d_lens;
    A.mass = e->d_mass;
    A.table_out = e->d_table_out;
    A.lens_out = e->d_lens_out;
    A.mass_out = e->d_mass_out;
    A.evicted = e->d_evicted;
    A.n_evicted = e->d_n_evicted;
    cudaStream_t st = (cudaStream_t)stream;
    // 64 sequences of 4001 blocks and 8 heads: 14.3 us held in registers, 18.4 otherwise; 16 of 150: 6.9 and 8.2
    if (kv->shape.kv_heads <= KV_EVICT_HEADS && most <= 1024) kv_evict_resident_kernel<256, 4><<<e->n_seqs, 256, 0, st>>>(kv->shape, A);
    else if (kv->shape.kv_heads <= KV_EVICT_HEADS && most <= 4096) kv_evict_resident_kernel<1024, 4><<<e->n_seqs, 1024, 0, st>>>(kv->shape, A);
    else kv_evict_kernel<<<e->n_seqs, KV_EVICT_THREADS, (size_t)A.keys * 4, st>>>(kv->shape, A);
    return kv_launched(kv);
}
