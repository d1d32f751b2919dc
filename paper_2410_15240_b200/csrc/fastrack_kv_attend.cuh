// fastrack_kv_attend.cuh -- attention of few query rows over the 8-bit cache: the kernel that single tokens take.
#pragma once
#include "fastrack_kv_device.cuh"

#define KV_WARPS 4
#define KV_ROWS 16          // (query, head of the group) rows of a CTA: the M of one matrix instruction
#define KV_TILE 16          // tokens of a warp's step, inside one block
#define KV_UNIT 16          // tokens whose weight is written down together
#define KV_LAZY 4.0f        // a running maximum is raised only when exceeded by this many powers of two
// Weights enter the second product as f16, times V's scale over its reference (at most 1), times this: 2^4 * 2^11 stays below
// f16's largest, and a weight down to 2^-25 of the largest keeps all 11 bits, so that a token of little weight whose values are
// orders above the others' is not lost.
#define KV_P_SCALE 2048.0f

struct KvAttend {
    KvRows q, out;
    float* lse;             // natural, or NULL
    int window;
    int splits, chunk;      // chunks of the span, tokens of a chunk (a multiple of the block)
    int row_tiles, units;   // units: per sequence, for weights
    float* part_o;          // [splits][total_new * q_heads][head_dim]
    float* part_ml;         // [splits][total_new * q_heads][2]
    float* lse2;            // [total_new * q_heads], base 2
    float* unit_l2;         // [n_seqs][kv_heads][units][max_new * group]: log2 of the sum of exponentials of a unit; NULL without weights
    const float* mass_in;
    float* mass_out;
    int mass_stride;
};

__device__ __forceinline__ float kv_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float kv_log2(float x)
{
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void kv_mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Two codes as two f16, exactly: of bytes J and K of the eight in (lo, hi).
//   int8: 0x64 in front of a byte u is the f16 number 1024 + u; with the code's sign bit flipped u = code + 128, so that
//         subtracting 1152 leaves the code.
//   e4m3: sign, exponent and fraction moved to their places in an f16, which has 8 more in its exponent bias: code * 2^-8.
//         Exact for subnormal codes too.  No code becomes a NaN.  The 2^8 is made good in the scale (KV_CODE_SCALE).
template <bool E4M3, int J, int K> __device__ __forceinline__ uint32_t kv_two(uint32_t lo, uint32_t hi)
{
    if (E4M3) {
        const uint32_t p = __byte_perm(lo, hi, J << 4 | K << 12);
        return (p & 0x80008000u) | ((p >> 1) & 0x3f803f80u);
    }
    const uint32_t p = (__byte_perm(lo, hi, J | K << 8) & 0x00ff00ffu) ^ 0x64806480u;
    const __half2 h = __hsub2(*(const __half2*)&p, __half2half2(__ushort_as_half(0x6480)));
    return *(const uint32_t*)&h;
}
template <bool E4M3> __device__ __forceinline__ float kv_code_scale() { return E4M3 ? 256.f : 1.f; }

// 2^e with 2^e <= x < 2^(e+1) for finite x > 0 (1 for zero, the largest for what is not finite): dividing by it is exact.
__device__ __forceinline__ float kv_power_below(uint32_t abs_bits)
{
    uint32_t e = abs_bits >> 23;
    if (abs_bits == 0) return 1.f;
    e = e < 2u ? 2u : e > 252u ? 252u : e;
    return __uint_as_float(e << 23);
}

// An infinite scale counts as NaN, so that a block with one shows in every answer that sees it.
__device__ __forceinline__ float kv_finite(float x) { return fabsf(x) < KV_INF ? x : __int_as_float(0x7fffffff); }

// One CTA: 16 rows of one kv head of one sequence, one chunk of the tokens they see.  Each of the four warps takes every fourth
// tile of 16 tokens with statistics and an accumulator of its own; they are joined in shared memory at the end.
//
// In the matrix instructions the channels that a lane holds are permuted so that what it needs of K is 16 (8 at 96 channels)
// bytes in a row of one token, and of V head_dim / 8 bytes in a row of four tokens: codes go from memory to registers in whole
// sectors, are widened there and enter the product, without passing through shared memory.
template <int D, bool BF, bool E4M3>
__global__ void __launch_bounds__(32 * KV_WARPS) kv_attend_kernel(const KvShape S, const KvBatch B, const KvAttend A)
{
    constexpr int PB = D % 64 == 0 ? 16 : 8, PW = PB / 4, STEPS = D / 16, NT = D / 8, VW = D / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    const int chunk = blockIdx.x, kh = blockIdx.y % S.kv_heads, tile_row = blockIdx.y / S.kv_heads * KV_ROWS, seq = blockIdx.z;
    const KvSeq q = kv_seq(S, B, seq);
    const KvSpan span = kv_span(S, q, A.window, tile_row, KV_ROWS);
    if (tile_row >= q.n * S.group) return;
    const int begin = span.begin + chunk * A.chunk, end = min(span.end, begin + A.chunk);
    if (begin >= end && chunk > 0) return;

    // queries: two rows per lane, as f16; a bf16 row is first divided by a power of two near its largest magnitude
    uint32_t qa[STEPS][4];
    float row_scale[2];
    int place[2];                                       // where the row's query stands; -1 for rows behind the last
#pragma unroll
    for (int r = 0; r < 2; r++) {
        const int row = tile_row + g + 8 * r;
        const bool valid = row < q.n * S.group;
        const int token = row / S.group, head = kh * S.group + row % S.group;
        place[r] = valid ? q.len - q.n + token : -1;
        const uint16_t* src = (const uint16_t*)A.q.data + (q.start + token) * A.q.token_stride + head * A.q.head_stride;
        uint2 raw[STEPS];
        uint32_t amax = 0;
#pragma unroll
        for (int s = 0; s < STEPS; s++) {
            raw[s] = valid ? *(const uint2*)(src + ((s / PW) * 4 + c) * PB + (s % PW) * 4) : make_uint2(0, 0);
            if (BF) {
                amax = max(amax, max(raw[s].x << 16 & 0x7fffffffu, raw[s].x & 0x7fff0000u));
                amax = max(amax, max(raw[s].y << 16 & 0x7fffffffu, raw[s].y & 0x7fff0000u));
            }
        }
        float p = 1.f;
        if (BF) {
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            p = kv_power_below(amax);
        }
        row_scale[r] = p * S.scale_log2 * kv_code_scale<E4M3>();
        const float inv = 1.f / p;
#pragma unroll
        for (int s = 0; s < STEPS; s++) {
            if (BF) {
                const float2 x = kv_unpack<true>(raw[s].x), y = kv_unpack<true>(raw[s].y);
                qa[s][r] = kv_pack<false>(x.x * inv, x.y * inv);
                qa[s][2 + r] = kv_pack<false>(y.x * inv, y.y * inv);
            } else {
                qa[s][r] = raw[s].x;
                qa[s][2 + r] = raw[s].y;
            }
        }
    }
    const int last_row = min(tile_row + KV_ROWS, q.n * S.group) - 1;
    const int see_all = q.len - q.n + tile_row / S.group;                    // tokens up to here are seen by every row (without a window)
    const int low_all = A.window > 0 ? q.len - q.n + last_row / S.group - A.window : -1;   // tokens behind here are in every row's window

    float o[NT][4];
#pragma unroll
    for (int i = 0; i < NT; i++) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m[2] = {-KV_INF, -KV_INF}, l[2] = {0.f, 0.f};
    float vref = 0.f;                                    // power of two that V's scales are measured by: o is in its units

    for (int t0 = begin + KV_TILE * warp; t0 < end; t0 += KV_TILE * KV_WARPS) {
        const int block = t0 >> S.block_shift, at = t0 & (S.block_tokens - 1);
        const bool tail = block == q.full;
        uint32_t kb[2][STEPS][2], vb[NT][2];
        float ks, vs;
        if (!tail) {
            const int page = kv_page(B, seq, block);
            if (page < 0) continue;
            const float2 sc = *(const float2*)(kv_scales(S, B, page) + 2 * kh);
            ks = kv_finite(sc.x);
            vs = kv_finite(sc.y);
            const uint8_t* kp = B.pool + (uint64_t)page * S.page_bytes + ((uint64_t)kh * S.block_tokens + at) * D;
            const uint8_t* vp = kp + S.codes_bytes;
            uint32_t kw[2][STEPS], vw[4][VW];
#pragma unroll
            for (int nt = 0; nt < 2; nt++)
#pragma unroll
                for (int p = 0; p < STEPS / PW; p++) {
                    const uint8_t* src = kp + (8 * nt + g) * D + (p * 4 + c) * PB;
                    if (PB == 16) *(uint4*)&kw[nt][p * PW] = __ldg((const uint4*)src);
                    else *(uint2*)&kw[nt][p * PW] = __ldg((const uint2*)src);
                }
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const uint8_t* src = vp + (2 * c + (j & 1) + (j >> 1) * 8) * D + g * (D / 8);
                if (VW == 4) *(uint4*)vw[j] = __ldg((const uint4*)src);
                else if (VW == 2) *(uint2*)vw[j] = __ldg((const uint2*)src);
                else
#pragma unroll
                    for (int w = 0; w < VW; w++) vw[j][w] = __ldg((const uint32_t*)src + w);
            }
#pragma unroll
            for (int nt = 0; nt < 2; nt++)
#pragma unroll
                for (int s = 0; s < STEPS; s++) {
                    kb[nt][s][0] = kv_two<E4M3, 0, 1>(kw[nt][s], 0);
                    kb[nt][s][1] = kv_two<E4M3, 2, 3>(kw[nt][s], 0);
                }
#pragma unroll
            for (int w = 0; w < VW; w++) {
                vb[4 * w][0] = kv_two<E4M3, 0, 4>(vw[0][w], vw[1][w]); vb[4 * w][1] = kv_two<E4M3, 0, 4>(vw[2][w], vw[3][w]);
                vb[4 * w + 1][0] = kv_two<E4M3, 1, 5>(vw[0][w], vw[1][w]); vb[4 * w + 1][1] = kv_two<E4M3, 1, 5>(vw[2][w], vw[3][w]);
                vb[4 * w + 2][0] = kv_two<E4M3, 2, 6>(vw[0][w], vw[1][w]); vb[4 * w + 2][1] = kv_two<E4M3, 2, 6>(vw[2][w], vw[3][w]);
                vb[4 * w + 3][0] = kv_two<E4M3, 3, 7>(vw[0][w], vw[1][w]); vb[4 * w + 3][1] = kv_two<E4M3, 3, 7>(vw[2][w], vw[3][w]);
            }
        } else {
            // the unfinished block: 16-bit values, tokens behind the last as zeros; bf16 goes to f16 by a power of two near the tile's largest
            const uint16_t* kp = (const uint16_t*)B.tail + (uint64_t)seq * S.tail_values + ((uint64_t)kh * 2 * S.block_tokens + at) * D;
            const uint16_t* vp = kp + (uint64_t)S.block_tokens * D;
            uint32_t kmax = 0, vmax = 0, raw[4][NT / 2];
#pragma unroll
            for (int nt = 0; nt < 2; nt++)
#pragma unroll
                for (int s = 0; s < STEPS; s++) {
                    const bool there = t0 + 8 * nt + g < q.len;
                    const uint2 w = there ? *(const uint2*)(kp + (8 * nt + g) * D + ((s / PW) * 4 + c) * PB + (s % PW) * 4) : make_uint2(0, 0);
                    kb[nt][s][0] = w.x;
                    kb[nt][s][1] = w.y;
                    if (BF) {
                        kmax = max(kmax, max(w.x << 16 & 0x7fffffffu, w.x & 0x7fff0000u));
                        kmax = max(kmax, max(w.y << 16 & 0x7fffffffu, w.y & 0x7fff0000u));
                    }
                }
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int t = 2 * c + (j & 1) + (j >> 1) * 8;
#pragma unroll
                for (int i = 0; i < NT / 2; i++) {
                    raw[j][i] = t0 + t < q.len ? *(const uint32_t*)(vp + t * D + g * (D / 8) + 2 * i) : 0u;
                    if (BF) vmax = max(vmax, max(raw[j][i] << 16 & 0x7fffffffu, raw[j][i] & 0x7fff0000u));
                }
            }
            float kp2 = 1.f, vp2 = 1.f;
            if (BF) {
                kp2 = kv_power_below(__reduce_max_sync(0xffffffffu, kmax));
                vp2 = kv_power_below(__reduce_max_sync(0xffffffffu, vmax));
                const float ki = 1.f / kp2, vi = 1.f / vp2;
#pragma unroll
                for (int nt = 0; nt < 2; nt++)
#pragma unroll
                    for (int s = 0; s < STEPS; s++)
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            const float2 x = kv_unpack<true>(kb[nt][s][h]);
                            kb[nt][s][h] = kv_pack<false>(x.x * ki, x.y * ki);
                        }
#pragma unroll
                for (int j = 0; j < 4; j++)
#pragma unroll
                    for (int i = 0; i < NT / 2; i++) {
                        const float2 x = kv_unpack<true>(raw[j][i]);
                        raw[j][i] = kv_pack<false>(x.x * vi, x.y * vi);
                    }
            }
#pragma unroll
            for (int i = 0; i < NT / 2; i++)
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    vb[2 * i][h] = __byte_perm(raw[2 * h][i], raw[2 * h + 1][i], 0x5410);
                    vb[2 * i + 1][h] = __byte_perm(raw[2 * h][i], raw[2 * h + 1][i], 0x7632);
                }
            ks = kp2 / kv_code_scale<E4M3>();
            vs = vp2 / kv_code_scale<E4M3>();
        }

        float s[2][4];
#pragma unroll
        for (int nt = 0; nt < 2; nt++) {
            s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
            for (int k = 0; k < STEPS; k++) kv_mma(s[nt], qa[k], kb[nt][k][0], kb[nt][k][1]);
#pragma unroll
            for (int e = 0; e < 4; e++) s[nt][e] *= ks * row_scale[e >> 1];
        }
        const bool ragged = t0 + KV_TILE - 1 > see_all || t0 <= low_all;
        if (ragged) {
#pragma unroll
            for (int nt = 0; nt < 2; nt++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int t = t0 + 8 * nt + 2 * c + (e & 1), at_row = place[e >> 1];
                    if (t > at_row || (A.window > 0 && t <= at_row - A.window)) s[nt][e] = -KV_INF;
                }
        }
        float top[2] = {fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1])), fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]))};
        if (__any_sync(0xffffffffu, top[0] > m[0] + KV_LAZY || top[1] > m[1] + KV_LAZY)) {
#pragma unroll
            for (int r = 0; r < 2; r++) {
                top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
                top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
                const float higher = fmaxf(m[r], top[r]);
                const float f = higher == -KV_INF ? 1.f : kv_exp2(m[r] - higher);
                m[r] = higher;
                l[r] *= f;
#pragma unroll
                for (int i = 0; i < NT; i++) { o[i][2 * r] *= f; o[i][2 * r + 1] *= f; }
            }
        }
        if (vs > vref) {                // the warp as a whole: vs is the tile's
            const float higher = 4.f * kv_power_below(__float_as_uint(vs));
            const float f = vref / higher;
#pragma unroll
            for (int i = 0; i < NT; i++) { o[i][0] *= f; o[i][1] *= f; o[i][2] *= f; o[i][3] *= f; }
            vref = higher;
        }
        const float vf = vref > 0.f ? vs / vref * KV_P_SCALE : vs;
        const float base[2] = {m[0] == -KV_INF ? 0.f : m[0], m[1] == -KV_INF ? 0.f : m[1]};
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int nt = 0; nt < 2; nt++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const bool hidden = ragged && s[nt][e] == -KV_INF;       // so that a masked token's scale, whatever it is, does not count
                const float p = kv_exp2(s[nt][e] - base[e >> 1]);
                sum[e >> 1] += p;
                s[nt][e] = hidden ? 0.f : p * vf;
            }
        l[0] += sum[0];
        l[1] += sum[1];
        if (A.unit_l2) {
#pragma unroll
            for (int r = 0; r < 2; r++) {
                sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], 1);
                sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], 2);
                const int row = tile_row + g + 8 * r;
                if (c == 0 && row < q.n * S.group)
                    A.unit_l2[(((int64_t)seq * S.kv_heads + kh) * A.units + t0 / KV_UNIT) * (B.max_new * S.group) + row] = kv_log2(sum[r]) + base[r];
            }
        }
        const uint32_t pa[4] = {kv_pack<false>(s[0][0], s[0][1]), kv_pack<false>(s[0][2], s[0][3]), kv_pack<false>(s[1][0], s[1][1]),
                                kv_pack<false>(s[1][2], s[1][3])};
#pragma unroll
        for (int i = 0; i < NT; i++) kv_mma(o[i], pa, vb[i][0], vb[i][1]);
    }

    // join the warps
    __shared__ float sm_o[KV_WARPS][KV_ROWS][D + 4], sm_m[KV_WARPS][KV_ROWS], sm_l[KV_WARPS][KV_ROWS];
#pragma unroll
    for (int r = 0; r < 2; r++) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        if (c == 0) { sm_m[warp][g + 8 * r] = m[r]; sm_l[warp][g + 8 * r] = l[r]; }
        const float unit = vref > 0.f ? vref * (kv_code_scale<E4M3>() / KV_P_SCALE) : 1.f;   // without a reference o is 0 or NaN
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
            for (int e = 0; e < 2; e++) sm_o[warp][g + 8 * r][(2 * c + e) * (D / 8) + i] = o[i][2 * r + e] * unit;
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < KV_ROWS * (D / 2); idx += 32 * KV_WARPS) {
        const int row = idx / (D / 2), ch = idx % (D / 2) * 2, all = tile_row + row;
        if (all >= q.n * S.group) break;
        float top = -KV_INF;
#pragma unroll
        for (int w = 0; w < KV_WARPS; w++) top = fmaxf(top, sm_m[w][row]);
        const float base = top == -KV_INF ? 0.f : top;
        float x = 0.f, y = 0.f, sum = 0.f;
#pragma unroll
        for (int w = 0; w < KV_WARPS; w++) {
            const float f = kv_exp2(sm_m[w][row] - base);
            sum += f * sm_l[w][row];
            x += f * sm_o[w][row][ch];
            y += f * sm_o[w][row][ch + 1];
        }
        const int64_t token = q.start + all / S.group;
        const int head = kh * S.group + all % S.group;
        if (A.splits == 1) {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            *(uint32_t*)((uint16_t*)A.out.data + token * A.out.token_stride + head * A.out.head_stride + ch) = kv_pack<BF>(x * inv, y * inv);
            if (ch == 0) {
                const float l2 = sum == 0.f ? -KV_INF : base + log2f(sum);
                if (A.lse) A.lse[token * S.q_heads + head] = l2 * 0.6931471805599453f;
                A.lse2[token * S.q_heads + head] = l2;
            }
        } else {
            const int64_t at = ((int64_t)chunk * B.total_new + token) * S.q_heads + head;
            *(float2*)(A.part_o + at * D + ch) = make_float2(x, y);
            if (ch == 0) *(float2*)(A.part_ml + 2 * at) = make_float2(top, sum);
        }
    }
}

// Joins the chunks of each row: a warp per row.
template <int D, bool BF>
__global__ void __launch_bounds__(256) kv_join_kernel(const KvShape S, const KvBatch B, const KvAttend A, const int rows_per_tile)
{
    constexpr int V = D / 32;
    const int lane = threadIdx.x & 31, seq = blockIdx.y, idx = blockIdx.x * 8 + (threadIdx.x >> 5);
    const KvSeq q = kv_seq(S, B, seq);
    if (idx >= q.n * S.q_heads) return;
    const int token = idx / S.q_heads, head = idx % S.q_heads;
    const int row = token * S.group + head % S.group;
    const KvSpan span = kv_span(S, q, A.window, row / rows_per_tile * rows_per_tile, rows_per_tile);
    const int chunks = max(1, (span.end - span.begin + A.chunk - 1) / A.chunk);
    const int64_t first = (int64_t)(q.start + token) * S.q_heads + head, step = (int64_t)B.total_new * S.q_heads;
    float m = -KV_INF, l = 0.f, acc[V];
#pragma unroll
    for (int i = 0; i < V; i++) acc[i] = 0.f;
    for (int k = 0; k < chunks; k++) {
        const float2 ml = *(const float2*)(A.part_ml + 2 * (first + k * step));
        const float* src = A.part_o + (first + k * step) * D + lane * V;
        const float top = fmaxf(m, ml.x), base = top == -KV_INF ? 0.f : top, f = kv_exp2(m - base), h = kv_exp2(ml.x - base);
        m = top;
        l = l * f + ml.y * h;
#pragma unroll
        for (int i = 0; i < V; i++) acc[i] = acc[i] * f + src[i] * h;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* dst = (uint16_t*)A.out.data + (q.start + token) * A.out.token_stride + head * A.out.head_stride + lane * V;
#pragma unroll
    for (int i = 0; i < V; i++) dst[i] = (uint16_t)kv_pack<BF>(acc[i] * inv, 0.f);
    if (lane == 0) {
        const float l2 = l == 0.f ? -KV_INF : m + log2f(l);
        if (A.lse) A.lse[first] = l2 * 0.6931471805599453f;
        A.lse2[first] = l2;
    }
}

// Weight of each block: a warp per block adds exp2(log2 of the unit's sum - log2 of the row's sum) over the block's units and the
// rows that see any of it, in an order of its own that never changes.
__global__ void __launch_bounds__(256) kv_mass_kernel(const KvShape S, const KvBatch B, const KvAttend A, const int unit_shift)
{
    const int lane = threadIdx.x & 31, block = blockIdx.x * 8 + (threadIdx.x >> 5), kh = blockIdx.y, seq = blockIdx.z;
    const KvSeq q = kv_seq(S, B, seq);
    if (block << S.block_shift >= q.len) return;
    const int rows = q.n * S.group, stride = B.max_new * S.group;
    const int unit0 = block << S.block_shift >> unit_shift, unit1 = (min((block + 1) << S.block_shift, q.len) - 1 >> unit_shift) + 1;
    float sum = 0.f;
    if (block == q.full || kv_page(B, seq, block) >= 0)
        for (int unit = unit0; unit < unit1; unit++) {
            const float* src = A.unit_l2 + (((int64_t)seq * S.kv_heads + kh) * A.units + unit) * stride;
            const int t0 = unit << unit_shift, t1 = t0 + (1 << unit_shift) - 1;
            for (int row = lane; row < rows; row += 32) {
                const int token = row / S.group, place = q.len - q.n + token;
                if (t0 > place || (A.window > 0 && t1 <= place - A.window)) continue;
                sum += kv_exp2(src[row] - A.lse2[(int64_t)(q.start + token) * S.q_heads + kh * S.group + row % S.group]);
            }
        }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) {
        const int64_t at = ((int64_t)seq * S.kv_heads + kh) * A.mass_stride + block;
        A.mass_out[at] = A.mass_in[at] + sum;
    }
}
