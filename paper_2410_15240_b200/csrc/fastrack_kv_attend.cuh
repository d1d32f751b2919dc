// fastrack_kv_attend.cuh -- attention of few query rows over the 8-bit cache: the kernel that single tokens take.
#pragma once
#include <cuda.h>
#include "fastrack_kv_device.cuh"

#define KV_WARPS 4
#define KV_HALF 16          // tokens that lie inside one block for sure
#define KV_TILE 32          // tokens of a warp's step: two halves
// What a token adds to the answer is exp2(s) * (V's scale) * (V's codes), s its score in base 2.  With y = log2 of V's scale, its weight
// enters the second product as f16 exp2(s + y - m), m the row's reference: s + y of every token that the row has seen is at most
// m + KV_P_MOST, which f16 holds.  Where one is above, m is raised to KV_P_BITS below it, and what was added up falls.  So what adds down to
// 2^-25 of the largest share keeps all 11 bits, whatever the scales of blocks that the row sees and of others.
// The sum of exponentials wants the weights without V's scale: the sum of every 16 tokens with one scale is multiplied by
// z = 2^-KV_L_BITS / scale.  The answer's accumulator is in units of 2^m, the sum l in units of 2^(m + KV_L_BITS): for scales from
// 2^-109 (append's smallest) to 2^121 neither z nor l of 2^30 tokens leaves the range of a float.  (An exponential that ends
// below 2^-126 is lost to the sum: that takes tokens of one row whose scales are 2^137 apart.)
#define KV_P_MOST 15.0f
#define KV_P_BITS 11.0f
#define KV_L_BITS 27.0f
#define KV_M_NONE -3.402823466e38f      // the reference of a row that has seen nothing: finite, so that a difference from it is a number
// The power of two that zeros are taken to be held over, in a page (scale 0) or in the unfinished block: they add nothing to any answer, but their
// weights count in the sum.  Low enough to leave other blocks' weights their bits, high enough for the sum beside large ones.
#define KV_V_ZERO 0x1p-72f

// Every span is cut into chunks, a CTA for each.  Where the chunks fill the SMs several times, they are equal pieces of whatever length
// a sequence has, so that one CTA's start and end pass under the others' loads; they are joined through the workspace by a kernel of its
// own.  Where there is less than the SMs hold, a span is cut into up to KV_CLUSTER equal chunks, whose CTAs are a cluster and join
// their answers through each other's shared memory.  (One sequence of 700 tokens: 9.2 us in a cluster, 10.4 us with the join's
// launch; 61 sequences of up to 4096: 75 and 67 us, because the CTAs of short sequences wait for nothing in a cluster's place.
// Tried instead: CTAs that stay and take equal runs of one line of all work; all of them start and end at the same time, 148 us.)
#define KV_CLUSTER 8
#define KV_STEP (KV_TILE * KV_WARPS)

struct KvAttend {
    KvRows q, out;
    float* lse;             // natural, or NULL
    int window;
    int rows;               // of a CTA: 8, 16 or 256
    int splits;             // most chunks of a span
    int chunk;              // tokens of a chunk; 0: the chunks of a span are a cluster and equal
    int row_tiles, units;   // units: per sequence, for weights, of
    int unit_shift;         // log2 of their tokens
    float* part_o;          // [splits][total_new * q_heads][head_dim]
    float* part_ml;         // [splits][total_new * q_heads][2]: m and l, see KV_P_MOST
    float* lse2;            // [total_new * q_heads], base 2, see kv_lse2_at
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
__device__ __forceinline__ void kv_mma(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t* b)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ uint32_t kv_transpose(uint32_t x)                 // an 8 x 8 matrix of f16 held by the warp
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// Codes as pairs of f16, exactly.
//   e4m3: every code is an f16 number; there is an instruction that widens two.
//   int8: 0x64 in front of a byte u is the f16 number 1024 + u; with the code's sign bit flipped u = code + 128, so that
//         subtracting 1152 leaves the code.
__device__ __forceinline__ uint32_t kv_widen_e4m3(uint32_t two)
{
    uint32_t d;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(d) : "r"(two));
    return d;
}
__device__ __forceinline__ uint32_t kv_minus_1152(uint32_t p)
{
    const __half2 h = __hsub2(*(const __half2*)&p, __half2half2(__ushort_as_half(0x6480)));
    return *(const uint32_t*)&h;
}
// bytes (0, 1) and (2, 3) of w
template <bool E4M3> __device__ __forceinline__ void kv_widen4(uint32_t w, uint32_t& b0, uint32_t& b1)
{
    if (E4M3) {
        b0 = kv_widen_e4m3(w);
        b1 = kv_widen_e4m3(w >> 16);
    } else {
        const uint32_t u = w ^ 0x80808080u;
        b0 = kv_minus_1152(__byte_perm(u, 0x64646464u, 0x4140));
        b1 = kv_minus_1152(__byte_perm(u, 0x64646464u, 0x4342));
    }
}
// byte i of w and of x, for i = 0 .. 3
template <bool E4M3> __device__ __forceinline__ void kv_widen_pairs(uint32_t w, uint32_t x, uint32_t* d)
{
    const uint32_t lo = __byte_perm(w, x, 0x5140), hi = __byte_perm(w, x, 0x7362);
    kv_widen4<E4M3>(lo, d[0], d[1]);
    kv_widen4<E4M3>(hi, d[2], d[3]);
}

// 16 rows of head_dim bytes from the pool, as tensor (head_dim, rows of a page, pages), to shared memory
__device__ __forceinline__ void kv_tma(uint32_t smem, const CUtensorMap* map, int row, int page, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(smem), "l"(map), "r"(0), "r"(row), "r"(page), "r"(bar) : "memory");
}
// Whether the barrier's phase of this parity has ended, after waiting for it a bounded number of times (each attempt gives up by
// itself after a while; in practice the first or second succeeds).
__device__ __forceinline__ bool kv_wait(uint32_t bar, uint32_t parity)
{
    uint32_t done = 0;
    for (int attempt = 0; attempt < 1 << 16 && !done; attempt++)
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}

__device__ __forceinline__ void kv_cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The same place in the shared memory of the cluster's CTA `rank`
__device__ __forceinline__ float2 kv_peer_load(const float2* p, int rank)
{
    uint32_t at;
    float2 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
    return v;
}

// 2^e with 2^e <= x < 2^(e+1) for finite x > 0 (1 for zero, the largest for what is not finite): dividing by it is exact.
__device__ __forceinline__ float kv_power_below(uint32_t abs_bits)
{
    uint32_t e = abs_bits >> 23;
    if (abs_bits == 0) return 1.f;
    e = e < 2u ? 2u : e > 252u ? 252u : e;
    return __uint_as_float(e << 23);
}

// V of the unfinished block is held over a power of two of at least this, which is what a page's smallest values are: a reference of
// that power still has an inverse, V below it keeps its bits down to 2^-124, and zeros do not take any from pages.
#define KV_V_LEAST 0x1p-100f

// y and z of a scale of V (see KV_P_MOST); NaN for NaN.  The exponent is taken off the logarithm's argument: y is as exact as its size
// allows, 2^-21 at most, and the sum sees the weights as the answer does.
__device__ __forceinline__ float2 kv_v_share(float scale)
{
    const float v = scale < 0x1p-110f ? KV_V_ZERO : scale;
    const uint32_t bits = __float_as_uint(v);
    const float exponent = __uint_as_float(0x4b000000u | bits >> 23) - (8388608.f + 127.f);
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(v));
    return make_float2(fmaf(v, 0.f, exponent + kv_log2(__uint_as_float((bits & 0x7fffffu) | 0x3f800000u))), inv * (1.f / 134217728));
}
// What an accumulated answer is multiplied by, for the sum l of its row: 2^-KV_L_BITS / l; 0 where the row saw nothing.
__device__ __forceinline__ float kv_over_sum(float l)
{
    const float inv = 1.f / (l < 1.f ? l * 134217728.f : l);                 // of a sum whose inverse is a float
    return l == 0.f ? 0.f : l < 1.f ? inv : inv * (1.f / 134217728);
}

// Of a power of two that one of these gave: its inverse, and y and z of V held over it
__device__ __forceinline__ float kv_power_inverse(float p) { return __uint_as_float(0x7f000000u - __float_as_uint(p)); }
__device__ __forceinline__ float2 kv_power_share(float p)
{
    return make_float2((float)((int)(__float_as_uint(p) >> 23) - 127), kv_power_inverse(p) * (1.f / 134217728));
}

// The power of two that V is held over, for values of at most this size (finite)
__device__ __forceinline__ float kv_v_power(float amax) { return amax == 0.f ? KV_V_ZERO : fmaxf(kv_power_below(__float_as_uint(amax)), KV_V_LEAST); }

// The larger of two 16-bit numbers, twice
__device__ __forceinline__ uint32_t kv_max2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// The largest magnitude of 8 values, as the bits of a float (bf16) or of an f16: 16-bit magnitudes are in the order of their bits
template <bool BF> __device__ __forceinline__ uint32_t kv_amax8(const uint4& w)
{
    const uint32_t m = 0x7fff7fffu, a = kv_max2(kv_max2(w.x & m, w.y & m), kv_max2(w.z & m, w.w & m)), most = max(a & 0xffffu, a >> 16);
    return BF ? most << 16 : most;
}

// Where a row's sum stands in lse2: the rows of a sequence and kv head are neighbours.
__device__ __forceinline__ int64_t kv_lse2_at(const KvShape& S, const KvSeq& q, int kh, int row)
{
    return ((int64_t)q.start * S.kv_heads + (int64_t)kh * q.n) * S.group + row;
}

// An infinite scale counts as NaN, so that a block with one shows in every answer that sees it.
__device__ __forceinline__ float kv_finite(float x) { return fabsf(x) < KV_INF ? x : __int_as_float(0x7fffffff); }

// How a warp computes 16 tokens.  K and V take the side of the matrix instruction m16n8k16 that is 16 wide, and the rows, of which a
// single token has few, the side of 8:
//     S^T[16 tokens, 8 rows] += K[16 tokens, 16 channels] q^T,     O^T[16 channels, 8 rows] += V^T[16 channels, 16 tokens] P^T.
// The channels may be permuted at will (those of q and of the answer alike), and so may the tokens of a half; both are, so that a
// lane's share of K and V is made of whole runs of bytes and is read from shared memory without bank conflicts:
//     K: lane (g, c) holds, of tokens token(g) and token(g) + 8, every fourth run of KB bytes from run c on;
//     V: of tokens token(2c), token(2c+1), token(2c) + 8, token(2c+1) + 8, head_dim / 8 bytes: 8 or 16 in a row, at 96 channels 8 and 4.
// The codes come by tensor copies, which turn the 16-byte pieces of a row around by the row's number (at 64 and 128 channels; a row of 96
// bytes needs none): with token(g) = 0 5 2 7 4 1 6 3 the eight lanes of a phase read eight different pieces.
// A warp has room for one tile: the next tile's K is sent for as soon as this one's is read, its V likewise, so that half a tile or
// more is on its way at any time; with 16 warps that is more than the 35 KB that an SM needs in flight, and the room that
// further stages would take goes to warps.
template <int D> struct KvTile {
    static constexpr int KB = D % 64 == 0 ? 16 : 8, KRUNS = D / (4 * KB);
    static constexpr int STEPS = D / 16;                                     // of QK^T along the channels, and tiles of 16 channels of O
    static constexpr int VW = D / 32;                                        // words of V per token and lane
    static constexpr int BYTES = KV_HALF * D;                                // K, or V, of a half
    static constexpr int STAGE = (4 * BYTES + 1023) / 1024 * 1024;           // K of both halves, V of both
    __device__ static int k_channel(int step, int c) { return ((step * 4 / KB) * 4 + c) * KB + step * 4 % KB; }
    __device__ static int v_channel(int g, int i) { return D != 96 ? g * (D / 8) + i : i < 8 ? 8 * g + i : 64 + 4 * g + i - 8; }
    __device__ static int token(int g) { return (g & 6) ^ ((g & 1) * 5); }
    // byte `at` (in a piece of 16 that does not cross) of a row
    __device__ static int place(int row, int at)
    {
        return row * D + (D == 128 ? at ^ (row & 7) << 4 : D == 64 ? at ^ (row >> 1 & 3) << 4 : at);
    }
};

template <int D> __host__ __device__ constexpr int kv_attend_smem(int rows)
{
    const int tiles = KV_WARPS * KvTile<D>::STAGE, join = KV_WARPS * rows * (D + 4) * 4 + KV_WARPS * rows * 8 + rows * 8;
    return tiles > join ? tiles : join;                                      // and 16 bytes of barriers per warp behind
}

// What a warp carries along its tokens.
template <int D, int NR> struct KvState {
    uint32_t qb[NR][D / 16][2];                          // queries as f16: row 8 r + g
    float factor[NR][2];                                 // of the scores of rows 8 r + 2 c + e
    float m[NR][2], l[NR][2];                            // see KV_P_MOST
    float o[NR][D / 16][4];                              // in units of 2^m
};

// s + y of scores and V's scales, -inf where hidden: raises the rows' references where one is exceeded and turns them into weights (unrounded).
template <int D, int NR, int HALVES>
__device__ __forceinline__ void kv_weigh(KvState<D, NR>& W, float (&s)[HALVES][NR][4])
{
    bool higher = false;
    float base[NR][2];
#pragma unroll
    for (int r = 0; r < NR; r++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
            float top = fmaxf(s[0][r][e], s[0][r][2 + e]);
            if (HALVES == 2) top = fmaxf(top, fmaxf(s[HALVES - 1][r][e], s[HALVES - 1][r][2 + e]));
            base[r][e] = top;
            higher |= top - W.m[r][e] > KV_P_MOST;       // exact, however large the two are
        }
    if (__any_sync(0xffffffffu, higher)) {
#pragma unroll
        for (int r = 0; r < NR; r++)
#pragma unroll
            for (int e = 0; e < 2; e++) {
                float top = base[r][e];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                top = fmaxf(W.m[r][e], __fadd_ru(top, -KV_P_BITS));          // up: what is rounded away would be above KV_P_MOST
                const float f = kv_exp2(W.m[r][e] - top);
                W.m[r][e] = top;
                W.l[r][e] *= f;
#pragma unroll
                for (int i = 0; i < D / 16; i++) { W.o[r][i][e] *= f; W.o[r][i][2 + e] *= f; }
            }
    }
#pragma unroll
    for (int r = 0; r < NR; r++)
#pragma unroll
        for (int e = 0; e < 2; e++)
#pragma unroll
            for (int h = 0; h < HALVES; h++) {
                s[h][r][e] = kv_exp2(s[h][r][e] - W.m[r][e]);
                s[h][r][2 + e] = kv_exp2(s[h][r][2 + e] - W.m[r][e]);
            }
}

// log2 of a row's sum of exponentials; and of a unit's, made for every tile, by the unit's instruction, which is off by at most 2^-22 of a
// logarithm of some 10 (the library's function took 15 us of the 315 of 3 x 1024 new tokens, 3 of the 67 of 61 single ones).
__device__ __forceinline__ float kv_sum_log2(float l, float m) { return l == 0.f ? -KV_INF : m + (KV_L_BITS + log2f(l)); }
__device__ __forceinline__ float kv_unit_log2(float l, float m) { return m + (KV_L_BITS - 16.f + kv_log2(l * 65536.f)); }    // no part of l is a denormal number then

// log2 of the rows' sums of exponentials of halves h0 .. h1 - 1, from the lanes' parts of l, to out[row]
template <int NR, int HALVES>
__device__ __forceinline__ void kv_note(const float (&part)[HALVES][NR][2], const float (&m)[NR][2], int h0, int h1, float* out, int rows_left, int g, int c)
{
#pragma unroll
    for (int r = 0; r < NR; r++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
            float sum = 0.f;
#pragma unroll
            for (int h = 0; h < HALVES; h++)
                if (h >= h0 && h < h1) sum += part[h][r][e];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            const int at = 8 * r + 2 * c + e;
            if (g == 0 && at < rows_left) out[at] = kv_unit_log2(sum, m[r][e]);
        }
}

// Weights of two rows as f16, as the second operand's share of a lane.  FINE (answers of 11 bits, where the rounding of the weights
// would show as much as that of the answer): what the rounding leaves out as another such number, which gets a product of its own.
// Answers of 8 bits do without: a weight's rounding, 2^-12 and of either sign, is an eighth of the answer's own even before it averages out
// over the tokens (error against 64 bits 0.0017 of the answer, as that of 32-bit weights).
template <bool FINE> __device__ __forceinline__ void kv_weights(float x, float y, uint32_t& hi, uint32_t& lo)
{
    hi = kv_pack<false>(x, y);
    if (FINE) {
        const float2 z = kv_unpack<false>(hi);
        lo = kv_transpose(kv_pack<false>(x - z.x, y - z.y));
    }
    hi = kv_transpose(hi);
}

// One tile of full blocks.  RAGGED: some of its tokens are hidden from some rows, or a half is not there.
// k_wait and v_wait wait for K and V, k_read and v_read are called when they have been read.
template <int D, bool FINE, bool E4M3, int NR, bool RAGGED, class KWait, class KRead, class VWait, class VRead>
__device__ __forceinline__ void kv_tile(KvState<D, NR>& W, const uint8_t* slot, int t0, const float (&ks)[2], const float (&vs)[2], const bool (&there)[2],
                                        const int (&place)[NR][2], int window, float* unit_out, int unit_stride, bool one_unit, int rows_left, int lane,
                                        KWait k_wait, KRead k_read, VWait v_wait, VRead v_read)
{
    using T = KvTile<D>;
    const int g = lane >> 2, c = lane & 3, token = T::token(g);
    float s[2][NR][4];
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
        for (int r = 0; r < NR; r++) s[h][r][0] = s[h][r][1] = s[h][r][2] = s[h][r][3] = 0.f;
    bool fine = k_wait();
#pragma unroll
    for (int p = 0; p < T::KRUNS; p++)
#pragma unroll
        for (int h = 0; h < 2; h++) {
            uint32_t w[2][T::KB / 4];
#pragma unroll
            for (int up = 0; up < 2; up++) {
                const uint8_t* const src = slot + h * T::BYTES + T::place(8 * up + token, (p * 4 + c) * T::KB);
                if (T::KB == 16) *(uint4*)w[up] = *(const uint4*)src;
                else *(uint2*)w[up] = *(const uint2*)src;
            }
#pragma unroll
            for (int i = 0; i < T::KB / 4; i++) {
                uint32_t a[4];
                kv_widen4<E4M3>(w[0][i], a[0], a[2]);
                kv_widen4<E4M3>(w[1][i], a[1], a[3]);
#pragma unroll
                for (int r = 0; r < NR; r++) kv_mma(s[h][r], a[0], a[1], a[2], a[3], W.qb[r][p * (T::KB / 4) + i]);
            }
        }
    k_read();
    const float2 share[2] = {kv_v_share(vs[0]), kv_v_share(vs[1])};
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
        for (int r = 0; r < NR; r++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                s[h][r][i] = fmaf(s[h][r][i], ks[h] * W.factor[r][i & 1], share[h].x);
                if (RAGGED) {                            // a masked token's scales, whatever they are, do not count
                    const int t = t0 + KV_HALF * h + 8 * (i >> 1) + token, at = place[r][i & 1];
                    if (t > at || (window > 0 && t <= at - window) || !there[h]) s[h][r][i] = -KV_INF;
                }
            }
    float part[2][NR][2];
    kv_weigh<D, NR, 2>(W, s);
#pragma unroll
    for (int r = 0; r < NR; r++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const float sum = s[h][r][e] + s[h][r][2 + e];
                part[h][r][e] = RAGGED && sum == 0.f ? 0.f : sum * share[h].y;
            }
            W.l[r][e] += part[0][r][e] + part[1][r][e];
        }
    if (unit_out) {
        if (one_unit) kv_note<NR, 2>(part, W.m, 0, 2, unit_out, rows_left, g, c);
        else {
            kv_note<NR, 2>(part, W.m, 0, 1, unit_out, rows_left, g, c);
            if (there[1]) kv_note<NR, 2>(part, W.m, 1, 2, unit_out + unit_stride, rows_left, g, c);
        }
    }
    fine = v_wait() && fine;
    if (!fine)                                           // bytes that never came: NaN answers
#pragma unroll
        for (int r = 0; r < NR; r++) W.l[r][0] = W.l[r][1] = __int_as_float(0x7fffffff);
#pragma unroll
    for (int h = 0; h < 2; h++) {
        uint32_t pb[NR][2], pl[NR][2];
#pragma unroll
        for (int r = 0; r < NR; r++)
#pragma unroll
            for (int up = 0; up < 2; up++) kv_weights<FINE>(s[h][r][2 * up], s[h][r][2 * up + 1], pb[r][up], pl[r][up]);
        uint32_t vw[4][T::VW];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint8_t* const src = slot + (2 + h) * T::BYTES;
            const int row = T::token(2 * c + (j & 1)) + 8 * (j >> 1);
            if (D == 128) *(uint4*)vw[j] = *(const uint4*)(src + T::place(row, 16 * g));
            else *(uint2*)vw[j] = *(const uint2*)(src + T::place(row, 8 * g));
            if (D == 96) vw[j][T::VW - 1] = *(const uint32_t*)(src + T::place(row, 64 + 4 * g));
            if (RAGGED && !there[h])
#pragma unroll
                for (int w = 0; w < T::VW; w++) vw[j][w] = 0u;
        }
#pragma unroll
        for (int w = 0; w < T::VW; w++) {
            uint32_t a[4], b[4];
            kv_widen_pairs<E4M3>(vw[0][w], vw[1][w], a);
            kv_widen_pairs<E4M3>(vw[2][w], vw[3][w], b);
#pragma unroll
            for (int r = 0; r < NR; r++) {
                kv_mma(W.o[r][2 * w], a[0], a[1], b[0], b[1], pb[r]);
                kv_mma(W.o[r][2 * w + 1], a[2], a[3], b[2], b[3], pb[r]);
                if (FINE) {
                    kv_mma(W.o[r][2 * w], a[0], a[1], b[0], b[1], pl[r]);
                    kv_mma(W.o[r][2 * w + 1], a[2], a[3], b[2], b[3], pl[r]);
                }
            }
        }
    }
    v_read();
}

// 16 tokens of the unfinished block: 16-bit values, tokens behind the last as zeros.  V, and bf16 K, go to f16 over a power of two near the token's
// largest value, so that no token, whatever it holds, reaches a row that does not see it.  What is not finite in V stays out of the product (a
// weight of 0 would not hide it there) and is added for the rows that see the token.
template <int D, bool BF, int NR>
__device__ __forceinline__ void kv_tail_tile(KvState<D, NR>& W, const uint16_t* k, const uint16_t* v, int t0, int len, const int (&place)[NR][2], int window,
                                             float* unit_out, int rows_left, int lane)
{
    using T = KvTile<D>;
    constexpr int STEPS = D / 16;
    const int g = lane >> 2, c = lane & 3;
    auto amax2 = [](uint32_t a, uint32_t w) { return max(a, max(w << 16 & 0x7fffffffu, w & 0x7fff0000u)); };
    auto narrow = [](uint32_t w, float inv) {
        if (!BF) return w;
        const float2 x = kv_unpack<true>(w);
        return kv_pack<false>(x.x * inv, x.y * inv);
    };
    float s[1][NR][4];
#pragma unroll
    for (int r = 0; r < NR; r++) s[0][r][0] = s[0][r][1] = s[0][r][2] = s[0][r][3] = 0.f;
    float k_scale[2] = {1.f, 1.f};                       // of tokens g and g + 8
    {
        uint2 lo[STEPS], hi[STEPS];
        uint32_t amax[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < STEPS; i++) {
            lo[i] = t0 + g < len ? *(const uint2*)(k + g * D + T::k_channel(i, c)) : make_uint2(0, 0);
            hi[i] = t0 + 8 + g < len ? *(const uint2*)(k + (8 + g) * D + T::k_channel(i, c)) : make_uint2(0, 0);
        }
        if (BF) {
#pragma unroll
            for (int i = 0; i < STEPS; i++) {
                amax[0] = amax2(amax2(amax[0], lo[i].x), lo[i].y);
                amax[1] = amax2(amax2(amax[1], hi[i].x), hi[i].y);
            }
#pragma unroll
            for (int up = 0; up < 2; up++) {
                amax[up] = max(amax[up], __shfl_xor_sync(0xffffffffu, amax[up], 1));
                amax[up] = max(amax[up], __shfl_xor_sync(0xffffffffu, amax[up], 2));
                k_scale[up] = kv_power_below(amax[up]);
            }
        }
        const float inv[2] = {kv_power_inverse(k_scale[0]), kv_power_inverse(k_scale[1])};
#pragma unroll
        for (int i = 0; i < STEPS; i++) {
            const uint32_t a0 = narrow(lo[i].x, inv[0]), a1 = narrow(hi[i].x, inv[1]), a2 = narrow(lo[i].y, inv[0]), a3 = narrow(hi[i].y, inv[1]);
#pragma unroll
            for (int r = 0; r < NR; r++) kv_mma(s[0][r], a0, a1, a2, a3, W.qb[r][i]);
        }
    }
    uint32_t w[STEPS][4];                                // V of tokens 2c, 2c+1, 2c+8, 2c+9, two channels each: on their way meanwhile
#pragma unroll
    for (int i = 0; i < STEPS; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int t = 2 * c + (j & 1) + (j >> 1) * 8;
            w[i][j] = t0 + t < len ? *(const uint32_t*)(v + t * D + T::v_channel(g, 2 * i)) : 0u;
        }
    // the tokens' largest magnitudes as 16 bits: low and high half of sizes[u] of tokens 8 u + 2 c and 8 u + 2 c + 1
    constexpr uint32_t INFINITE = BF ? 0x7f80u : 0x7c00u;
    uint32_t sizes[2], odd = 0;                          // odd: tokens with values that are not finite
    auto measure = [&] {
#pragma unroll
        for (int u = 0; u < 2; u++) {
            uint32_t a[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < STEPS; i++)
#pragma unroll
                for (int k = 0; k < 2; k++) a[k] = kv_max2(a[k], w[i][2 * u + k] & 0x7fff7fffu);
            sizes[u] = max(a[0] & 0xffffu, a[0] >> 16) | max(a[1] & 0xffffu, a[1] >> 16) << 16;
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) sizes[u] = kv_max2(sizes[u], __shfl_xor_sync(0xffffffffu, sizes[u], d));
        }
    };
    measure();
    const uint32_t both = kv_max2(sizes[0], sizes[1]);
    if (__any_sync(0xffffffffu, (both & 0xffffu) >= INFINITE || both >> 16 >= INFINITE)) {
#pragma unroll
        for (int u = 0; u < 2; u++) odd |= ((sizes[u] & 0xffffu) >= INFINITE ? 1u : 0u) << (8 * u + 2 * c) | (sizes[u] >> 16 >= INFINITE ? 2u : 0u) << (8 * u + 2 * c);
        odd = __reduce_or_sync(0xffffffffu, odd);
#pragma unroll
        for (int i = 0; i < STEPS; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                if ((w[i][j] & 0x7fffu) >= INFINITE) w[i][j] &= 0xffff0000u;
                if ((w[i][j] >> 16 & 0x7fffu) >= INFINITE) w[i][j] &= 0xffffu;
            }
        measure();
    }
    auto power = [](uint32_t size) { return kv_v_power(BF ? __uint_as_float(size << 16) : __half2float(__ushort_as_half((unsigned short)size))); };
    float2 share[2];                                     // of tokens g and g + 8
    float inv[4];                                        // of the tokens of w
#pragma unroll
    for (int u = 0; u < 2; u++) {
        const uint32_t two = __shfl_sync(0xffffffffu, sizes[u], g >> 1);
        share[u] = kv_power_share(power(g & 1 ? two >> 16 : two & 0xffffu));
        inv[2 * u] = kv_power_inverse(power(sizes[u] & 0xffffu));
        inv[2 * u + 1] = kv_power_inverse(power(sizes[u] >> 16));
    }
#pragma unroll
    for (int r = 0; r < NR; r++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            s[0][r][i] = fmaf(s[0][r][i] * k_scale[i >> 1], W.factor[r][i & 1], share[i >> 1].x);
            const int t = t0 + 8 * (i >> 1) + g, at = place[r][i & 1];
            if (t > at || (window > 0 && t <= at - window)) s[0][r][i] = -KV_INF;
        }
    kv_weigh<D, NR, 1>(W, s);
    float part[1][NR][2];
#pragma unroll
    for (int r = 0; r < NR; r++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
            part[0][r][e] = s[0][r][e] * share[0].y + s[0][r][2 + e] * share[1].y;
            W.l[r][e] += part[0][r][e];
        }
    if (unit_out) kv_note<NR, 1>(part, W.m, 0, 1, unit_out, rows_left, g, c);
    uint32_t pb[NR][2], pl[NR][2];
#pragma unroll
    for (int r = 0; r < NR; r++)
#pragma unroll
        for (int up = 0; up < 2; up++)
            kv_weights<!BF>(s[0][r][2 * up], s[0][r][2 * up + 1], pb[r][up], pl[r][up]);
#pragma unroll
    for (int i = 0; i < STEPS; i++) {
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const float2 x = kv_unpack<BF>(w[i][j]);
            w[i][j] = kv_pack<false>(x.x * inv[j], x.y * inv[j]);
        }
        const uint32_t a0 = __byte_perm(w[i][0], w[i][1], 0x5410), a1 = __byte_perm(w[i][0], w[i][1], 0x7632), a2 = __byte_perm(w[i][2], w[i][3], 0x5410),
                       a3 = __byte_perm(w[i][2], w[i][3], 0x7632);
#pragma unroll
        for (int r = 0; r < NR; r++) {
            kv_mma(W.o[r][i], a0, a1, a2, a3, pb[r]);
            if (!BF) kv_mma(W.o[r][i], a0, a1, a2, a3, pl[r]);
        }
    }
    if (odd == 0) return;
    auto not_finite = [](float x) { return fabsf(x) < KV_INF ? 0.f : x; };
#pragma unroll 1
    for (int t = 0; t < KV_HALF; t++) {
        if (!(odd >> t & 1)) continue;
#pragma unroll
        for (int i = 0; i < STEPS; i++) {
            const float2 x = kv_unpack<BF>(*(const uint32_t*)(v + t * D + T::v_channel(g, 2 * i)));
#pragma unroll
            for (int r = 0; r < NR; r++)
#pragma unroll
                for (int e = 0; e < 2; e++)
                    if (t0 + t <= place[r][e] && (window == 0 || t0 + t > place[r][e] - window)) {
                        W.o[r][i][e] += not_finite(x.x);
                        W.o[r][i][2 + e] += not_finite(x.y);
                    }
        }
    }
}

// One CTA: 8 NR rows of one kv head of one sequence, one chunk of the tokens they see.  Each of the four warps takes every fourth
// tile with statistics and an accumulator of its own; they are joined in shared memory at the end.
// Bound by the codes' way from memory: 4 sequences of up to 131072 tokens (int8, f16 queries with their second product, 913 MB) in 159 us,
// 5.8 TB/s; next to it stands the widening (56 % of the ALU's cycles, 0.65 instructions a cycle and scheduler).  What it came from, with
// bf16 queries: codes loaded straight to registers by a warp, rows on the 16-wide side of the instruction 372 us; copies lane by lane
// into a ring 342; K and V on the 16-wide side 236; 32 tokens a step and a path without masks 211; tensor copies, which free the lanes of
// addresses and waits, 160.  A reference for V's scales apart from the maximum of the scores took f16 queries 176 us.
template <int D, bool BF, bool E4M3, int NR>
__global__ void __launch_bounds__(32 * KV_WARPS, NR == 1 ? (D == 64 ? 6 : 4) : 3) kv_attend_kernel(const KvShape S, const KvBatch B, const KvAttend A,
                                                                                  const __grid_constant__ CUtensorMap pool)
{
    using T = KvTile<D>;
    constexpr int STEPS = T::STEPS, ROWS = 8 * NR;
    extern __shared__ __align__(1024) uint8_t kv_smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    const int chunk = blockIdx.y, kh = blockIdx.x % S.kv_heads, tile_row = blockIdx.x / S.kv_heads * ROWS, seq = blockIdx.z;
    asm volatile("griddepcontrol.launch_dependents;");   // the join may take its place; it waits for this kernel's end
    const KvSeq q = kv_seq(S, B, seq);
    const KvSpan span = kv_span(S, q, A.window, tile_row, ROWS);
    const int rows = q.n * S.group;
    if (tile_row >= rows) return;                        // the cluster as a whole
    const int size = A.chunk ? A.chunk : (max((span.end - span.begin + A.splits - 1) / A.splits, 1) + KV_STEP - 1) / KV_STEP * KV_STEP, begin = span.begin + chunk * size, end = min(span.end, begin + size);
    const bool cluster = A.chunk == 0 && A.splits > 1;
    if (begin >= end && chunk > 0 && !cluster) return;

    // tiles begin + 32 (warp + 4 i) of full blocks; a half behind the last full block, or on an absent page, is not there
    uint8_t* const slot = kv_smem + warp * T::STAGE;
    const uint32_t slot_at = (uint32_t)__cvta_generic_to_shared(slot), bars = (uint32_t)__cvta_generic_to_shared(kv_smem + kv_attend_smem<D>(ROWS) + 16 * warp);
    const int tail_begin = q.full << S.block_shift, full_end = min(end, tail_begin);
    const int32_t* const table = B.table + (int64_t)seq * B.table_stride;
    if (lane == 0) {
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars) : "memory");
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars + 8) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    auto page_of = [&](int t) {
        const int b = t >> S.block_shift, p = t < full_end && b < B.table_stride ? __ldg(table + b) : -1;
        return p < B.pool_pages ? p : -1;
    };
    // K (which = 0) or V (1) of the tile: lane 0 sends for the halves that are there; the barrier's phase ends when they have arrived
    auto fetch = [&](int which, int t0, int2 pages) {
        if (lane == 0 && t0 < full_end) {
            const uint32_t bar = bars + 8 * which, at = slot_at + 2 * which * T::BYTES;
            const int row = (which * S.kv_heads + kh) * S.block_tokens, bytes = ((pages.x >= 0) + (pages.y >= 0)) * T::BYTES;
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
            if (pages.x >= 0) kv_tma(at, &pool, row + (t0 & (S.block_tokens - 1)), pages.x, bar);
            if (pages.y >= 0) kv_tma(at + T::BYTES, &pool, row + ((t0 + KV_HALF) & (S.block_tokens - 1)), pages.y, bar);
        }
    };
    auto scales_of = [&](int page) { return page >= 0 ? __ldg((const float2*)(kv_scales(S, B, page) + 2 * kh)) : make_float2(0.f, 0.f); };
    constexpr int STRIDE = KV_TILE * KV_WARPS;
    const int first = begin + KV_TILE * warp;
    int2 pages = make_int2(page_of(first), page_of(first + KV_HALF)), next = make_int2(page_of(first + STRIDE), page_of(first + STRIDE + KV_HALF));
    fetch(0, first, pages);
    fetch(1, first, pages);
    float2 scale[2] = {scales_of(pages.x), scales_of(pages.y)};

    // queries: row g (and g + 8) of a lane, as f16; a bf16 row is first divided by a power of two near its largest magnitude.  The
    // products come out with rows 2c and 2c + 1 in a lane: their factors and places.
    KvState<D, NR> W;
    int place[NR][2];
#pragma unroll
    for (int r = 0; r < NR; r++) {
        const int row = tile_row + 8 * r + g;
        const bool valid = row < rows;
        const uint16_t* src = (const uint16_t*)A.q.data + (q.start + row / S.group) * A.q.token_stride + (kh * S.group + row % S.group) * A.q.head_stride;
        uint32_t amax = 0;
#pragma unroll
        for (int s = 0; s < STEPS; s++) {
            const uint2 raw = valid ? *(const uint2*)(src + T::k_channel(s, c)) : make_uint2(0, 0);
            W.qb[r][s][0] = raw.x;
            W.qb[r][s][1] = raw.y;
            if (BF) {
                amax = max(amax, max(raw.x << 16 & 0x7fffffffu, raw.x & 0x7fff0000u));
                amax = max(amax, max(raw.y << 16 & 0x7fffffffu, raw.y & 0x7fff0000u));
            }
        }
        float p = 1.f;
        if (BF) {
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            p = kv_power_below(amax);
            const float inv = kv_power_inverse(p);
#pragma unroll
            for (int s = 0; s < STEPS; s++)
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const float2 x = kv_unpack<true>(W.qb[r][s][h]);
                    W.qb[r][s][h] = kv_pack<false>(x.x * inv, x.y * inv);
                }
        }
#pragma unroll
        for (int e = 0; e < 2; e++) {
            const int mine = tile_row + 8 * r + 2 * c + e;
            W.factor[r][e] = S.scale_log2 * __shfl_sync(0xffffffffu, p, 4 * (2 * c + e));
            place[r][e] = mine < rows ? q.len - q.n + mine / S.group : -1;
            W.m[r][e] = KV_M_NONE;
            W.l[r][e] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < STEPS; i++) W.o[r][i][0] = W.o[r][i][1] = W.o[r][i][2] = W.o[r][i][3] = 0.f;
    }
    const int last_row = min(tile_row + ROWS, rows) - 1;
    const int see_all = q.len - q.n + tile_row / S.group;                    // tokens up to here are seen by every row (without a window)
    const int low_all = A.window > 0 ? q.len - q.n + last_row / S.group - A.window : -1;   // tokens behind here are in every row's window
    const int unit_stride = B.max_new * S.group;
    float* const units = A.unit_l2 ? A.unit_l2 + ((int64_t)seq * S.kv_heads + kh) * A.units * unit_stride + tile_row : nullptr;
    const bool one_unit = S.block_tokens >= KV_TILE;

    // the tail first: its loads pass while the first tiles come; by the last warps, which have a tile less where their number is not a multiple of four
    // (61 sequences of up to 4096 tokens 66.2 us, by the first warps 66.9)
    const uint16_t* const tail_k = (const uint16_t*)B.tail + (uint64_t)seq * S.tail_values + (uint64_t)kh * 2 * S.block_tokens * D;
    for (int t0 = max(begin, tail_begin) + KV_HALF * (KV_WARPS - 1 - warp); t0 < end; t0 += KV_HALF * KV_WARPS)
        kv_tail_tile<D, BF, NR>(W, tail_k + (t0 - tail_begin) * D, tail_k + (S.block_tokens + t0 - tail_begin) * D, t0, q.len, place, A.window,
                                units ? units + (int64_t)(t0 / KV_HALF) * unit_stride : nullptr, rows - tile_row, lane);

    uint32_t phase = 0;
    for (int t0 = first; t0 < full_end; t0 += STRIDE) {
        float* const unit_out = units ? units + (int64_t)(t0 / KV_HALF) * unit_stride : nullptr;
        const bool there[2] = {pages.x >= 0, pages.y >= 0};
        const float ks[2] = {kv_finite(scale[0].x), kv_finite(scale[1].x)}, vs[2] = {kv_finite(scale[0].y), kv_finite(scale[1].y)};
        auto k_wait = [&] { return kv_wait(bars, phase); };
        auto k_read = [&] { __syncwarp(); fetch(0, t0 + STRIDE, pages); };
        auto v_wait = [&] { return kv_wait(bars + 8, phase); };
        auto v_read = [&] { __syncwarp(); fetch(1, t0 + STRIDE, pages); };
        pages = next;
        scale[0] = scales_of(pages.x);
        scale[1] = scales_of(pages.y);
        next = make_int2(page_of(t0 + 2 * STRIDE), page_of(t0 + 2 * STRIDE + KV_HALF));
        if (t0 + KV_TILE - 1 <= see_all && t0 > low_all && there[0] && there[1])
            kv_tile<D, !BF, E4M3, NR, false>(W, slot, t0, ks, vs, there, place, A.window, unit_out, unit_stride, one_unit, rows - tile_row, lane, k_wait, k_read, v_wait, v_read);
        else
            kv_tile<D, !BF, E4M3, NR, true>(W, slot, t0, ks, vs, there, place, A.window, unit_out, unit_stride, one_unit, rows - tile_row, lane, k_wait, k_read, v_wait, v_read);
        phase ^= 1;
    }
    // join the warps, in the tiles' memory
    __syncthreads();
    float (*const sm_o)[ROWS][D + 4] = (float (*)[ROWS][D + 4])kv_smem;
    float (*const sm_m)[ROWS] = (float (*)[ROWS])(kv_smem + KV_WARPS * ROWS * (D + 4) * 4);
    float (*const sm_l)[ROWS] = sm_m + KV_WARPS;
#pragma unroll
    for (int r = 0; r < NR; r++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
            const int row = 8 * r + 2 * c + e;
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) W.l[r][e] += __shfl_xor_sync(0xffffffffu, W.l[r][e], d);
            if (g == 0) { sm_m[warp][row] = W.m[r][e]; sm_l[warp][row] = W.l[r][e]; }
#pragma unroll
            for (int i = 0; i < STEPS; i++) {
                sm_o[warp][row][T::v_channel(g, 2 * i)] = W.o[r][i][e];
                sm_o[warp][row][T::v_channel(g, 2 * i + 1)] = W.o[r][i][2 + e];
            }
        }
    __syncthreads();
    // A chunk's answer: rows' maxima and sums, and o relative to the maximum, over the first warp's (a thread reads what it writes over).
    float2* const sm_ml = (float2*)(sm_l + KV_WARPS);
    auto answer = [&](int row, int ch, float top, float sum, float x, float y) {
        const int all = tile_row + row, head = kh * S.group + all % S.group;
        const int64_t token = q.start + all / S.group;
        const float inv = kv_over_sum(sum);
        *(uint32_t*)((uint16_t*)A.out.data + token * A.out.token_stride + head * A.out.head_stride + ch) = kv_pack<BF>(x * inv, y * inv);
        if (ch == 0) {
            const float l2 = kv_sum_log2(sum, top);
            if (A.lse) A.lse[token * S.q_heads + head] = l2 * 0.6931471805599453f;
            A.lse2[kv_lse2_at(S, q, kh, all)] = l2;
        }
    };
    for (int idx = threadIdx.x; idx < ROWS * (D / 2); idx += 32 * KV_WARPS) {
        const int row = idx / (D / 2), ch = idx % (D / 2) * 2, all = tile_row + row;
        if (all >= rows) break;
        float top = sm_m[0][row];
#pragma unroll
        for (int w = 1; w < KV_WARPS; w++) top = fmaxf(top, sm_m[w][row]);
        float x = 0.f, y = 0.f, sum = 0.f;
#pragma unroll
        for (int w = 0; w < KV_WARPS; w++) {
            const float f = kv_exp2(sm_m[w][row] - top);
            sum += f * sm_l[w][row];
            x += f * sm_o[w][row][ch];
            y += f * sm_o[w][row][ch + 1];
        }
        if (A.splits == 1) {
            answer(row, ch, top, sum, x, y);
        } else if (cluster) {
            *(float2*)&sm_o[0][row][ch] = make_float2(x, y);
            if (ch == 0) sm_ml[row] = make_float2(top, sum);
        } else {
            const int64_t at = ((int64_t)chunk * B.total_new + q.start + all / S.group) * S.q_heads + kh * S.group + all % S.group;
            *(float2*)(A.part_o + at * D + ch) = make_float2(x, y);
            if (ch == 0) *(float2*)(A.part_ml + 2 * at) = make_float2(top, sum);
        }
    }
    if (!cluster) return;
    // every CTA of the cluster joins its share of the answers
    kv_cluster_sync();
    for (int idx = chunk * 32 * KV_WARPS + threadIdx.x; idx < ROWS * (D / 2); idx += A.splits * 32 * KV_WARPS) {
        const int row = idx / (D / 2), ch = idx % (D / 2) * 2;
        if (tile_row + row >= rows) break;
        float2 ml[KV_CLUSTER], o[KV_CLUSTER];
        float top = -KV_INF;
#pragma unroll
        for (int k = 0; k < KV_CLUSTER; k++) {
            ml[k] = k < A.splits ? kv_peer_load(&sm_ml[row], k) : make_float2(-KV_INF, 0.f);
            o[k] = k < A.splits ? kv_peer_load((const float2*)&sm_o[0][row][ch], k) : make_float2(0.f, 0.f);
        }
#pragma unroll
        for (int k = 0; k < KV_CLUSTER; k++) top = fmaxf(top, ml[k].x);
        float x = 0.f, y = 0.f, sum = 0.f;
#pragma unroll
        for (int k = 0; k < KV_CLUSTER; k++) {
            const float f = kv_exp2(ml[k].x - top);
            sum += f * ml[k].y;
            x += f * o[k].x;
            y += f * o[k].y;
        }
        answer(row, ch, top, sum, x, y);
    }
    kv_cluster_sync();                                   // nobody leaves while others read its memory
}

// Sum over a block's units and the rows that see any of one of exp2(log2 of the unit's sum - log2 of the row's sum): the block's weight.
// A thread takes every EVERY-th row from its first.
template <int EVERY, int UNROLL>
__device__ __forceinline__ float kv_block_weight(const KvShape& S, const KvBatch& B, const KvAttend& A, const KvSeq& q, int seq, int kh, int block, int first, const float* l2)
{
    const int stride = B.max_new * S.group;
    const int unit0 = block << S.block_shift >> A.unit_shift, unit1 = (min((block + 1) << S.block_shift, q.len) - 1 >> A.unit_shift) + 1;
    const int step = A.unit_shift == 4 && block < q.full && S.block_tokens >= KV_TILE ? KV_TILE / KV_HALF : 1; // of kv_attend_kernel's full blocks: a sum per tile
    float sum = 0.f;
    if (block < q.full && kv_page(B, seq, block) < 0) return sum;
    for (int unit = unit0; unit < unit1; unit += step) {
        const float* src = A.unit_l2 + (((int64_t)seq * S.kv_heads + kh) * A.units + unit) * stride;
        const int t0 = unit << A.unit_shift, t1 = t0 + (step << A.unit_shift) - 1;
        // the first token whose query sees the unit at all, and the last that has it in its window
        const int lo = max(t0 - (q.len - q.n), 0), hi = A.window > 0 ? min(q.n - 1, t1 - (q.len - q.n) + A.window - 1) : q.n - 1;
#pragma unroll UNROLL
        for (int row = lo * S.group + first; row < (hi + 1) * S.group; row += EVERY) sum += kv_exp2(src[row] - l2[row]);
    }
    return sum;
}

// One kv head's blocks from first_block on, one to a thread, after `sums` has log2 of each row's sum.
__device__ __forceinline__ void kv_weigh_blocks(const KvShape& S, const KvBatch& B, const KvAttend& A, const KvSeq& q, int seq, int kh, int first_block, const float* sums)
{
    const int block = first_block + threadIdx.x;
    if (block << S.block_shift >= q.len) return;
    const int64_t at = ((int64_t)seq * S.kv_heads + kh) * A.mass_stride + block;
    A.mass_out[at] = A.mass_in[at] + kv_block_weight<1, 4>(S, B, A, q, seq, kh, block, 0, sums);
}

#define KV_MASS_ROWS 32                                  // rows per sequence and kv head up to which a thread weighs a block

// Joins the chunks of each row: a CTA per row, of which a warp takes every fourth chunk.  With few rows CTAs behind these weigh blocks:
// each works out the rows' sums again, a half warp to a row, instead of a launch that waits for them (4 sequences of up to 131072
// tokens 180.4 us in all, 181.6 with it; 61 of up to 4096 67.0, 68.1).
template <int D, bool BF>
__global__ void __launch_bounds__(32 * KV_WARPS) kv_join_kernel(const KvShape S, const KvBatch B, const KvAttend A)
{
    constexpr int V = D / 32;
    __shared__ float sm_acc[KV_WARPS][D], sm_sum[KV_WARPS], sm_rows[KV_MASS_ROWS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, seq = blockIdx.y;
    const int joins = B.max_new * S.q_heads;
    asm volatile("griddepcontrol.launch_dependents;");
    const KvSeq q = kv_seq(S, B, seq);
    const int64_t stride = (int64_t)B.total_new * S.q_heads;
    auto chunks_of = [&](int row) {
        const KvSpan span = kv_span(S, q, A.window, row / A.rows * A.rows, A.rows);
        return max(1, (span.end - span.begin + A.chunk - 1) / A.chunk);
    };
    if ((int)blockIdx.x >= joins) {
        const int kh = ((int)blockIdx.x - joins) % S.kv_heads, first_block = ((int)blockIdx.x - joins) / S.kv_heads * 32 * KV_WARPS;
        if (first_block << S.block_shift >= q.len) return;
        asm volatile("griddepcontrol.wait;" ::: "memory");
        for (int row0 = 0; row0 < q.n * S.group; row0 += 2 * KV_WARPS) {
            const int row = row0 + (threadIdx.x >> 4), n = row < q.n * S.group ? chunks_of(row) : 0;
            const float* src = A.part_ml + 2 * ((int64_t)(q.start + row / S.group) * S.q_heads + kh * S.group + row % S.group);
            float m = -KV_INF, l = 0.f;
            for (int k = lane & 15; k < n; k += 16) m = fmaxf(m, src[2 * k * stride]);
#pragma unroll
            for (int d = 8; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
            for (int k = lane & 15; k < n; k += 16) {
                const float2 ml = *(const float2*)(src + 2 * k * stride);
                l += ml.y * kv_exp2(ml.x - m);
            }
#pragma unroll
            for (int d = 8; d; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
            if ((lane & 15) == 0 && n) sm_rows[row] = kv_sum_log2(l, m);
        }
        __syncthreads();
        kv_weigh_blocks(S, B, A, q, seq, kh, first_block, sm_rows);
        return;
    }
    const int token = blockIdx.x / S.q_heads, head = blockIdx.x % S.q_heads, chunks = chunks_of(token * S.group + head % S.group);
    const int64_t first = (int64_t)(q.start + token) * S.q_heads + head;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (token >= q.n) return;
    // the largest maximum first, then every chunk's sum and answer by its distance from it: loads that do not wait for one another
    float m = -KV_INF, l = 0.f, acc[V];
    for (int k = lane; k < chunks; k += 32) m = fmaxf(m, A.part_ml[2 * (first + k * stride)]);
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
#pragma unroll
    for (int i = 0; i < V; i++) acc[i] = 0.f;
#pragma unroll 8
    for (int k = warp; k < chunks; k += KV_WARPS) {
        const float2 ml = *(const float2*)(A.part_ml + 2 * (first + k * stride));
        const float* src = A.part_o + (first + k * stride) * D + lane;
        const float h = kv_exp2(ml.x - m);
        l += ml.y * h;
#pragma unroll
        for (int i = 0; i < V; i++) acc[i] += src[32 * i] * h;
    }
#pragma unroll
    for (int i = 0; i < V; i++) sm_acc[warp][32 * i + lane] = acc[i];
    if (lane == 0) sm_sum[warp] = l;
    __syncthreads();
    l = 0.f;
#pragma unroll
    for (int w = 0; w < KV_WARPS; w++) l += sm_sum[w];
    const float inv = kv_over_sum(l);
    if (threadIdx.x < D / 2) {
        float2 x = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < KV_WARPS; w++) { x.x += sm_acc[w][2 * threadIdx.x]; x.y += sm_acc[w][2 * threadIdx.x + 1]; }
        *(uint32_t*)((uint16_t*)A.out.data + (q.start + token) * A.out.token_stride + head * A.out.head_stride + 2 * threadIdx.x) = kv_pack<BF>(x.x * inv, x.y * inv);
    }
    if (threadIdx.x == 0) {
        const float l2 = kv_sum_log2(l, m);
        if (A.lse) A.lse[first] = l2 * 0.6931471805599453f;
        A.lse2[kv_lse2_at(S, q, head / S.group, token * S.group + head % S.group)] = l2;
    }
}

// Weight of each block.  FEW (at most KV_MASS_ROWS rows per sequence and kv head): a thread per block; otherwise a CTA per block (a warp
// per block took 20 us longer for 4096 rows).  The order of the sum is always the same.
template <bool FEW>
__global__ void __launch_bounds__(256) kv_mass_kernel(const KvShape S, const KvBatch B, const KvAttend A)
{
    const int kh = blockIdx.y, seq = blockIdx.z, first_block = FEW ? blockIdx.x * 256 : blockIdx.x;
    __shared__ float shared[KV_MASS_ROWS];               // FEW: the rows' sums; else the warps'
    const KvSeq q = kv_seq(S, B, seq);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (first_block << S.block_shift >= q.len) return;   // the CTA as a whole
    const float* const l2 = A.lse2 + kv_lse2_at(S, q, kh, 0);
    if (FEW) {
        if (threadIdx.x < q.n * S.group) shared[threadIdx.x] = l2[threadIdx.x];
        __syncthreads();
        kv_weigh_blocks(S, B, A, q, seq, kh, first_block, shared);
        return;
    }
    float sum = kv_block_weight<256, 8>(S, B, A, q, seq, kh, first_block, threadIdx.x, l2);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x) return;
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < 8; w++) sum += shared[w];
    const int64_t at = ((int64_t)seq * S.kv_heads + kh) * A.mass_stride + first_block;
    A.mass_out[at] = A.mass_in[at] + sum;
}
