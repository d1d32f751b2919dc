// fastrack_kv_device.cuh -- what the key-value cache kernels share: the parameters, the view of one sequence, 16-bit and
// 8-bit conversions, and the rotation of one unit of 16 channels.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#define KV_MAX_PAIRS 64
#define KV_INF __int_as_float(0x7f800000)

struct KvShape {                        // constants of a handle
    int q_heads, kv_heads, group, head_dim, block_tokens, block_shift;
    int rotary, rotary_dim;
    float rotary_gain, scale_log2;      // softmax scale times log2(e)
    uint32_t codes_bytes;               // K codes of a page; V's follow, then the scales
    uint64_t page_bytes, tail_values;   // tail_values: 16-bit values in a sequence's tail row
    const uint64_t* turns;              // device: frequency of each pair in turns per position, times 2^64
};

struct KvRows { void* data; int64_t token_stride, head_stride; };

struct KvBatch {
    int n_seqs, total_new, max_new, max_len, pool_pages, table_stride;
    uint8_t* pool;
    void* tail;
    const int32_t *table, *lens, *starts;
    const int64_t* positions;
};

// One sequence as the device's numbers give it, clamped to the bounds that buffers were sized for: whatever stands in
// lens and starts, every index that follows from these stays inside them.
struct KvSeq { int len, start, n, full; };   // tokens held, first packed row, new tokens, full blocks

__device__ __forceinline__ KvSeq kv_seq(const KvShape& S, const KvBatch& B, int i)
{
    KvSeq q;
    q.len = min(max(B.lens[i], 0), B.max_len);
    q.start = min(max(B.starts[i], 0), B.total_new);
    q.n = min(max(min(B.starts[i + 1], B.total_new) - q.start, 0), B.max_new);
    q.full = q.len >> S.block_shift;
    return q;
}

// Page of a full block, or -1 where it is absent.
__device__ __forceinline__ int kv_page(const KvBatch& B, int seq, int block)
{
    if (block >= B.table_stride) return -1;
    const int p = B.table[(int64_t)seq * B.table_stride + block];
    return p >= 0 && p < B.pool_pages ? p : -1;
}

__device__ __forceinline__ const float* kv_scales(const KvShape& S, const KvBatch& B, int page)
{
    return (const float*)(B.pool + (uint64_t)page * S.page_bytes + 2u * (uint64_t)S.codes_bytes);
}

template <bool BF> __device__ __forceinline__ float2 kv_unpack(uint32_t w)
{
    if (BF) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    return __half22float2(*(const __half2*)&w);
}
template <bool BF> __device__ __forceinline__ uint32_t kv_pack(float a, float b)
{
    if (BF) { __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *(uint32_t*)&h; }
    __half2 h = __floats2half2_rn(a, b);
    return *(uint32_t*)&h;
}

// A unit is 16 channels that one thread turns: 8 pairs.  half layout: 8 channels of the first half and the 8 they pair
// with; interleaved and unturned channels: 16 in a row.
struct KvUnit { int a, b; bool turned; };   // first channel of the two runs of 8
__device__ __forceinline__ KvUnit kv_unit(const KvShape& S, int u)
{
    const bool turned = 16 * u < S.rotary_dim;
    if (turned && S.rotary == 1) return {8 * u, 8 * u + S.rotary_dim / 2, true};
    return {16 * u, 16 * u + 8, turned};
}

// sin and cos of a phase in turns times 2^32.  The nearest quarter turn is taken off in whole numbers; what is left, at most an eighth of
// a turn, is a float to 2^-24 of itself, and the power series of sin and cos up to the 9th and 10th power are off by less than 2^-29
// there.  (About 20 instructions, half of the general function's.)
__device__ __forceinline__ void kv_sincos(uint32_t phase, float& s, float& c)
{
    const uint32_t quarter = phase + 0x20000000u;
    const float x = (float)(int32_t)((quarter & 0x3fffffffu) - 0x20000000u) * (6.283185307179586f * 0x1p-32f), y = x * x;
    float u = fmaf(y, 1.f / 362880, -1.f / 5040), w = fmaf(y, -1.f / 3628800, 1.f / 40320);
    w = fmaf(y, w, -1.f / 720);
    u = fmaf(y, u, 1.f / 120);
    w = fmaf(y, w, 1.f / 24);
    u = fmaf(y, u, -1.f / 6);
    w = fmaf(y, w, -.5f);
    u = fmaf(x * y, u, x);
    w = fmaf(y, w, 1.f);
    const bool swap = quarter & 0x40000000u;
    s = __uint_as_float(__float_as_uint(swap ? w : u) ^ (quarter & 0x80000000u));
    c = __uint_as_float(__float_as_uint(swap ? u : w) ^ ((quarter ^ (quarter << 1)) & 0x80000000u));
}

// cos and sin of the unit's 8 angles times the gain.  The angle in turns is position * turns mod 1: the top 32 bits of a 64-bit product
// that wraps.  What the table's numbers lack below 2^-64 counts once per position: 2^-63 of a turn with their own rounding.
__device__ __forceinline__ void kv_angles(const KvShape& S, int u, int64_t position, bool inverse, float* cs, float* sn)
{
    const float gain = inverse ? -S.rotary_gain : S.rotary_gain;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        kv_sincos((uint32_t)((uint64_t)position * S.turns[8 * u + i] >> 32), sn[i], cs[i]);
        cs[i] *= S.rotary_gain;
        sn[i] *= gain;
    }
}

// x[0..7] and x[8..15]: the unit's two runs.
__device__ __forceinline__ void kv_turn(const KvShape& S, float* x, const float* cs, const float* sn)
{
    if (S.rotary == 1) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float a = x[i], b = x[8 + i];
            x[i] = a * cs[i] - b * sn[i];
            x[8 + i] = b * cs[i] + a * sn[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float a = x[2 * i], b = x[2 * i + 1];
            x[2 * i] = a * cs[i] - b * sn[i];
            x[2 * i + 1] = b * cs[i] + a * sn[i];
        }
    }
}

template <bool BF> __device__ __forceinline__ void kv_widen8(const uint4& w, float* x)
{
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; i++) { const float2 f = kv_unpack<BF>(v[i]); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
}
template <bool BF> __device__ __forceinline__ uint4 kv_narrow8(const float* x)
{
    return make_uint4(kv_pack<BF>(x[0], x[1]), kv_pack<BF>(x[2], x[3]), kv_pack<BF>(x[4], x[5]), kv_pack<BF>(x[6], x[7]));
}

// Codes of 4 values that were multiplied by top / amax (so that rounding leaves none above the top).  int8: the sum with 1.5 * 2^23 is
// rounded to a whole number, to even, whose last byte is the code.  A NaN gives some code, but none that is a NaN.
template <bool E4M3> __device__ __forceinline__ uint32_t kv_codes4(const float* x)
{
    if constexpr (E4M3) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(fmaxf(x[0], -448.f), fmaxf(x[1], -448.f)), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(fmaxf(x[2], -448.f), fmaxf(x[3], -448.f)), __NV_SATFINITE, __NV_E4M3);
        return lo | hi << 16;
    } else {
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; i++) y[i] = __float_as_uint(__fadd_rn(x[i], 12582912.f));
        return __byte_perm(__byte_perm(y[0], y[1], 0x0040), __byte_perm(y[2], y[3], 0x0040), 0x5410);
    }
}
// The larger of a and |x|; a NaN wins
__device__ __forceinline__ float kv_max_nan(float a, float x)
{
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(fabsf(x)));
    return a;
}
template <bool E4M3> __device__ __forceinline__ void kv_decode4(uint32_t w, float scale, float* x)
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t b = w >> (8 * i) & 255u;
        if (E4M3) {
            __nv_fp8_e4m3 f;
            f.__x = (__nv_fp8_storage_t)b;
            x[i] = (float)f * scale;
        } else {
            x[i] = (float)(int8_t)b * scale;
        }
    }
}

// The tokens that rows first_row .. first_row + rows - 1 of a sequence's (query, head of the group) rows see between them, from a
// block's start on: where the work on these rows begins and ends.  Rows behind the last give nothing.
struct KvSpan { int begin, end; };
__device__ __forceinline__ KvSpan kv_span(const KvShape& S, const KvSeq& q, int window, int first_row, int rows)
{
    const int last_row = min(first_row + rows, q.n * S.group) - 1;
    if (first_row > last_row) return {0, 0};
    const int first_place = q.len - q.n + first_row / S.group, last_place = q.len - q.n + last_row / S.group;
    KvSpan s;
    s.end = max(last_place + 1, 0);
    s.begin = window > 0 ? max(first_place - window + 1, 0) >> S.block_shift << S.block_shift : 0;
    if (s.begin > s.end) s.begin = s.end;
    return s;
}
