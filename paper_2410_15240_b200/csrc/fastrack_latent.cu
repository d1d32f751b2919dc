// fastrack_latent.cu -- handle, launches and small kernels of the latent cache operators (include/fastrack_latent.h).
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>
#include <atomic>
#include <new>

#include "../../include/fastrack_latent.h"
#include "fastrack_latent_attend.cuh"
#include "fastrack_latent_expand.cuh"
#include "fastrack_latent_prompt.cuh"

// ------------------------------------------------------------------------------------------------ append ----

#define LT_APPEND_THREADS 256           // a warp per token

struct LtAppend { KvRows latent, key, q, q_out; const uint16_t* weight; int token_ctas, q_per; };

// A unit is 16 channels that one thread turns, in two runs of 8: from 8 u on, and from half of the channels further.  The threads of a row so have
// neighbouring runs in either layout, and their accesses whole sectors (17 478 tokens of 128 heads: 115 us; with 16 channels in a row per thread 121).
__device__ __forceinline__ void lt_angles(const KvShape& S, int u, int64_t position, float* cs, float* sn)
{
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int pair = S.rotary == 1 ? 8 * u + i : i < 4 ? 4 * u + i : S.head_dim / 4 + 4 * u + i - 4;
        kv_sincos((uint32_t)((uint64_t)position * S.turns[pair] >> 32), sn[i], cs[i]);
        cs[i] *= S.rotary_gain;
        sn[i] *= S.rotary_gain;
    }
}
// Heads h0 .. h0 + per - 1 of a token: the unit's cosines and sines are made once for them, while the first heads' values are on their way.
#define LT_TURN_AHEAD 2                 // heads whose values are on their way (4: 119 us, 8: 169)
template <bool BF>
__device__ __forceinline__ void lt_turn_heads(const KvShape& S, const KvRows& in, const KvRows& out, const int64_t* positions, int64_t token, int u, int h0, int per, int heads)
{
    const uint16_t* src = (const uint16_t*)in.data + token * in.token_stride + h0 * in.head_stride + 8 * u;
    uint16_t* dst = (uint16_t*)out.data + token * out.token_stride + h0 * out.head_stride + 8 * u;
    const int n = min(per, heads - h0), other = S.head_dim / 2;
    float cs[8], sn[8];
    for (int h = 0; h < n; h += LT_TURN_AHEAD) {
        uint4 a[LT_TURN_AHEAD], b[LT_TURN_AHEAD];
#pragma unroll
        for (int k = 0; k < LT_TURN_AHEAD; k++)
            if (h + k < n) {
                a[k] = *(const uint4*)(src + (h + k) * in.head_stride);
                b[k] = *(const uint4*)(src + (h + k) * in.head_stride + other);
            }
        if (h == 0 && S.rotary) lt_angles(S, u, positions[token], cs, sn);
#pragma unroll
        for (int k = 0; k < LT_TURN_AHEAD; k++)
            if (h + k < n) {
                if (S.rotary) kv_turn_raw<BF>(S, cs, sn, a[k], b[k]);
                *(uint4*)(dst + (h + k) * out.head_stride) = a[k];
                *(uint4*)(dst + (h + k) * out.head_stride + other) = b[k];
            }
    }
}

// The first CTAs store tokens, a warp each: the latent's values stay in registers between the sum of squares and the rounding.  The rest turn
// the queries' part.
template <bool BF> __global__ void __launch_bounds__(LT_APPEND_THREADS) lt_append_kernel(const LtShape S, const LtBatch B, const LtAppend A)
{
    asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if ((int)blockIdx.x >= A.token_ctas) {
        const int units = S.rope / 16, groups = (S.heads + A.q_per - 1) / A.q_per;
        const int64_t i = (int64_t)(blockIdx.x - A.token_ctas) * LT_APPEND_THREADS + threadIdx.x, token = i / units / groups;
        // rows that belong to no sequence are left alone
        if (token < B.total_new && token >= B.starts[0] && token < B.starts[B.n_seqs]) lt_turn_heads<BF>(S.turn, A.q, A.q_out, B.positions, token, (int)(i % units), (int)(i / units % groups) * A.q_per, A.q_per, S.heads);
        return;
    }
    const int per_seq = (B.max_new + LT_APPEND_THREADS / 32 - 1) / (LT_APPEND_THREADS / 32);
    const int seq = blockIdx.x / per_seq, j = blockIdx.x % per_seq * (LT_APPEND_THREADS / 32) + warp;
    const LtSeq q = lt_seq(B, seq);
    if (j >= q.n) return;
    const int place = q.len - q.n + j;
    uint16_t* const dst = place < q.len ? lt_token(S, B, seq, place) : nullptr;
    if (!dst) return;
    const uint16_t* const src = (const uint16_t*)A.latent.data + (q.start + (int64_t)j) * A.latent.token_stride;
    const uint16_t* const key = (const uint16_t*)A.key.data + (q.start + (int64_t)j) * A.key.token_stride;
    const int pieces = S.latent / 8;
    uint4 w[2], kw[2];
#pragma unroll
    for (int k = 0; k < 2; k++)
        if (lane + 32 * k < pieces) w[k] = *(const uint4*)(src + 8 * (lane + 32 * k));
    if (lane < S.rope / 16) {
        kw[0] = *(const uint4*)(key + 8 * lane);
        kw[1] = *(const uint4*)(key + 8 * lane + S.rope / 2);
    }
    if (A.weight) {
        float x[2][8], sum = 0.f;
#pragma unroll
        for (int k = 0; k < 2; k++)
            if (lane + 32 * k < pieces) {
                kv_widen8<BF>(w[k], x[k]);
#pragma unroll
                for (int e = 0; e < 8; e++) sum = fmaf(x[k][e], x[k][e], sum);
            }
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const float by = 1.f / sqrtf(sum / (float)S.latent + S.norm_eps);
#pragma unroll
        for (int k = 0; k < 2; k++)
            if (lane + 32 * k < pieces) {
                float g[8];
                kv_widen8<BF>(*(const uint4*)(A.weight + 8 * (lane + 32 * k)), g);
#pragma unroll
                for (int e = 0; e < 8; e++) x[k][e] = x[k][e] * by * g[e];
                w[k] = kv_narrow8<BF>(x[k]);
            }
    }
#pragma unroll
    for (int k = 0; k < 2; k++)
        if (lane + 32 * k < pieces) *(uint4*)(dst + 8 * (lane + 32 * k)) = w[k];
    if (lane < S.rope / 16) {
        if (S.turn.rotary) {
            float cs[8], sn[8];
            lt_angles(S.turn, lane, B.positions[q.start + j], cs, sn);
            kv_turn_raw<BF>(S.turn, cs, sn, kw[0], kw[1]);
        }
        *(uint4*)(dst + S.latent + 8 * lane) = kw[0];
        *(uint4*)(dst + S.latent + 8 * lane + S.rope / 2) = kw[1];
    }
}

// ------------------------------------------------------------------------------------------------ accept ----

#define LT_ACCEPT_THREADS 128
#define LT_ACCEPT_AHEAD 8               // rows between their reading and their writing

struct LtAccept { const int32_t *parents, *tokens, *choices; int32_t *path, *n_accepted, *next, *lens_out; };

// A CTA per sequence: the tree comes to shared memory, one warp walks it (a step there is some 100 cycles, in global memory 1200), then every thread
// moves its 16 bytes of all accepted rows.
__global__ void __launch_bounds__(LT_ACCEPT_THREADS) lt_accept_kernel(const LtShape S, const LtBatch B, const LtAccept A)
{
    __shared__ int parent[FASTRACK_LATENT_TREE_MOST], token[FASTRACK_LATENT_TREE_MOST], chosen[FASTRACK_LATENT_TREE_MOST], path[FASTRACK_LATENT_TREE_MOST], accepted;
    asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");
    const int seq = blockIdx.x, lane = threadIdx.x & 31;
    const LtSeq q = lt_seq(B, seq);
    for (int j = threadIdx.x; j < q.n; j += LT_ACCEPT_THREADS) {
        parent[j] = A.parents ? A.parents[q.start + j] : j - 1;
        token[j] = A.tokens[q.start + j];
        chosen[j] = A.choices[q.start + j];
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        int n = 0, at = 0, choice = -1;
        while (q.n > 0) {
            if (lane == 0) path[n] = at;
            n++;
            choice = chosen[at];
            int found = -1;
            for (int j0 = at + 1; j0 < q.n && found < 0; j0 += 32) {         // a child is behind its parent
                const int j = j0 + lane;
                const bool child = j < q.n && parent[j] == at && token[j] == choice;
                const uint32_t some = __ballot_sync(0xffffffffu, child);
                if (some) found = j0 + __ffs(some) - 1;
            }
            if (found < 0) break;
            at = found;
        }
        if (lane == 0) {
            accepted = n;
            A.n_accepted[seq] = n;
            A.next[seq] = choice;
        }
    }
    __syncthreads();
    const int n = accepted, base = q.len - q.n;
    for (int k = threadIdx.x; k < q.n; k += LT_ACCEPT_THREADS) A.path[q.start + k] = k < n ? path[k] : -1;
    if (threadIdx.x == 0) A.lens_out[seq] = max(base + n, 0);
    // Row k of the path, k or more, goes to place k, in front of all rows that come later in the path: reading ahead of writing and writing in
    // order is all it takes.
    for (int piece = threadIdx.x; piece < S.row / 8; piece += LT_ACCEPT_THREADS)
        for (int k0 = 0; k0 < n; k0 += LT_ACCEPT_AHEAD) {
            uint4 w[LT_ACCEPT_AHEAD];
            bool there[LT_ACCEPT_AHEAD];
#pragma unroll
            for (int e = 0; e < LT_ACCEPT_AHEAD; e++) {
                const uint16_t* src = k0 + e < n && path[k0 + e] != k0 + e ? lt_token(S, B, seq, base + path[k0 + e]) : nullptr;
                there[e] = src != nullptr;
                if (src) w[e] = *(const uint4*)(src + 8 * piece);
            }
#pragma unroll
            for (int e = 0; e < LT_ACCEPT_AHEAD; e++) {
                uint16_t* dst = there[e] ? lt_token(S, B, seq, base + k0 + e) : nullptr;
                if (dst) *(uint4*)(dst + 8 * piece) = w[e];
            }
        }
}

// ------------------------------------------------------------------------------------------------ handle ----

struct fastrack_latent {
    fastrack_latent_config config;
    LtShape shape;
    int device, num_sms;
    uint64_t* d_turns;
    PFN_cuTensorMapEncodeTiled_v12000 encode;
    std::atomic<int> last_cuda_error;
    std::atomic<uint64_t> launches;
};

static int lt_cuda(fastrack_latent* lt, cudaError_t e)
{
    if (e == cudaSuccess) return FASTRACK_OK;
    lt->last_cuda_error = (int)e;
    (void)cudaGetLastError();
    return FASTRACK_ERR_CUDA;
}
// A launch whose start may overlap the end of the kernel before it in the stream; the kernel waits (griddepcontrol.wait) before it reads
// or writes anything that another may have to do with.  An error stays for cudaGetLastError.
template <class... P, class... Q> static void lt_launch(cudaStream_t stream, dim3 grid, int threads, int smem, void (*kernel)(P...), const Q&... args)
{
    cudaLaunchConfig_t c = {};
    cudaLaunchAttribute overlap;
    overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    overlap.val.programmaticStreamSerializationAllowed = 1;
    c.gridDim = grid;
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = stream;
    c.attrs = &overlap;
    c.numAttrs = 1;
    (void)cudaLaunchKernelEx(&c, kernel, P(args)...);
}
static int lt_launched(fastrack_latent* lt, int count = 1)
{
    lt->launches += (uint64_t)count;
    return lt_cuda(lt, cudaGetLastError());
}
static int lt_check_device(fastrack_latent* lt)
{
    int dev = -1;
    const int rc = lt_cuda(lt, cudaGetDevice(&dev));
    return rc != FASTRACK_OK ? rc : dev == lt->device ? FASTRACK_OK : FASTRACK_ERR_ARG;
}
static bool lt_misaligned(const void* p, size_t a) { return p == nullptr || ((uintptr_t)p & (a - 1)) != 0; }
static bool lt_bad_rows(const fastrack_kv_rows* r) { return !r || lt_misaligned(r->data, 16) || (r->token_stride & 7) || (r->head_stride & 7); }
static KvRows lt_rows(const fastrack_kv_rows* r) { return {r->data, r->token_stride, r->head_stride}; }
static int lt_log2i(int x) { int s = 0; while ((1 << s) < x) s++; return s; }

using LtAttendKernel = void (*)(LtShape, LtBatch, LtAttend, CUtensorMap, CUtensorMap);
struct LtAttendKind { LtAttendKernel kernel; int smem; };
static const LtAttendKind lt_attend_kinds[8] = {          // [latent / 128 - 1][bf16]
    {(LtAttendKernel)lt_attend_kernel<1, false>, LtTile<1>::SMEM}, {(LtAttendKernel)lt_attend_kernel<1, true>, LtTile<1>::SMEM},
    {(LtAttendKernel)lt_attend_kernel<2, false>, LtTile<2>::SMEM}, {(LtAttendKernel)lt_attend_kernel<2, true>, LtTile<2>::SMEM},
    {(LtAttendKernel)lt_attend_kernel<3, false>, LtTile<3>::SMEM}, {(LtAttendKernel)lt_attend_kernel<3, true>, LtTile<3>::SMEM},
    {(LtAttendKernel)lt_attend_kernel<4, false>, LtTile<4>::SMEM}, {(LtAttendKernel)lt_attend_kernel<4, true>, LtTile<4>::SMEM}};
static_assert(LtTile<4>::SMEM <= 232448 && LtTile<2>::SMEM <= 232448, "");

// news: whether the call is about new tokens
static bool lt_bad_batch(const fastrack_latent* lt, const fastrack_latent_batch* b, bool news = true)
{
    if (!b || b->n_seqs < 0 || b->total_new < 0 || b->max_new < 0 || b->max_len < 0 || b->max_len > 1 << 30 || b->pool_pages < 0 || b->table_stride < 0) return true;
    if (b->n_seqs > 65535 || (news && b->max_new > b->total_new) || (b->max_len + lt->config.block_tokens - 1) / lt->config.block_tokens > b->table_stride) return true;
    if (news && ((int64_t)b->max_new * lt->config.heads > 1 << 30 || (int64_t)b->total_new * lt->config.heads > INT32_MAX)) return true;
    if (b->n_seqs == 0) return false;
    if (b->pool_pages > 0 && lt_misaligned(b->d_pool, 16)) return true;
    return lt_misaligned(b->d_lens, 4) || (news && lt_misaligned(b->d_starts, 4)) || (b->table_stride > 0 && lt_misaligned(b->d_table, 4));
}
static LtBatch lt_batch(const fastrack_latent_batch* b)
{
    return {b->n_seqs, b->total_new, b->max_new, b->max_len, b->pool_pages, b->table_stride, (uint16_t*)b->d_pool, b->d_table, b->d_lens, b->d_starts,
            b->d_positions};
}

#define LT_SMEM_MOST 232448

extern "C" int fastrack_latent_create(const fastrack_latent_config* c, fastrack_latent** out)
{
    if (out) *out = nullptr;
    if (!c || !out) return FASTRACK_ERR_ARG;
    if (c->dtype != FASTRACK_KV_BF16 && c->dtype != FASTRACK_KV_F16) return FASTRACK_ERR_ARG;
    if (c->heads < 1 || c->heads > 1024 || c->latent_dim < 128 || c->latent_dim > 512 || c->latent_dim % 128) return FASTRACK_ERR_ARG;
    if ((c->rope_dim != 32 && c->rope_dim != 64) || (c->key_dim != 64 && c->key_dim != 128) || (c->value_dim != 64 && c->value_dim != 128)) return FASTRACK_ERR_ARG;
    if (c->block_tokens != 16 && c->block_tokens != 32 && c->block_tokens != 64 && c->block_tokens != 128) return FASTRACK_ERR_ARG;
    if (c->rotary < FASTRACK_ROTARY_NONE || c->rotary > FASTRACK_ROTARY_INTERLEAVED) return FASTRACK_ERR_ARG;
    if (c->rotary == FASTRACK_ROTARY_NONE ? c->frequencies != nullptr : !c->frequencies || !isfinite(c->rotary_gain)) return FASTRACK_ERR_ARG;
    if (!isfinite(c->softmax_scale) || c->softmax_scale < 0.f || !isfinite(c->norm_eps) || c->norm_eps < 0.f) return FASTRACK_ERR_ARG;
    uint64_t turns[KV_MAX_PAIRS] = {0};
    for (int i = 0; c->rotary && i < c->rope_dim / 2; i++) {
        if (!isfinite(c->frequencies[i])) return FASTRACK_ERR_ARG;
        const long double t = (long double)c->frequencies[i] / 6.283185307179586476925286766559L;
        const long double part = floorl((t - floorl(t)) * 18446744073709551616.0L);
        turns[i] = part < 18446744073709551616.0L ? (uint64_t)part : 0u;
    }
    fastrack_latent* lt = new (std::nothrow) fastrack_latent();
    if (!lt) return FASTRACK_ERR_NOMEM;
    lt->config = *c;
    lt->config.frequencies = nullptr;
    lt->last_cuda_error = 0;
    lt->launches = 0;
    LtShape& S = lt->shape;
    S.heads = c->heads;
    S.latent = c->latent_dim;
    S.rope = c->rope_dim;
    S.row = c->latent_dim + c->rope_dim;
    S.key = c->key_dim;
    S.value = c->value_dim;
    S.block_tokens = c->block_tokens;
    S.block_shift = lt_log2i(c->block_tokens);
    S.norm_eps = c->norm_eps;
    S.scale_log2 = (c->softmax_scale == 0.f ? 1.f / sqrtf((float)(c->key_dim + c->rope_dim)) : c->softmax_scale) * 1.4426950408889634f;
    S.turn.head_dim = c->rope_dim;
    S.turn.rotary = c->rotary;
    S.turn.rotary_dim = c->rotary ? c->rope_dim : 0;
    S.turn.rotary_gain = c->rotary_gain;
    cudaError_t e = cudaGetDevice(&lt->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&lt->num_sms, cudaDevAttrMultiProcessorCount, lt->device);
    void* encode = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (e == cudaSuccess) e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &encode, 12000, cudaEnableDefault, &found);
    if (e == cudaSuccess && (found != cudaDriverEntryPointSuccess || !encode)) e = cudaErrorNotSupported;
    lt->encode = (PFN_cuTensorMapEncodeTiled_v12000)encode;
    if (e == cudaSuccess) e = cudaMalloc(&lt->d_turns, sizeof turns);
    if (e == cudaSuccess) e = cudaMemcpy(lt->d_turns, turns, sizeof turns, cudaMemcpyHostToDevice);
    auto ask = [&](const void* kernel, int bytes) { if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); };
    for (const LtAttendKind& kind : lt_attend_kinds) ask((const void*)kind.kernel, kind.smem);
    ask((const void*)lt_expand_kernel<true>, LT_SMEM_MOST);
    ask((const void*)lt_expand_kernel<false>, LT_SMEM_MOST);
    ask((const void*)lt_prompt_kernel<true>, LT_SMEM_MOST);
    ask((const void*)lt_prompt_kernel<false>, LT_SMEM_MOST);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        fastrack_latent_destroy(lt);
        return e == cudaErrorMemoryAllocation ? FASTRACK_ERR_NOMEM : FASTRACK_ERR_CUDA;
    }
    S.turn.turns = lt->d_turns;
    *out = lt;
    return FASTRACK_OK;
}

extern "C" void fastrack_latent_destroy(fastrack_latent* lt)
{
    if (!lt) return;
    if (lt->d_turns) (void)cudaFree(lt->d_turns);
    delete lt;
}

extern "C" size_t fastrack_latent_page_bytes(const fastrack_latent* lt) { return lt ? (size_t)lt->shape.row * lt->shape.block_tokens * 2 : 0; }
extern "C" int fastrack_latent_last_cuda_error(const fastrack_latent* lt) { return lt ? lt->last_cuda_error.load() : 0; }
extern "C" uint64_t fastrack_latent_launch_count(const fastrack_latent* lt) { return lt ? lt->launches.load() : 0; }

extern "C" int fastrack_latent_append(fastrack_latent* lt, const fastrack_latent_batch* batch, const fastrack_kv_rows* latents, const fastrack_kv_rows* key,
                                      const void* d_norm_weight, const fastrack_kv_rows* q, const fastrack_kv_rows* q_out, void* stream)
{
    if (!lt || lt_bad_batch(lt, batch) || !q != !q_out) return FASTRACK_ERR_ARG;
    if (batch->n_seqs == 0 || batch->total_new == 0 || batch->max_new == 0) return FASTRACK_OK;
    if (lt_bad_rows(latents) || lt_bad_rows(key) || (q && (lt_bad_rows(q) || lt_bad_rows(q_out)))) return FASTRACK_ERR_ARG;
    if ((d_norm_weight && lt_misaligned(d_norm_weight, 16)) || (lt->config.rotary && lt_misaligned(batch->d_positions, 8))) return FASTRACK_ERR_ARG;
    if (q && q->data == q_out->data && (q->token_stride != q_out->token_stride || q->head_stride != q_out->head_stride)) return FASTRACK_ERR_ARG;
    if (int rc = lt_check_device(lt)) return rc;
    const LtShape& S = lt->shape;
    LtAppend A;
    memset(&A, 0, sizeof A);
    A.latent = lt_rows(latents);
    A.key = lt_rows(key);
    A.weight = (const uint16_t*)d_norm_weight;
    const int64_t token_ctas = (int64_t)batch->n_seqs * ((batch->max_new + LT_APPEND_THREADS / 32 - 1) / (LT_APPEND_THREADS / 32));
    int64_t turn = 0;
    A.q_per = 1;
    if (q) {
        A.q = lt_rows(q);
        A.q_out = lt_rows(q_out);
        // heads that one thread turns: as many as still leave every SM two CTAs
        auto threads = [&](int per) { return (int64_t)batch->total_new * (S.rope / 16) * ((S.heads + per - 1) / per); };
        for (A.q_per = 8; A.q_per > 1 && threads(A.q_per) < (int64_t)2 * LT_APPEND_THREADS * lt->num_sms;) A.q_per /= 2;
        turn = (threads(A.q_per) + LT_APPEND_THREADS - 1) / LT_APPEND_THREADS;
    }
    if (token_ctas + turn > INT32_MAX) return FASTRACK_ERR_ARG;
    A.token_ctas = (int)token_ctas;
    auto kernel = lt->config.dtype == FASTRACK_KV_BF16 ? lt_append_kernel<true> : lt_append_kernel<false>;
    lt_launch((cudaStream_t)stream, dim3((unsigned)(token_ctas + turn)), LT_APPEND_THREADS, 0, kernel, S, lt_batch(batch), A);
    return lt_launched(lt);
}

extern "C" int fastrack_latent_accept(fastrack_latent* lt, const fastrack_latent_batch* batch, const fastrack_latent_acceptance* a, void* stream)
{
    if (!lt || lt_bad_batch(lt, batch) || batch->max_new > FASTRACK_LATENT_TREE_MOST || !a) return FASTRACK_ERR_ARG;
    if (batch->n_seqs == 0) return FASTRACK_OK;
    if (lt_misaligned(a->d_n_accepted, 4) || lt_misaligned(a->d_next, 4) || lt_misaligned(a->d_lens_out, 4) || ((uintptr_t)a->d_parents & 3)) return FASTRACK_ERR_ARG;
    if (batch->total_new > 0 && (lt_misaligned(a->d_tokens, 4) || lt_misaligned(a->d_choices, 4) || lt_misaligned(a->d_path, 4))) return FASTRACK_ERR_ARG;
    if (int rc = lt_check_device(lt)) return rc;
    const LtAccept A = {a->d_parents, a->d_tokens, a->d_choices, a->d_path, a->d_n_accepted, a->d_next, a->d_lens_out};
    lt_launch((cudaStream_t)stream, dim3(batch->n_seqs), LT_ACCEPT_THREADS, 0, lt_accept_kernel, lt->shape, lt_batch(batch), A);
    return lt_launched(lt);
}

// ------------------------------------------------------------------------------------------------ attention ----

struct LtPlan { int groups, group_tiles, seq_groups; size_t ml, cuts, total; };      // byte offsets in the workspace, part_o at 0

// CTAs that read the same tokens side by side, one per row tile: all row tiles of a sequence up to 8 (an SM in 148 / 8 may be left over),
// and beyond that the number between 5 and 8 that wastes the fewest CTAs on row tiles that are not there or SMs that are left.
static LtPlan lt_plan(const fastrack_latent* lt, const fastrack_latent_batch* b)
{
    const LtShape& S = lt->shape;
    LtPlan p;
    const int64_t rows = (int64_t)b->max_new * S.heads, row_tiles = rows > LT_ROWS ? (rows + LT_ROWS - 1) / LT_ROWS : 1;
    const int sms = lt->num_sms < LT_JOIN_CUTS ? lt->num_sms : LT_JOIN_CUTS;
    p.group_tiles = (int)(row_tiles < 8 ? row_tiles : 8);
    if (row_tiles > 8) {
        double best = 0;
        for (int t = 8; t >= 5; t--) {
            const double used = (double)row_tiles / (double)((row_tiles + t - 1) / t * t) * (sms / t * t);
            if (used > best) {
                best = used;
                p.group_tiles = t;
            }
        }
    }
    if (p.group_tiles > sms) p.group_tiles = sms;
    p.groups = sms / p.group_tiles;
    p.seq_groups = (int)((row_tiles + p.group_tiles - 1) / p.group_tiles);
    const size_t slots = (size_t)p.groups * 2 * p.group_tiles * LT_ROWS;
    p.ml = slots * S.latent * 4;
    p.cuts = p.ml + slots * 8;
    p.total = p.cuts + (size_t)p.groups * 16;
    return p;
}

extern "C" size_t fastrack_latent_attention_workspace(const fastrack_latent* lt, const fastrack_latent_batch* batch)
{
    if (!lt || lt_bad_batch(lt, batch)) return 0;
    return lt_plan(lt, batch).total;
}

// A tensor map of 16-bit values (x: row's values, y: rows, z, and w if there is one), whose boxes are 64 values wide
static int lt_map(fastrack_latent* lt, CUtensorMap* map, void* data, int64_t width, int64_t y, int64_t z, int64_t y_bytes, int64_t z_bytes, int box_y, int64_t w = 0,
                  int64_t w_bytes = 0, int box_z = 1)
{
    const cuuint64_t dims[4] = {(cuuint64_t)width, (cuuint64_t)y, (cuuint64_t)z, (cuuint64_t)w}, strides[3] = {(cuuint64_t)y_bytes, (cuuint64_t)z_bytes, (cuuint64_t)w_bytes};
    const cuuint32_t box[4] = {64, (cuuint32_t)box_y, (cuuint32_t)box_z, 1}, steps[4] = {1, 1, 1, 1};
    auto encode = [&] {
        return lt->encode(map, lt->config.dtype == FASTRACK_KV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, w ? 4 : 3, data, dims, strides, box, steps,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    };
    CUresult r = encode();
    // a thread that has made no runtime call yet has no context, which the driver's function wants: setting the device, which is current
    // by number already, makes it so
    if (r == CUDA_ERROR_INVALID_CONTEXT && lt_cuda(lt, cudaSetDevice(lt->device)) == FASTRACK_OK) r = encode();
    if (r == CUDA_SUCCESS) return FASTRACK_OK;
    lt->last_cuda_error = (int)r;
    return FASTRACK_ERR_CUDA;
}
// The pool: rows of a page, pages; boxes of up to 64 tokens of one page
static int lt_pool_map(fastrack_latent* lt, const LtBatch& B, CUtensorMap* map)
{
    const LtShape& S = lt->shape;
    memset(map, 0, sizeof *map);
    if (B.pool_pages == 0) return FASTRACK_OK;           // every page is absent
    return lt_map(lt, map, B.pool, S.row, S.block_tokens, B.pool_pages, 2 * S.row, (int64_t)2 * S.row * S.block_tokens, S.block_tokens < LT_TOKENS ? S.block_tokens : LT_TOKENS);
}

// The pool's latents by 64 channels: channels, rows of a page, which 64, pages; boxes of 64 tokens and 128 channels (blocks of 64 tokens or more)
static int lt_pairs_map(fastrack_latent* lt, const LtBatch& B, CUtensorMap* map)
{
    const LtShape& S = lt->shape;
    memset(map, 0, sizeof *map);
    if (B.pool_pages == 0 || S.block_tokens < LT_TOKENS) return FASTRACK_OK;
    return lt_map(lt, map, B.pool, 64, S.block_tokens, S.latent / 64, 2 * S.row, 128, LT_TOKENS, B.pool_pages, (int64_t)2 * S.row * S.block_tokens, 2);
}

extern "C" int fastrack_latent_attention(fastrack_latent* lt, const fastrack_latent_batch* batch, const fastrack_kv_rows* q, const fastrack_kv_rows* q_rope,
                                         const fastrack_kv_rows* out, float* d_lse, const int32_t* d_parents, void* d_workspace, size_t workspace_bytes, void* stream)
{
    if (!lt || lt_bad_batch(lt, batch) || (d_parents && batch->max_new > FASTRACK_LATENT_TREE_MOST)) return FASTRACK_ERR_ARG;
    if (batch->n_seqs == 0 || batch->total_new == 0 || batch->max_new == 0) return FASTRACK_OK;
    if (lt_bad_rows(q) || lt_bad_rows(q_rope) || lt_bad_rows(out) || ((uintptr_t)d_lse & 3) || ((uintptr_t)d_parents & 3)) return FASTRACK_ERR_ARG;
    const LtPlan p = lt_plan(lt, batch);
    if (lt_misaligned(d_workspace, 16) || workspace_bytes < p.total) return FASTRACK_ERR_ARG;
    if (int rc = lt_check_device(lt)) return rc;
    const LtShape& S = lt->shape;
    const LtBatch B = lt_batch(batch);
    char* const ws = (char*)d_workspace;
    LtAttend A;
    memset(&A, 0, sizeof A);
    A.q = lt_rows(q);
    A.q_rope = lt_rows(q_rope);
    A.out = lt_rows(out);
    A.lse = d_lse;
    A.parents = d_parents;
    A.groups = p.groups;
    A.group_tiles = p.group_tiles;
    A.seq_groups = p.seq_groups;
    A.least = 2;
    A.part_o = (float*)ws;
    A.part_ml = (float*)(ws + p.ml);
    A.cuts = (int*)(ws + p.cuts);
    CUtensorMap pool, pairs;
    if (int rc = lt_pool_map(lt, B, &pool)) return rc;
    if (int rc = lt_pairs_map(lt, B, &pairs)) return rc;
    const bool bf = lt->config.dtype == FASTRACK_KV_BF16;
    const cudaStream_t st = (cudaStream_t)stream;
    const LtAttendKind& kind = lt_attend_kinds[2 * (S.latent / 128 - 1) + bf];
    lt_launch(st, dim3(p.groups * p.group_tiles), LT_A_THREADS, kind.smem, kind.kernel, S, B, A, pool, pairs);
    lt_launch(st, dim3(16 * lt->num_sms), LT_JOIN_THREADS, 0, bf ? lt_join_kernel<true> : lt_join_kernel<false>, S, B, A);
    return lt_launched(lt, 2);
}

// ------------------------------------------------------------------------------------------------ expanded ----

extern "C" int fastrack_latent_expand(fastrack_latent* lt, const fastrack_latent_batch* batch, const void* d_weights, const fastrack_kv_rows* k_out,
                                      const fastrack_kv_rows* v_out, const int32_t* d_key_starts, int total_keys, void* stream)
{
    if (!lt || lt_bad_batch(lt, batch, false) || total_keys < 0) return FASTRACK_ERR_ARG;
    if (batch->n_seqs == 0 || batch->max_len == 0 || total_keys == 0) return FASTRACK_OK;
    if (lt_misaligned(d_weights, 16) || lt_bad_rows(k_out) || lt_bad_rows(v_out) || lt_misaligned(d_key_starts, 4)) return FASTRACK_ERR_ARG;
    if (int rc = lt_check_device(lt)) return rc;
    const LtShape& S = lt->shape;
    const LtBatch B = lt_batch(batch);
    const LtExpand A = {lt_rows(k_out), lt_rows(v_out), d_key_starts, total_keys, S.heads};
    CUtensorMap pool, weights;
    const int64_t row = (int64_t)2 * S.latent;
    const int width = S.key + S.value;
    if (int rc = lt_pool_map(lt, B, &pool)) return rc;
    if (int rc = lt_map(lt, &weights, const_cast<void*>(d_weights), S.latent, width, S.heads, row, row * width, width / 2)) return rc;
    auto kernel = lt->config.dtype == FASTRACK_KV_BF16 ? lt_expand_kernel<true> : lt_expand_kernel<false>;
    lt_launch((cudaStream_t)stream, dim3(lt->num_sms / 2 * 2), LT_E_THREADS, lt_expand_smem(S.latent), kernel, S, B, A, pool, weights);
    return lt_launched(lt);
}

// Rows of keys or values as a tensor (x: channels, y: rows, z: heads, or one where they share their rows); boxes of `box` rows
static int lt_keys_map(fastrack_latent* lt, const fastrack_kv_rows* r, int width, int total_keys, int box, CUtensorMap* map)
{
    memset(map, 0, sizeof *map);
    if (total_keys == 0) return FASTRACK_OK;             // nobody sees anything
    const int heads = r->head_stride ? lt->shape.heads : 1;
    return lt_map(lt, map, r->data, width, total_keys, heads, r->token_stride ? 2 * r->token_stride : 2 * width, r->head_stride ? 2 * r->head_stride : 2 * width, box);
}
// Strides that a tensor map takes
static bool lt_bad_keys(const fastrack_kv_rows* r, int total_keys)
{
    return lt_bad_rows(r) || r->token_stride < (total_keys > 1) || r->head_stride < 0 || r->token_stride >= (int64_t)1 << 38 || r->head_stride >= (int64_t)1 << 38;
}

// Where 512 queries of each head and sequence do not fill the pairs of SMs, pairs share a job's tokens between them: as many as there is room for, with
// LT_P_LEAST steps each at least of those that a query sees on average in the longest sequence that there may be.
// One pair a job against shares, one sequence, bf16, device time: 16 heads, 512 new of 4000 tokens 81 -> 41 us, of 16000 272 -> 86; 130 new of 32000
// 489 -> 135; 32 heads, 1 new of 8000 129 -> 72; 2 heads, 10 new of 800 (two shares of 3 steps) 20.1 -> 16.7.  Where the average query sees fewer steps,
// sharing costs: 16 heads, 1000 new of 1000, whose first queries see little, 32.6 whole and 35.7 in two shares.
#define LT_P_LEAST 3
struct LtPromptPlan { int tiles, splits; size_t ml, total; };                // byte offsets in the workspace, part_o at 0
static LtPromptPlan lt_prompt_plan(const fastrack_latent* lt, const fastrack_latent_batch* b)
{
    LtPromptPlan p;
    p.tiles = (b->max_new + 4 * LT_P_ROWS - 1) / (4 * LT_P_ROWS);
    const int64_t jobs = (int64_t)p.tiles * lt->shape.heads * b->n_seqs, steps = ((int64_t)b->max_len - b->max_new / 2) / LT_P_TOKENS;
    int64_t splits = jobs > 0 ? lt->num_sms / 2 / jobs : 1;
    if (splits > steps / LT_P_LEAST) splits = steps / LT_P_LEAST;
    p.splits = splits > 1 ? (int)splits : 1;
    const size_t rows = p.splits > 1 ? (size_t)p.splits * b->total_new * lt->shape.heads : 0;
    p.ml = rows * lt->shape.value * 4;
    p.total = p.ml + rows * 8;
    return p;
}

extern "C" size_t fastrack_latent_prompt_workspace(const fastrack_latent* lt, const fastrack_latent_batch* batch)
{
    if (!lt || lt_bad_batch(lt, batch)) return 0;
    return lt_prompt_plan(lt, batch).total;
}

extern "C" int fastrack_latent_prompt(fastrack_latent* lt, const fastrack_latent_batch* batch, const fastrack_kv_rows* q, const fastrack_kv_rows* q_rope,
                                      const fastrack_kv_rows* k, const fastrack_kv_rows* v, const int32_t* d_key_starts, int total_keys, const fastrack_kv_rows* out,
                                      float* d_lse, void* d_workspace, size_t workspace_bytes, void* stream)
{
    if (!lt || lt_bad_batch(lt, batch) || total_keys < 0) return FASTRACK_ERR_ARG;
    if (batch->n_seqs == 0 || batch->total_new == 0 || batch->max_new == 0) return FASTRACK_OK;
    if (lt_bad_rows(q) || lt_bad_rows(q_rope) || lt_bad_rows(out) || ((uintptr_t)d_lse & 3) || lt_misaligned(d_key_starts, 4)) return FASTRACK_ERR_ARG;
    if (total_keys > 0 && (lt_bad_keys(k, total_keys) || lt_bad_keys(v, total_keys))) return FASTRACK_ERR_ARG;
    const LtPromptPlan p = lt_prompt_plan(lt, batch);
    if (p.total > 0 && (lt_misaligned(d_workspace, 16) || workspace_bytes < p.total)) return FASTRACK_ERR_ARG;
    if (int rc = lt_check_device(lt)) return rc;
    const LtShape& S = lt->shape;
    const LtBatch B = lt_batch(batch);
    LtPrompt A;
    memset(&A, 0, sizeof A);
    A.q = lt_rows(q);
    A.q_rope = lt_rows(q_rope);
    A.out = lt_rows(out);
    A.lse = d_lse;
    A.key_starts = d_key_starts;
    A.total_keys = total_keys;
    A.tiles = p.tiles;
    A.splits = p.splits;
    A.part_o = (float*)d_workspace;
    A.part_ml = (float*)((char*)d_workspace + p.ml);
    CUtensorMap pool, k_map, v_map;
    memset(&k_map, 0, sizeof k_map);
    memset(&v_map, 0, sizeof v_map);
    if (int rc = lt_pool_map(lt, B, &pool)) return rc;
    if (total_keys > 0) {
        A.v = (const uint16_t*)v->data;
        A.v_token_stride = v->token_stride;
        A.v_head_stride = v->head_stride;
        A.k_heads = k->head_stride != 0;
        A.v_heads = v->head_stride != 0;
        if (int rc = lt_keys_map(lt, k, S.key, total_keys, LT_P_TOKENS / 2, &k_map)) return rc;
        if (int rc = lt_keys_map(lt, v, S.value, total_keys, LT_P_TOKENS, &v_map)) return rc;
    }
    const bool bf = lt->config.dtype == FASTRACK_KV_BF16;
    const cudaStream_t st = (cudaStream_t)stream;
    lt_launch(st, dim3(2u * A.tiles * S.heads, A.splits, batch->n_seqs), LT_P_THREADS, lt_prompt_smem(S), bf ? lt_prompt_kernel<true> : lt_prompt_kernel<false>, S, B, A, pool, k_map,
              v_map);
    if (A.splits == 1) return lt_launched(lt);
    const unsigned rows = (unsigned)(((int64_t)batch->max_new * S.heads + LT_P_JOIN_THREADS / 32 - 1) / (LT_P_JOIN_THREADS / 32));
    lt_launch(st, dim3(rows, batch->n_seqs), LT_P_JOIN_THREADS, 0, bf ? lt_prompt_join_kernel<true> : lt_prompt_join_kernel<false>, S, B, A);
    return lt_launched(lt, 2);
}
