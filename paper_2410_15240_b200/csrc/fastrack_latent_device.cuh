// fastrack_latent_device.cuh -- what the latent cache's kernels share: parameters, the view of one sequence, copies into swizzled tiles.
#pragma once
#include <cuda.h>
#include "fastrack_kv_prompt.cuh"

struct LtShape {                        // constants of a handle
    KvShape turn;                       // for the rotation: a "head" of rope channels
    int heads, latent, rope, row;       // row: latent + rope, the values of a token
    int key, value, block_tokens, block_shift;
    float scale_log2, norm_eps;         // softmax scale times log2(e)
};

struct LtBatch {
    int n_seqs, total_new, max_new, max_len, pool_pages, table_stride;
    uint16_t* pool;
    const int32_t *table, *lens, *starts;
    const int64_t* positions;
};

// One sequence as the device's numbers give it, clamped to the bounds that buffers were sized for.
struct LtSeq { int len, start, n; };    // tokens held, first packed row, new tokens

__device__ __forceinline__ int lt_len(const LtBatch& B, int i) { return min(max(B.lens[i], 0), B.max_len); }
__device__ __forceinline__ LtSeq lt_seq(const LtBatch& B, int i)
{
    LtSeq q;
    q.len = lt_len(B, i);
    q.start = min(max(B.starts[i], 0), B.total_new);
    q.n = min(max(min(B.starts[i + 1], B.total_new) - q.start, 0), B.max_new);
    return q;
}

// Page of a block, or -1 where it is absent.
__device__ __forceinline__ int lt_page(const LtBatch& B, int seq, int block)
{
    if (block < 0 || block >= B.table_stride) return -1;
    const int p = B.table[(int64_t)seq * B.table_stride + block];
    return p >= 0 && p < B.pool_pages ? p : -1;
}

// The vector at a place of a sequence, or NULL where its page is absent.
__device__ __forceinline__ uint16_t* lt_token(const LtShape& S, const LtBatch& B, int seq, int place)
{
    const int page = place < 0 ? -1 : lt_page(B, seq, place >> S.block_shift);
    return page < 0 ? nullptr : B.pool + ((int64_t)page * S.block_tokens + (place & (S.block_tokens - 1))) * S.row;
}

// A tile in shared memory is made of chunks of 64 channels: rows of 128 bytes, whose 16-byte pieces are swizzled by the row's number.
#define LT_CHUNK_ROW 128
__device__ __forceinline__ uint32_t lt_at(int row, int piece) { return (uint32_t)(row * LT_CHUNK_ROW + ((piece ^ (row & 7)) << 4)); }

// A warp as a whole comes to the copies and products below, and one thread of it issues them: the operands then are where the compiler knows them
// to be the same for all lanes, in the registers that these instructions want.  (Issued by `if (lane == 0)`, a copy held up its warp for 800
// cycles and a product for 500.)  So must be what the operands come from: a page number goes through lt_uniform.
__device__ __forceinline__ int lt_uniform(int x, int lane)                   // lane's x; not below -1
{
    return (int)__reduce_max_sync(0xffffffffu, (threadIdx.x & 31) == (unsigned)lane ? (unsigned)(x + 1) : 0u) - 1;
}
// A box of the tensor (x, y, z) to shared memory
__device__ __forceinline__ void lt_tma(uint32_t smem, const CUtensorMap* map, int x, int y, int z, uint32_t bar)
{
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
                 "@e cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n\t}"
                 ::"r"(smem), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void lt_tma(uint32_t smem, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar)
{
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
                 "@e cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}"
                 ::"r"(smem), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}
// Asks for memory to come to L2
__device__ __forceinline__ void lt_prefetch(const void* at, uint32_t bytes)
{
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t@e cp.async.bulk.prefetch.L2.global [%0], %1;\n\t}" ::"l"(at), "r"(bytes) : "memory");
}
__device__ __forceinline__ void lt_expect(uint32_t bar, uint32_t bytes)      // and arrive
{
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t@e mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar), "r"(bytes) : "memory");
}
// N products of 16 channels or tokens each, D += A B, from shared memory; SA, SB: steps of the descriptors
template <int N, int SA, int SB> __device__ __forceinline__ void lt_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add)
{
    asm volatile("{\n\t.reg .pred p, e, t;\n\t.reg .b64 a, b;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.eq.u32 t, 0, 0;\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t"
                 "add.u64 a, %1, %5;\n\tadd.u64 b, %2, %6;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(what), "r"((uint32_t)add), "n"(SA), "n"(SB) : "memory");
    if constexpr (N > 2) lt_mma_ss<N - 2, SA, SB>(d, a + 2 * SA, b + 2 * SB, what, true);
}
__device__ __forceinline__ void lt_init(uint32_t bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }

// 16 bytes to shared memory without waiting; zeros where there is no source
__device__ __forceinline__ void lt_copy16(uint32_t smem, const void* src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void lt_copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Whether any of a group's threads says so: barrier `id` of `threads` threads
__device__ __forceinline__ bool lt_any(int id, int threads, bool mine)
{
    uint32_t any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %3, 0;\n\tbarrier.cta.red.or.pred q, %1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(any) : "r"(id), "r"(threads), "r"((uint32_t)mine) : "memory");
    return any != 0;
}
__device__ __forceinline__ void lt_sync(int id, int threads) { asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// 16-bit values that are infinite or NaN, each of the two of a word, become zero
template <bool BF> __device__ __forceinline__ uint32_t lt_finite2(uint32_t w)
{
    constexpr uint32_t exponent = BF ? 0x7f80u : 0x7c00u;
    if ((w & exponent) == exponent) w &= 0xffff0000u;
    if ((w >> 16 & exponent) == exponent) w &= 0x0000ffffu;
    return w;
}

// Two CTAs of a cluster whose SMs work on one product (cta_group::2): each has its own half of A's rows, of B's columns and of D's rows.  The first of
// the pair issues; barriers that it waits for are its own, and what both wait for is told to both.  (No copy is multicast: each brings its half.)
__device__ __forceinline__ uint32_t lt_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t lt_of_first(uint32_t smem)               // the same place in the pair's first CTA
{
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(smem));
    return at;
}
// A box to this CTA's shared memory; a barrier of either of the two is told
__device__ __forceinline__ void lt_pair_tma(uint32_t smem, const CUtensorMap* map, int x, int y, int z, uint32_t cluster_bar)
{
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
                 "@e cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n\t}"
                 ::"r"(smem), "l"(map), "r"(x), "r"(y), "r"(z), "r"(cluster_bar) : "memory");
}
// For a whole warp, when all its lanes have come: an arrival at a barrier of either CTA.  The first is for what was done in tensor memory (whose own
// fence stands in front of it); the second for what was written to shared memory, too, and holds the warp up for 1300 cycles.
__device__ __forceinline__ void lt_pair_arrive(uint32_t cluster_bar)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void lt_pair_release(uint32_t cluster_bar)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void lt_pair_commit(uint32_t bar)                  // to both
{
    asm volatile("{\n\t.reg .pred e;\n\t.reg .b16 both;\n\tmov.b16 both, 3;\n\telect.sync _|e, 0xffffffff;\n\t"
                 "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], both;\n\t}" ::"r"(bar) : "memory");
}
template <int N, int SA, int SB> __device__ __forceinline__ void lt_pair_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add)
{
    asm volatile("{\n\t.reg .pred p, e, t;\n\t.reg .b64 a, b;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.eq.u32 t, 0, 0;\n\t"
                 "@e tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t"
                 "add.u64 a, %1, %5;\n\tadd.u64 b, %2, %6;\n\t@e tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %3, t;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(what), "r"((uint32_t)add), "n"(SA), "n"(SB) : "memory");
    if constexpr (N > 2) lt_pair_mma_ss<N - 2, SA, SB>(d, a + 2 * SA, b + 2 * SB, what, true);
}
// The same with A in tensor memory, 8 columns a step
template <int N, int SB> __device__ __forceinline__ void lt_pair_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add)
{
    asm volatile("{\n\t.reg .pred p, e, t;\n\t.reg .b32 a;\n\t.reg .b64 b;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.eq.u32 t, 0, 0;\n\t"
                 "@e tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t"
                 "add.u32 a, %1, 8;\n\tadd.u64 b, %2, %5;\n\t@e tcgen05.mma.cta_group::2.kind::f16 [%0], [a], b, %3, t;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(what), "r"((uint32_t)add), "n"(SB) : "memory");
    if constexpr (N > 2) lt_pair_mma_ts<N - 2, SB>(d, a + 16, b + 2 * SB, what, true);
}
// As kv_ended and kv_warp_wait, for barriers that the other CTA arrives at
__device__ __forceinline__ uint32_t lt_pair_ended(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done;
}
__device__ __forceinline__ bool lt_pair_wait(uint32_t bar, uint32_t parity, volatile int* stop)
{
    bool done = false;
#pragma unroll 1
    for (int i = 0; i < 1 << 18 && !done; i++) {
        uint32_t d;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(d) : "r"(bar), "r"(parity) : "memory");
        done = d;
        if (!done && (i & 15) == 15 && *stop) break;
    }
    if (!done) *stop = 1;
    return __all_sync(0xffffffffu, done);
}

// S of 64 rows (tensor memory, 16 lanes of each warp's 32), 32 columns: lane l of the warp gets of its 16 rows the rows l / 4 and l / 4 + 8, and of every
// 8 columns the columns 2 (l % 4) and the next: x[4 k], x[4 k + 1] of the first row and x[4 k + 2], x[4 k + 3] of the second, columns 8 k on.
__device__ __forceinline__ void lt_tmem_load_quads(uint32_t (&x)[16], uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : KV_R8(x, 0), KV_R8(x, 8) : "r"(at) : "memory");
}

// A line of work: items one behind the other, `size(item)` units each.  Every thread of a CTA adds up a stretch of items, and the one in whose
// stretch a unit lies looks for its item.
struct LtStretch {
    int64_t item, before, units, total;     // the stretch's first item, the units in front of it and in it, and in the line
    __device__ __forceinline__ bool holds(int64_t unit) const { return before <= unit && unit < before + units; }
    template <class F> __device__ __forceinline__ void find(int64_t unit, F size)
    {
        for (int64_t n; before + (n = size(item)) <= unit; item++) before += n;
    }
};
// warp_sum: room for a number per warp, which the CTA's next barrier leaves free again
template <int THREADS, class F> __device__ __forceinline__ LtStretch lt_stretch(int64_t items, F size, int64_t* warp_sum)
{
    const int64_t per = (items + THREADS - 1) / THREADS, lo = min(items, threadIdx.x * per), hi = min(items, lo + per);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    LtStretch s = {lo, 0, 0, 0};
    for (int64_t item = lo; item < hi; item++) s.units += size(item);
    s.before = s.units;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, s.before, d);
        if (lane >= d) s.before += v;
    }
    if (lane == 31) warp_sum[warp] = s.before;
    __syncthreads();
    s.before -= s.units;
#pragma unroll
    for (int w = 0; w < THREADS / 32; w++) {
        if (w < warp) s.before += warp_sum[w];
        s.total += warp_sum[w];
    }
    return s;
}
