// attention_internal.cuh -- what the two attention kernels share: a sequence's
// bounds, the split of the work over the grid, the partial results and their
// merge, TMA and mbarrier access.
#pragma once

#include <cuda.h>

#include "decode_internal.cuh"

namespace ctr {

constexpr unsigned kWaitLimit = 1u << 22;  // bounded mbarrier polling (a wait is a few microseconds)

// the new tokens of sequence b and its length in the cache, both held to their bounds
struct Seq {
    int64_t row0;
    int n_new, len, context;
};
__device__ __forceinline__ Seq seq_of(const AttentionParams& P, int b)
{
    Seq s;
    const int64_t lo = __ldg(P.q_start + b), hi = __ldg(P.q_start + b + 1);
    s.row0 = lo < 0 ? 0 : lo;
    int64_t n = hi - lo;
    n = n > P.max_nodes ? P.max_nodes : n;
    n = s.row0 + n > P.n_rows ? P.n_rows - s.row0 : n;
    s.n_new = n < 0 ? 0 : (int)n;
    const int64_t most = (int64_t)P.table_stride << P.page_log2;
    const int64_t len = __ldg(P.kv_len + b);
    s.len = len < 0 ? 0 : len > most ? (int)most : (int)len;
    s.context = s.len - (int)(hi - lo);
    return s;
}

// ---------------------------------------------------------------- shared memory, mbarriers, TMA
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// false where the bound ran out
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity)
{
    uint32_t done = 0;
    for (unsigned it = 0; it < kWaitLimit && !done; ++it)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(bar), "r"(parity)
            : "memory");
    return done != 0;
}
// a box of a cache's map: 64 dimensions from x (0 or 64), tokens of a page from y, one head, one page
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int head, int page)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(head), "r"(page), "r"(bar)
        : "memory");
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// ---------------------------------------------------------------- the split of the work
// A sequence's KV head is an item of ceil(len / kUnit) units, one at least; the units of all items, in order, are cut
// into equal ranges, one a block.  A range holds whole items and at most two parts of items, its first and last;
// such a part leaves its sums in the block's first (an item begun by an earlier block) or second slot of the
// workspace, and the merge kernel joins the slots of an item in the order of its blocks.
struct SplitSlot {           // the item that a block begins and does not end
    int32_t b, h, last;      // sequence (-1: none), KV head, the block that ends it
    int32_t reserved;
};

template <int kUnit>
__device__ __forceinline__ int64_t units_of(const Seq& s)
{
    return s.n_new == 0 ? 0 : s.len <= kUnit ? 1 : (s.len + kUnit - 1) / kUnit;
}

// The range of block c: `count` units from unit `begin` of `total` on, which is unit `within` of sequence b0 (over
// all of its KV heads); `blocks`, the grid's on entry, becomes the number of blocks with work, each of which has a
// unit at least.  By all threads of the block; scratch: kThreads / 32 + 4 words of 64 bits.
template <int kUnit, int kThreads>
__device__ void find_range(const AttentionParams& P, int c, int64_t* scratch, int& blocks, int64_t& total, int64_t& begin,
                           int64_t& count, int& b0, int64_t& within)
{
    constexpr int kWarps = kThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int per = (P.n_seqs + kThreads - 1) / kThreads;
    const int first = min(tid * per, P.n_seqs), last = min(first + per, P.n_seqs);
    int64_t mine = 0;
    for (int b = first; b < last; ++b) mine += units_of<kUnit>(seq_of(P, b)) * P.cache.n_kv_heads;
    int64_t sum = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int64_t v = __shfl_up_sync(~0u, sum, off);
        if (lane >= off) sum += v;
    }
    if (lane == 31) scratch[wid] = sum;
    __syncthreads();
    int64_t all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w == wid) sum += all;
        all += scratch[w];
    }
    total = all;
    if (all < blocks) blocks = (int)all;
    count = 0;
    if (c >= blocks) return;  // the whole block
    begin = all * c / blocks;
    count = all * (c + 1) / blocks - begin;
    int64_t at = sum - mine;
    if (at <= begin && begin < sum) {
        for (int b = first; b < last; ++b) {
            const int64_t n = units_of<kUnit>(seq_of(P, b)) * P.cache.n_kv_heads;
            if (begin < at + n) {
                scratch[kWarps] = b;
                scratch[kWarps + 1] = begin - at;
                break;
            }
            at += n;
        }
    }
    __syncthreads();
    b0 = (int)scratch[kWarps];
    within = scratch[kWarps + 1];
}

// the block whose range holds unit u: the largest c with floor(total c / blocks) <= u (blocks <= total)
__device__ __forceinline__ int block_of(int64_t u, int64_t total, int blocks)
{
    return (int)(((u + 1) * blocks - 1) / total);
}

// Workspace: blocks SplitSlots, then per block and slot the partial sums of up to `rows` rows: their maxima and
// weight sums, and `rows` x head_dim fp32 outputs.
__host__ __device__ __forceinline__ size_t slots_bytes(int blocks) { return ((size_t)blocks * sizeof(SplitSlot) + 255) / 256 * 256; }
__host__ __device__ __forceinline__ size_t part_floats(int rows, int d) { return (size_t)rows * (d + 2); }
__device__ __forceinline__ SplitSlot* split_slots(const AttentionParams& P) { return reinterpret_cast<SplitSlot*>(P.ws); }
__device__ __forceinline__ float* part_of_item(const AttentionParams& P, int blocks, int rows, int d, int block, int slot)
{
    return reinterpret_cast<float*>(P.ws + slots_bytes(blocks)) + (size_t)(2 * block + slot) * part_floats(rows, d);
}

cudaError_t make_cache_maps(const AttentionParams& p, int box_tokens, CUtensorMap* k, CUtensorMap* v);
cudaError_t launch_merge(const AttentionParams& p, int blocks, int rows, cudaStream_t stream);

int stream_blocks();  // of the kernel for few rows a KV head
cudaError_t launch_stream(const AttentionParams& p, cudaStream_t stream);

}  // namespace ctr
