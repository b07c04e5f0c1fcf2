// tree_attention.cu -- attention of new tokens over a paged KV cache
// (ctr_tree_attention): the choice of the kernel, the caches' TMA maps, and the
// merge of items that several blocks worked on.
//
// A row's output is a softmax-weighted mean of values, taken in one pass over
// the keys with the running maximum m and sum l of the softmax: a key of score
// s moves m to m' = max(m, s), scales l and the partial output by 2^(m - m')
// and adds 2^(s - m') and 2^(s - m') v.  Scores carry log2 e, so that every
// exponential is a power of two.  Parts of a row's keys join the same way.
#include "attention_internal.cuh"

namespace ctr {
namespace {

constexpr int kThreads = 128;

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) attention_kernel(const AttentionParams P)
{
    constexpr int kPer = D / 32;  // dimensions of a lane
    __shared__ float sm_o[kThreads / 32][D], sm_m[kThreads / 32], sm_l[kThreads / 32];
    wait_for_previous_kernels();
    const int b = blockIdx.x / P.max_nodes, node = blockIdx.x % P.max_nodes, h = blockIdx.y;
    const Seq s = seq_of(P, b);
    if (node >= s.n_new) return;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int64_t row = s.row0 + node;
    const uint64_t mask = P.tree_mask ? P.tree_mask[row] : ~0ull >> (63 - node);
    const int64_t head = (h / P.group) * P.cache.head_stride;
    const T* q = static_cast<const T*>(P.q.ptr) + row * P.q.token_stride + h * P.q.head_stride + lane * kPer;
    float qv[kPer], o[kPer], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        qv[j] = to_float(q[j]);
        o[j] = 0.f;
    }
    for (int p = wid; p < s.len; p += kThreads / 32) {
        const int n = p - s.context;
        if (n >= 0 && !(mask >> n & 1)) continue;
        const int64_t page = P.page_table[(int64_t)b * P.table_stride + (p >> P.page_log2)];
        const bool there = page >= 0 && page < P.cache.n_pages;
        const int64_t at = page * P.cache.page_stride + head + (p & (P.cache.page_tokens - 1)) * P.cache.token_stride + lane * kPer;
        float dot = 0.f, v[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            dot += qv[j] * (there ? to_float(static_cast<const T*>(P.cache.k)[at + j]) : 0.f);
            v[j] = there ? to_float(static_cast<const T*>(P.cache.v)[at + j]) : 0.f;
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) dot += __shfl_xor_sync(~0u, dot, off);
        dot *= P.scale_log2;
        const float mn = fmaxf(m, dot), fix = m == -INFINITY ? 0.f : exp2f(m - mn), w = exp2f(dot - mn);
        l = l * fix + w;
#pragma unroll
        for (int j = 0; j < kPer; ++j) o[j] = o[j] * fix + w * v[j];
        m = mn;
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) sm_o[wid][lane * kPer + j] = o[j];
    sm_m[wid] = m;
    sm_l[wid] = l;
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) top = fmaxf(top, sm_m[w]);
    float sum = 0.f, part[kThreads / 32];
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        part[w] = sm_m[w] == -INFINITY ? 0.f : exp2f(sm_m[w] - top);
        sum += part[w] * sm_l[w];
    }
    T* out = static_cast<T*>(P.out.ptr) + row * P.out.token_stride + h * P.out.head_stride;
    for (int j = threadIdx.x; j < D; j += kThreads) {
        float acc = 0.f;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) acc += part[w] * sm_o[w][j];
        out[j] = from_float<T>(sum > 0.f ? acc / sum : 0.f);
    }
    if (threadIdx.x == 0 && P.lse)
        P.lse[row * P.n_q_heads + h] = sum > 0.f ? (top + log2f(sum)) * 0x1.62e43p-1f : -INFINITY;
}

// One row of an item that several blocks worked on: their parts in the order of the blocks, a fourth of them to a warp.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) merge_kernel(const AttentionParams P, int blocks, int rows)
{
    constexpr int kPer = D / 32;
    __shared__ float sm_o[kThreads / 32][D], sm_m[kThreads / 32], sm_l[kThreads / 32];
    wait_for_previous_kernels();
    const SplitSlot d = split_slots(P)[blockIdx.x];
    if (d.b < 0) return;
    const Seq s = seq_of(P, d.b);
    const int r = blockIdx.y;
    if (r >= s.n_new * P.group) return;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, first = blockIdx.x, n = d.last - first + 1;
    float o[kPer], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) o[j] = 0.f;
    const int per = (n + kThreads / 32 - 1) / (kThreads / 32);
#pragma unroll 4
    for (int i = wid * per; i < min((wid + 1) * per, n); ++i) {
        const float* part = part_of_item(P, blocks, rows, D, first + i, i == 0 ? 1 : 0);
        const float pm = part[r], pl = part[rows + r];
        float po[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) po[j] = part[2 * rows + (size_t)r * D + lane * kPer + j];
        const float mn = fmaxf(m, pm), fa = m == -INFINITY ? 0.f : exp2_fast(m - mn), fb = pm == -INFINITY ? 0.f : exp2_fast(pm - mn);
        l = l * fa + pl * fb;
#pragma unroll
        for (int j = 0; j < kPer; ++j) o[j] = o[j] * fa + (pm == -INFINITY ? 0.f : po[j] * fb);
        m = mn;
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) sm_o[wid][lane * kPer + j] = o[j];
    sm_m[wid] = m;
    sm_l[wid] = l;
    __syncthreads();
    float top = -INFINITY, sum = 0.f, part[kThreads / 32];
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) top = fmaxf(top, sm_m[w]);
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        part[w] = sm_m[w] == -INFINITY ? 0.f : exp2_fast(sm_m[w] - top);
        sum += part[w] * sm_l[w];
    }
    const int node = r / P.group;
    const int64_t row = s.row0 + node, h = d.h * P.group + r - node * P.group;
    T* out = static_cast<T*>(P.out.ptr) + row * P.out.token_stride + h * P.out.head_stride;
    for (int j = threadIdx.x; j < D; j += kThreads) {
        float acc = 0.f;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) acc += part[w] == 0.f ? 0.f : part[w] * sm_o[w][j];
        out[j] = from_float<T>(sum > 0.f ? acc / sum : 0.f);
    }
    if (threadIdx.x == 0 && P.lse) P.lse[row * P.n_q_heads + h] = sum > 0.f ? (top + log2f(sum)) * 0x1.62e43p-1f : -INFINITY;
}

template <typename T>
cudaError_t launch_typed(const AttentionParams& p, cudaStream_t stream)
{
    const dim3 grid((unsigned)(p.n_seqs * p.max_nodes), (unsigned)p.n_q_heads);
    if (p.cache.head_dim == 64) return launch_dependent(attention_kernel<T, 64>, grid, dim3(kThreads), 0, 1, stream, p);
    return launch_dependent(attention_kernel<T, 128>, grid, dim3(kThreads), 0, 1, stream, p);
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// the driver's encoder of tensor maps, looked up once
EncodeTiled encoder()
{
    static const EncodeTiled found = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &r) != cudaSuccess ||
            r != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<EncodeTiled>(f);
    }();
    return found;
}

constexpr int kStreamRows = 32;  // most rows of a KV head that the streaming kernel takes

}  // namespace

// The cache as a 4-d tensor (dimension, token of a page, head, page) of boxes of 64 dimensions x box_tokens tokens;
// a page outside it reads as zeros.
cudaError_t make_cache_maps(const AttentionParams& p, int box_tokens, CUtensorMap* k, CUtensorMap* v)
{
    const EncodeTiled encode = encoder();
    if (!encode) return cudaErrorNotSupported;
    const ctr_kv_cache& c = p.cache;
    const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_tokens, (cuuint64_t)c.n_kv_heads, (cuuint64_t)c.n_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)c.token_stride * 2, (cuuint64_t)c.head_stride * 2, (cuuint64_t)c.page_stride * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)box_tokens, 1, 1}, step[4] = {1, 1, 1, 1};
    const CUtensorMapDataType type = c.dtype == CTR_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    for (int i = 0; i < 2; ++i)
        if (encode(i ? v : k, type, 4, i ? c.v : c.k, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    return cudaSuccess;
}

cudaError_t launch_merge(const AttentionParams& p, int blocks, int rows, cudaStream_t stream)
{
    const dim3 grid((unsigned)blocks, (unsigned)(p.group * p.max_nodes));
    const bool bf = p.cache.dtype == CTR_BF16, wide = p.cache.head_dim == 128;
    auto kernel = bf ? (wide ? merge_kernel<__nv_bfloat16, 128> : merge_kernel<__nv_bfloat16, 64>)
                     : (wide ? merge_kernel<__half, 128> : merge_kernel<__half, 64>);
    return launch_dependent(kernel, grid, dim3(kThreads), 0, 1, stream, p, blocks, rows);
}

size_t attention_workspace(const ctr_kv_cache& cache, int32_t n_q_heads, int32_t, int32_t max_nodes)
{
    const int rows = n_q_heads / cache.n_kv_heads * max_nodes;
    if (rows > kStreamRows) return 256;
    const int blocks = stream_blocks();
    return slots_bytes(blocks) + (size_t)blocks * 2 * part_floats(rows > 16 ? 32 : 16, cache.head_dim) * sizeof(float);
}

cudaError_t launch_attention(const AttentionParams& p, cudaStream_t stream)
{
    if (p.group * p.max_nodes <= kStreamRows) return launch_stream(p, stream);
    return p.cache.dtype == CTR_BF16 ? launch_typed<__nv_bfloat16>(p, stream) : launch_typed<__half>(p, stream);
}

}  // namespace ctr
