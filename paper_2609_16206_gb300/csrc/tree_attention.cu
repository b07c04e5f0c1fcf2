// tree_attention.cu -- attention of new tokens over a paged KV cache
// (ctr_tree_attention).
//
// A row's output is a softmax-weighted mean of values, taken in one pass over
// the keys with the running maximum m and sum l of the softmax: a key of score
// s moves m to m' = max(m, s), scales l and the partial output by 2^(m - m')
// and adds 2^(s - m') and 2^(s - m') v.  Scores carry log2 e, so that every
// exponential is a power of two.
#include "decode_internal.cuh"

namespace ctr {
namespace {

constexpr int kThreads = 128;

// the new tokens of sequence b and its length in the cache, both held to their bounds
struct Seq {
    int64_t row0;
    int n_new, len, context;
};
__device__ __forceinline__ Seq seq_of(const AttentionParams& P, int b)
{
    Seq s;
    const int64_t lo = P.q_start[b], hi = P.q_start[b + 1];
    s.row0 = lo < 0 ? 0 : lo;
    int64_t n = hi - lo;
    n = n > P.max_nodes ? P.max_nodes : n;
    n = s.row0 + n > P.n_rows ? P.n_rows - s.row0 : n;
    s.n_new = n < 0 ? 0 : (int)n;
    const int64_t most = (int64_t)P.table_stride << P.page_log2;
    const int64_t len = P.kv_len[b];
    s.len = len < 0 ? 0 : len > most ? (int)most : (int)len;
    s.context = s.len - (int)(hi - lo);
    return s;
}

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

template <typename T>
cudaError_t launch_typed(const AttentionParams& p, cudaStream_t stream)
{
    const dim3 grid((unsigned)(p.n_seqs * p.max_nodes), (unsigned)p.n_q_heads);
    if (p.cache.head_dim == 64) return launch_dependent(attention_kernel<T, 64>, grid, dim3(kThreads), 0, 1, stream, p);
    return launch_dependent(attention_kernel<T, 128>, grid, dim3(kThreads), 0, 1, stream, p);
}

}  // namespace

size_t attention_workspace(const ctr_kv_cache&, int32_t, int32_t, int32_t) { return 256; }

cudaError_t launch_attention(const AttentionParams& p, cudaStream_t stream)
{
    return p.cache.dtype == CTR_BF16 ? launch_typed<__nv_bfloat16>(p, stream) : launch_typed<__half>(p, stream);
}

}  // namespace ctr
