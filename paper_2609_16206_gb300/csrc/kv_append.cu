// kv_append.cu -- rotary positions and the append to a paged KV cache
// (ctr_kv_append).
//
// A pair (x, y) of a head turns by phi = 2 pi frac(position * turns / 2^64):
// scale * (x cos phi - y sin phi, x sin phi + y cos phi).  The product is a
// 64-bit integer one, exact modulo a turn at any position; its top 32 bits are
// the signed half-turns whose sine and cosine the fp32 functions give within
// 2^-24 of the circle.  Everything is fp32 and rounded once to the cache's type.
//
// Every input is read once and every output written once, so the bound is the
// memory system's (a decode step's few tokens: a launch's latency).  A warp
// takes one token's heads, 16 elements of a head to a lane in two 16-byte
// vectors that hold both halves of its pairs; the sines of a lane's pairs are
// the same in every head and computed once a warp.
#include "decode_internal.cuh"

namespace ctr {
namespace {

constexpr int kThreads = 128;

// sine and cosine of pair i at the position, times scale
__device__ __forceinline__ void turn_of(const AppendParams& P, int i, int64_t position, float& c, float& s)
{
    const uint64_t product = (uint64_t)position * __ldg(reinterpret_cast<const unsigned long long*>(P.rope.turns) + i);
    sincospif((float)(int32_t)(product >> 32) * 0x1p-31f, &s, &c);
    c *= P.rope.scale;
    s *= P.rope.scale;
}

// where a token goes in the cache, -1 for nowhere
__device__ __forceinline__ int64_t cache_offset(const AppendParams& P, int64_t slot)
{
    const int64_t page = slot >> P.page_log2;
    if (slot < 0 || page >= P.cache.n_pages) return -1;
    return page * P.cache.page_stride + (slot & (P.cache.page_tokens - 1)) * P.cache.token_stride;
}

// One element or pair at a time: odd shapes and unaligned views.
template <typename T>
__global__ void __launch_bounds__(kThreads) append_plain_kernel(const AppendParams P)
{
    wait_for_previous_kernels();
    const int64_t t = blockIdx.x;
    const int d = P.cache.head_dim, rot = P.rope.rot_dim, half = rot / 2, kv = P.cache.n_kv_heads;
    const int64_t at = cache_offset(P, P.slots[t]);
    const int64_t position = rot > 0 ? P.positions[t] : 0;
    const int units = half + (d - rot);  // of a head: its pairs, then its other elements
    for (int u = threadIdx.x; u < units; u += kThreads) {
        const bool pair = u < half;
        const int a = !pair ? rot + u - half : P.rope.interleaved ? 2 * u : u;
        const int b = !pair ? a : P.rope.interleaved ? a + 1 : a + half;
        float c = 1.f, s = 0.f;
        if (pair) turn_of(P, u, position, c, s);
        for (int h = 0; h < P.n_q_heads + kv; ++h) {
            const bool is_q = h < P.n_q_heads;
            if (!is_q && at < 0) break;
            const int hk = h - P.n_q_heads;
            const T* src = is_q ? static_cast<const T*>(P.q.ptr) + t * P.q.token_stride + h * P.q.head_stride
                                : static_cast<const T*>(P.k.ptr) + t * P.k.token_stride + hk * P.k.head_stride;
            T* dst = is_q ? static_cast<T*>(P.q_out.ptr) + t * P.q_out.token_stride + h * P.q_out.head_stride
                          : static_cast<T*>(P.cache.k) + at + hk * P.cache.head_stride;
            if (!pair) {
                dst[a] = src[a];
                continue;
            }
            const float x = to_float(src[a]), y = to_float(src[b]);
            dst[a] = from_float<T>(x * c - y * s);
            dst[b] = from_float<T>(x * s + y * c);
        }
    }
    if (at < 0) return;
    for (int h = 0; h < kv; ++h) {
        const T* src = static_cast<const T*>(P.v.ptr) + t * P.v.token_stride + h * P.v.head_stride;
        T* dst = static_cast<T*>(P.cache.v) + at + h * P.cache.head_stride;
        for (int j = threadIdx.x; j < d; j += kThreads) dst[j] = src[j];
    }
}

}  // namespace

cudaError_t launch_append(const AppendParams& p, cudaStream_t stream)
{
    const dim3 grid((unsigned)p.n_tokens);
    if (p.cache.dtype == CTR_BF16)
        return launch_dependent(append_plain_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, 1, stream, p);
    return launch_dependent(append_plain_kernel<__half>, grid, dim3(kThreads), 0, 1, stream, p);
}

}  // namespace ctr
