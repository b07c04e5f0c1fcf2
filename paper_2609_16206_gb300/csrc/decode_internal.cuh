// decode_internal.cuh -- declarations shared by the translation units behind
// include/ctr_decode.h (kernel parameter blocks and launchers).  Not part of
// the ABI.
#pragma once

#include <atomic>
#include <cstdint>
#include <cstring>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "../../include/ctr_decode.h"

namespace ctr {

// A launch that may be scheduled while the kernel before it drains; the kernel
// waits for its grid dependencies before its first access.
template <typename... KArgs, typename... Args>
cudaError_t launch_dependent(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t stream,
                             Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)cluster;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    cfg.attrs = attr;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, args...);
    return err != cudaSuccess ? err : cudaGetLastError();
}

// More dynamic shared memory than 48 KB for a kernel, asked for once on each device: `most` for all of its launches.
template <typename Kernel>
cudaError_t allow_shared(Kernel* kernel, int most, std::atomic<uint64_t>& devices)
{
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess) return err;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (devices.load(std::memory_order_acquire) & bit)) return cudaSuccess;
    err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (err == cudaSuccess) devices.fetch_or(bit, std::memory_order_release);
    return err;
}

__device__ __forceinline__ void wait_for_previous_kernels()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// the two 16-bit types
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(float x) { return x; }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
// two values in one 32-bit register, the first in the low half; kExpOne: the unit of both exponents
template <typename T> struct Pair;
template <> struct Pair<__nv_bfloat16> {
    static constexpr uint32_t kExpOne = 0x00800080u;
    static __device__ __forceinline__ float2 split(uint32_t v)
    {
        return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t join(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
};
template <> struct Pair<__half> {
    static constexpr uint32_t kExpOne = 0x04000400u;
    static __device__ __forceinline__ float2 split(uint32_t v)
    {
        __half2 h;
        memcpy(&h, &v, 4);
        return __half22float2(h);
    }
    static __device__ __forceinline__ uint32_t join(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
};

// two fp32 in one 64-bit register, and the operations on both
__device__ __forceinline__ uint64_t pack(float a, float b) { return (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a); }
__device__ __forceinline__ float low_of(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float high_of(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// sign bits set where a half is infinite or NaN: an exponent of all ones carries into it
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t v)
{
    return ((v & 0x7fff7fffu) + Pair<T>::kExpOne) & 0x80008000u;
}

// ---------------------------------------------------------------- cache append
struct AppendParams {
    ctr_kv_cache cache;
    ctr_rope rope;
    ctr_rows q, k, v, q_out;
    int64_t n_tokens;
    int32_t n_q_heads;
    int32_t page_log2;
    const int64_t* positions;
    const int64_t* slots;
};
cudaError_t launch_append(const AppendParams& p, cudaStream_t stream);

// ---------------------------------------------------------------- attention
struct AttentionParams {
    ctr_kv_cache cache;
    ctr_rows q, out;
    int64_t n_rows;
    int32_t n_q_heads, group, n_seqs, max_nodes, table_stride, page_log2;
    const int32_t* q_start;
    const int32_t* kv_len;
    const int32_t* page_table;
    const uint64_t* tree_mask;
    float scale_log2;           // scale times log2 e
    uint32_t group_magic;       // ceil(2^20 / group): r / group = r * magic >> 20 for the rows r < 64 group
    float* lse;
    int32_t* status;
    unsigned char* ws;
};
size_t attention_workspace(const ctr_kv_cache& cache, int32_t n_q_heads, int32_t n_seqs, int32_t max_nodes);
cudaError_t launch_attention(const AttentionParams& p, cudaStream_t stream);

// ---------------------------------------------------------------- sampling
struct SampleParams {
    const void* logits;
    int32_t dtype, vocab;
    int64_t row_stride, n_rows;
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    const float* u;
    int32_t* token;
    float* logprob;
    int32_t* n_kept;
    uint64_t minus_zeros;       // two fp32 -0 (see Scale in sample.cu)
};
cudaError_t launch_sample(const SampleParams& p, cudaStream_t stream);

}  // namespace ctr
