// sample.cu -- a token per row of logits (ctr_sample).
//
// The weight of a logit x is the integer w = round(2^31 2^y), y = (x - max)
// log2(e) / temperature, with 2^y by a degree-5 polynomial whose fp32 steps are
// each rounded on their own: every sum of weights is then an exact integer,
// whatever its order, and the token is a function of the inputs alone.
#include "decode_internal.cuh"

namespace ctr {
namespace {

constexpr int kThreads = 512;
constexpr uint32_t kEmptyKey = 0;  // of -inf and NaN

// Monotone 32-bit key of a logit: larger logits have larger keys, equal ones
// (-0 and 0 among them) equal keys, -inf and NaN the key 0.
__device__ __forceinline__ uint32_t key_of(float x)
{
    if (!(x > -INFINITY)) return kEmptyKey;
    const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// 2^f on [-1/2, 1/2] as 1 + f (c1 + f (c2 + ...)): a minimax fit with constant term 1, relative error 9.2e-8
// before rounding and 1.9e-7 with every fp32 step rounded
__device__ __forceinline__ uint32_t weight_of(float x, float top, float rate)
{
    if (!(x > -INFINITY)) return 0;
    const float y = x == top ? 0.f : fmaxf(__fmul_rn(__fsub_rn(x, top), rate), -64.f);
    const float k = rintf(y), f = __fsub_rn(y, k);
    float p = 0x1.5bba14p-10f;
    p = __fadd_rn(__fmul_rn(p, f), 0x1.3cea88p-7f);
    p = __fadd_rn(__fmul_rn(p, f), 0x1.c6b752p-5f);
    p = __fadd_rn(__fmul_rn(p, f), 0x1.ebf9bcp-3f);
    p = __fadd_rn(__fmul_rn(p, f), 0x1.62e42ap-1f);
    p = __fadd_rn(__fmul_rn(p, f), 1.f);
    return __float2uint_rn(__fmul_rn(p, __uint_as_float((uint32_t)((int)k + 31 + 127) << 23)));
}

// floor(total part / 2^31)
__device__ __forceinline__ uint64_t share_of(uint64_t total, uint32_t part)
{
    return (total >> 31) * part + (((total & 0x7fffffffu) * part) >> 31);
}
__device__ __forceinline__ uint32_t part_of(float x, uint32_t most)
{
    const uint32_t v = __float2uint_rd(fminf(fmaxf(x, 0.f), 1.f) * 0x1p31f);  // a NaN gives 0
    return v < most ? v : most;
}

struct Tally {
    uint64_t mass;
    uint32_t count, top;
};
__device__ __forceinline__ Tally join(const Tally& a, const Tally& b)
{
    return Tally{a.mass + b.mass, a.count + b.count, a.top > b.top ? a.top : b.top};
}

__device__ Tally block_tally(Tally v, Tally* scratch)
{
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
        v = join(v, Tally{__shfl_xor_sync(~0u, v.mass, off), __shfl_xor_sync(~0u, v.count, off),
                          __shfl_xor_sync(~0u, v.top, off)});
    if (lane == 0) scratch[wid] = v;
    __syncthreads();
    v = scratch[lane & (kThreads / 32 - 1)];
#pragma unroll
    for (int off = kThreads / 64; off > 0; off >>= 1)
        v = join(v, Tally{__shfl_xor_sync(~0u, v.mass, off), __shfl_xor_sync(~0u, v.count, off),
                          __shfl_xor_sync(~0u, v.top, off)});
    __syncthreads();
    return v;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleParams P)
{
    __shared__ Tally scratch[kThreads / 32];
    __shared__ uint64_t sums[kThreads];
    wait_for_previous_kernels();
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(P.logits) + row * P.row_stride;
    const int V = P.vocab, tid = threadIdx.x;
    auto key_at = [&](int i) { return key_of(to_float(x[i])); };

    // the row's largest logit
    Tally t = {0, 0, 0};
    for (int i = tid; i < V; i += kThreads) t.top = max(t.top, key_at(i));
    const uint32_t top_key = block_tally(t, scratch).top;
    if (top_key == kEmptyKey) {
        if (tid == 0) {
            P.token[row] = -1;
            if (P.logprob) P.logprob[row] = -INFINITY;
            if (P.n_kept) P.n_kept[row] = 0;
        }
        return;
    }
    const float top = value_of(top_key);
    const float temperature = P.temperature[row];
    const bool greedy = !(temperature > 0.f);
    const float rate = greedy ? 1.f : fminf(__fdiv_rn(0x1.715476p+0f, temperature), 3e38f);
    const int32_t k_in = P.top_k ? P.top_k[row] : 0;
    const uint32_t k = greedy ? 1u : k_in > 0 ? (uint32_t)k_in : 0xffffffffu;
    const uint32_t p_part = P.top_p && P.top_p[row] < 1.f ? part_of(P.top_p[row], 0x7fffffffu) : 0x80000000u;
    const uint32_t least = P.min_p ? max(1u, part_of(P.min_p[row], 0x80000000u)) : 1u;

    // The kept tokens are those before a cut in the order: keys above cut_key, and those equal to it up to cut_index.
    uint32_t cut_key = 1;
    int cut_index = V - 1;
    auto in_cut = [&](uint32_t key, int i) { return key > cut_key || (key == cut_key && i <= cut_index); };
    auto tally_from = [&](uint32_t from) {  // over the cut's keys >= from
        Tally s = {0, 0, 0};
        for (int i = tid; i < V; i += kThreads) {
            const uint32_t key = key_at(i);
            if (key >= from && in_cut(key, i)) s = join(s, Tally{weight_of(value_of(key), top, rate), 1, 0});
        }
        return block_tally(s, scratch);
    };
    // moves the cut to the first tokens of the order that reach `count` tokens or `mass`
    auto cut_at = [&](uint32_t count, uint64_t mass) {
        uint32_t lo = cut_key, hi = top_key;  // the largest key from which on the goal is reached
        while (lo < hi) {
            const uint32_t mid = hi - (hi - lo) / 2;
            const Tally s = tally_from(mid);
            if (s.count >= count || s.mass >= mass) lo = mid;
            else hi = mid - 1;
        }
        const Tally above = lo == 0xffffffffu ? Tally{0, 0, 0} : tally_from(lo + 1);
        const uint32_t w = weight_of(value_of(lo), top, rate);
        // of the tokens equal to it, those still needed, by index
        uint64_t need = count - above.count;
        if (w > 0 && mass != ~0ull) {
            const uint64_t by_mass = mass > above.mass ? (mass - above.mass + w - 1) / w : 0;
            need = by_mass < need ? by_mass : need;
        }
        if (need < 1 && above.count == 0) need = 1;
        int a = -1, b = lo == cut_key ? cut_index : V - 1;  // the smallest index with `need` of them at or below
        while (a + 1 < b) {
            const int mid = a + (b - a) / 2;
            Tally s = {0, 0, 0};
            for (int i = tid; i <= mid; i += kThreads) s.count += key_at(i) == lo;
            if (block_tally(s, scratch).count >= need) b = mid;
            else a = mid;
        }
        cut_key = lo;
        cut_index = need == 0 ? -1 : b;
    };
    if (k != 0xffffffffu) cut_at(k, ~0ull);
    if (p_part < 0x80000000u && !greedy) {
        const uint64_t goal = share_of(tally_from(1).mass, p_part);
        cut_at(0xffffffffu, goal > 0 ? goal : 1);
    }

    // the kept tokens' weights, a contiguous part of the vocabulary to a thread
    const int per = (V + kThreads - 1) / kThreads;
    const int begin = min(tid * per, V), end = min(begin + per, V);
    auto kept_weight = [&](int i) {
        const uint32_t key = key_at(i);
        if (key == kEmptyKey || !in_cut(key, i)) return 0u;
        const uint32_t w = weight_of(value_of(key), top, rate);
        return w >= least ? w : 0u;
    };
    Tally s = {0, 0, 0};
    for (int i = begin; i < end; ++i) {
        const uint32_t w = kept_weight(i);
        s.mass += w;
        s.count += w > 0;
    }
    sums[tid] = s.mass;
    const Tally all = block_tally(s, scratch);
    const uint64_t goal = share_of(all.mass, part_of(P.u[row], 0x7fffffffu));
    uint64_t before = 0;
    for (int i = 0; i < tid; ++i) before += sums[i];
    if (before <= goal && goal < before + s.mass) {
        for (int i = begin; i < end; ++i) {
            const uint32_t w = kept_weight(i);
            before += w;
            if (before > goal) {
                P.token[row] = i;
                if (P.logprob) P.logprob[row] = (float)log((double)w / (double)all.mass);
                if (P.n_kept) P.n_kept[row] = (int32_t)all.count;
                break;
            }
        }
    }
}

}  // namespace

cudaError_t launch_sample(const SampleParams& p, cudaStream_t stream)
{
    const dim3 grid((unsigned)p.n_rows);
    if (p.dtype == CTR_BF16) return launch_dependent(sample_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, 1, stream, p);
    if (p.dtype == CTR_F16) return launch_dependent(sample_kernel<__half>, grid, dim3(kThreads), 0, 1, stream, p);
    return launch_dependent(sample_kernel<float>, grid, dim3(kThreads), 0, 1, stream, p);
}

}  // namespace ctr
