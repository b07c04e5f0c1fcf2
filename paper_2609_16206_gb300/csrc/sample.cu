// sample.cu -- a token per row of logits (ctr_sample).
//
// The weight of a logit x is the integer w = round(2^31 2^y), y = (x - max)
// log2(e) / temperature, with 2^y by a degree-5 polynomial whose fp32 steps are
// each rounded on their own: every sum of weights is then an exact integer,
// whatever its order, and the token is a function of the inputs alone.
//
// A cluster of blocks holds a row in its shared memory, read once by bulk
// copies; everything after is passes over that copy and exchanges of a few
// words over the cluster.  The kept tokens are the ones before a cut in the
// order (falling logits, then index):
//   * few of them (top-k up to kList, or a nucleus that is): every warp shows
//     the largest of its lanes' maxima to the cluster, and the k-th largest of
//     those is a bound that at least k logits reach and not many more do; those
//     go to the first block, which ranks them;
//   * a nucleus cut off by min-p anyway needs no cut: the mass of what min-p
//     keeps, summed with the whole row's, shows it;
//   * else the cut is found from the masses (or counts) of 512 bins of y, then
//     of 512 parts of the bin that holds it, then by bisection over the part's
//     keys, and over equal keys by index.
// Warps take contiguous runs of a block's part, so that the warps' sums say
// where the drawn token lies, and only that run is gone through again.
#include "decode_internal.cuh"

namespace ctr {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kList = 256;          // tokens that the first block ranks
constexpr int kGather = 1024;       // candidates of the cluster, an equal share of them to a block
constexpr int kBins = 512;
constexpr int kPieces = 4;          // of a block's part of the row, each a bulk copy
constexpr uint32_t kEmptyKey = 0;   // of -inf and NaN
constexpr unsigned kWaitLimit = 1u << 20;

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

// ---------------------------------------------------------------- weights
__device__ __forceinline__ uint64_t pack(float a, float b) { return (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a); }
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

// What a row's weights need: its maximum, the rate, and the two fp32 -0 that make a fused multiply-add a product
// rounded on its own (from the kernel's parameters: a plain product the assembler contracts into the sum behind it).
struct Scale {
    float top, rate;
    uint64_t mz;
};

// y = max((x - top) rate, -64) of two logits; NaN, and -inf at a rate of 0, give -64
__device__ __forceinline__ void exponents(const Scale& s, float x0, float x1, float& y0, float& y1)
{
    const uint64_t y = fma2(add2(pack(x0, x1), pack(-s.top, -s.top)), pack(s.rate, s.rate), s.mz);
    y0 = fmaxf(__uint_as_float((uint32_t)y), -64.f);
    y1 = fmaxf(__uint_as_float((uint32_t)(y >> 32)), -64.f);
}

// round(2^31 2^y): y = k + f with k its nearest integer (by adding 1.5 2^23, whose low bits are then k), 2^f =
// 1 + f (c1 + f (c2 + ...)), a minimax fit on [-1/2, 1/2] with constant term 1: relative error 9.2e-8 before
// rounding and 1.9e-7 with every fp32 step rounded.
__device__ __forceinline__ void weights(const Scale& s, float y0, float y1, uint32_t& w0, uint32_t& w1)
{
    const uint64_t y = pack(y0, y1), magic = pack(0x1.8p+23f, 0x1.8p+23f);
    const uint64_t t = add2(y, magic), k = add2(t, pack(-0x1.8p+23f, -0x1.8p+23f));
    const uint64_t f = fma2(k, pack(-1.f, -1.f), y);
    uint64_t p = pack(0x1.5bba14p-10f, 0x1.5bba14p-10f);
    p = add2(fma2(p, f, s.mz), pack(0x1.3cea88p-7f, 0x1.3cea88p-7f));
    p = add2(fma2(p, f, s.mz), pack(0x1.c6b752p-5f, 0x1.c6b752p-5f));
    p = add2(fma2(p, f, s.mz), pack(0x1.ebf9bcp-3f, 0x1.ebf9bcp-3f));
    p = add2(fma2(p, f, s.mz), pack(0x1.62e42ap-1f, 0x1.62e42ap-1f));
    p = add2(fma2(p, f, s.mz), pack(1.f, 1.f));
    w0 = __float2uint_rn(__uint_as_float((uint32_t)p + ((uint32_t)t << 23) + (31u << 23)));
    w1 = __float2uint_rn(__uint_as_float((uint32_t)(p >> 32) + ((uint32_t)(t >> 32) << 23) + (31u << 23)));
}
__device__ __forceinline__ uint32_t weight_of(const Scale& s, float x)
{
    float y0, y1;
    uint32_t w0, w1;
    exponents(s, x, x, y0, y1);
    weights(s, y0, y1, w0, w1);
    return w0;
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

// ---------------------------------------------------------------- blocks and clusters
struct Sums {  // of weights and a count
    uint64_t a, b, c;
    uint32_t n;
};
struct Words {  // two maxima and a count
    uint32_t top, high, n;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void remote_store(uint32_t addr, uint64_t v)
{
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ void remote_store32(uint32_t addr, uint32_t v)
{
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ uint32_t remote_load(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
struct __align__(16) Shared {
    uint64_t gather[kGather];       // first block: (key, ~index) of the candidates
    uint64_t list[kGather];         // the same without gaps
    uint32_t weight[kGather];       // theirs
    uint32_t kept[kGather];         // the same, 0 where not kept
    uint32_t bins[3][kBins];        // low and high halves of the masses, counts
    Sums warp[kWarps];
    Words warp_words[kWarps];
    Sums peers[2][kMaxCluster];     // exchanges alternate between the two
    Words peer_words[2][kMaxCluster];
    uint32_t shown[kThreads];       // the largest maxima of every warp of the cluster
    uint64_t warp_mass[kWarps];     // what each warp's run holds of the kept tokens
    uint64_t found[3];
    uint32_t counts[kMaxCluster];   // candidates of each block
    uint32_t n_mine, n_list;
    uint64_t bar[kPieces];
};

// ln(w / mass) for 0 < w <= mass < 2^49, to about half a unit of fp32: the quotient as the sum q + r of two fp32, q =
// 2^e m with m in [0.7, 1.42), ln m = 2 atanh((m - 1) / (m + 1)) by its series, whose first term is carried in two.
__device__ __forceinline__ float log_share(uint32_t w, uint64_t mass)
{
    const float wh = __uint2float_rn(w), wl = (float)(int32_t)(w - (uint32_t)(uint64_t)wh);
    const float mh = __ull2float_rn(mass), ml = (float)(int64_t)(mass - (uint64_t)mh);
    const float q = wh / mh, r = (fmaf(-q, mh, wh) + (wl - q * ml)) / mh;
    if (w == mass) return 0.f;
    const uint32_t bits = __float_as_uint(q);
    int e = (int)(bits >> 23) - 127;
    float m = __uint_as_float((bits & 0x7fffffu) | 0x3f800000u);
    if (m > 1.41421354f) {
        m *= 0.5f;
        e += 1;
    }
    const float n = m - 1.f, d = m + 1.f, dl = n - (d - 2.f);  // m + 1 = d + dl
    const float s1 = n / d, s2 = (fmaf(-s1, d, n) - s1 * dl) / d, z = s1 * s1;
    float p = 2.f / 13.f;
    p = fmaf(p, z, 2.f / 11.f);
    p = fmaf(p, z, 2.f / 9.f);
    p = fmaf(p, z, 2.f / 7.f);
    p = fmaf(p, z, 2.f / 5.f);
    p = fmaf(p, z, 2.f / 3.f);
    const float small = fmaf(p * z, s1, 2.f * s2) + r / q;
    const float a = (float)e * 0x1.62e4p-1f, b = 2.f * s1;  // ln 2 in 16 bits and the rest: e times the first is exact
    const float sum = a + b, t = sum - a, err = (a - (sum - t)) + (b - t);
    return sum + (err + fmaf((float)e, 0x1.7f7d1cp-20f, small));
}

template <typename T> struct Vec {  // logits of 16 bytes
    static constexpr int kN = 8;
    static __device__ __forceinline__ void split(const uint4& v, float (&x)[8])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = Pair<T>::split(w[i]);
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
    static __device__ __forceinline__ T lowest() { return from_float<T>(-INFINITY); }
};
template <> struct Vec<float> {
    static constexpr int kN = 4;
    static __device__ __forceinline__ void split(const uint4& v, float (&x)[4])
    {
        x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ float lowest() { return -INFINITY; }
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const SampleParams P)
{
    constexpr int kN = Vec<T>::kN;
    __shared__ Shared sm;
    extern __shared__ __align__(16) unsigned char part_smem[];
    uint4* part = reinterpret_cast<uint4*>(part_smem);
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const uint32_t rank = cluster_rank(), blocks = cluster_size();
    const int64_t row = blockIdx.x / blocks;

    if (tid == 0) {
        for (int i = 0; i < kPieces; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&sm.bar[i])) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        sm.n_mine = sm.n_list = 0;
    }
    wait_for_previous_kernels();

    // ---- this block's part of the row, in the 16-byte vectors of memory: logit i is element i + shift of them
    const T* x = static_cast<const T*>(P.logits) + row * P.row_stride;
    const int shift = (int)(((uintptr_t)x & 15u) / sizeof(T));
    const int n_vec = (P.vocab + shift + kN - 1) / kN, per = (n_vec + (int)blocks - 1) / (int)blocks;
    const int v0 = min((int)rank * per, n_vec), count = min(per, n_vec - v0);
    const int base = v0 * kN - shift;                       // index of the part's first element
    const int whole0 = v0 == 0 && shift > 0 ? 1 : 0;        // vectors that lie inside the row
    const int whole1 = v0 + count == n_vec && (P.vocab + shift) % kN != 0 ? count - 1 : count;
    const int chunk = (per + kWarps - 1) / kWarps;          // vectors of a warp's run
    const int piece = chunk * (kWarps / kPieces);
    __syncthreads();
    if (tid == 0) {
        for (int i = 0; i < kPieces; ++i) {
            const int a = max(i * piece, whole0), b = min((i + 1) * piece, whole1);
            const uint32_t bytes = b > a ? (uint32_t)(b - a) * 16u : 0u, bar = smem_u32(&sm.bar[i]);
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
            if (bytes)
                asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(part + a)),
                             "l"(x + base + (int64_t)a * kN), "r"(bytes), "r"(bar)
                             : "memory");
        }
    }
    // the row's ragged ends, -inf outside it
    for (int i = tid; i < 2 * kN; i += kThreads) {
        const int v = i < kN ? 0 : count - 1, e = i % kN, at = base + v * kN + e;
        const bool ragged = count > 0 && (i < kN ? whole0 == 1 : whole1 < count && !(count == 1 && whole0 == 1));
        if (ragged) reinterpret_cast<T*>(part)[v * kN + e] = at >= 0 && at < P.vocab ? x[at] : Vec<T>::lowest();
    }
    const float temperature = P.temperature[row];
    const bool greedy = !(temperature > 0.f);
    const int32_t k_in = P.top_k ? P.top_k[row] : 0;
    const uint32_t k = greedy ? 1u : k_in > 0 ? (uint32_t)k_in : 0xffffffffu;
    const uint32_t p_part = P.top_p && P.top_p[row] < 1.f && !greedy ? part_of(P.top_p[row], 0x7fffffffu) : 0x80000000u;
    const uint32_t least = P.min_p ? max(1u, part_of(P.min_p[row], 0x80000000u)) : 1u;
    const uint32_t u_part = part_of(P.u[row], 0x7fffffffu);
    __syncthreads();

    // ---- the row's maximum, this thread's, and the r-th largest of its warp's
    auto wait_piece = [&](int i) {
        uint32_t done = 0;
        for (unsigned it = 0; it < kWaitLimit && !done; ++it)
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], 0;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                         : "=r"(done)
                         : "r"(smem_u32(&sm.bar[i]))
                         : "memory");
        return done != 0;
    };
    const int run0 = wid * chunk, run1 = min(run0 + chunk, count);  // this warp's run
    float most = -INFINITY;
    // (a block leaves only after every piece has landed: each has warps that wait for it, and the exchange is behind
    // them; a wait that runs out, never expected, is given a second bound for that and spoils the row)
    bool fine = wait_piece(wid / (kWarps / kPieces));
    fine = __all_sync(~0u, fine);
    if (!fine) wait_piece(wid / (kWarps / kPieces));
    for (int v = run0 + lane; v < run1; v += 32) {
        float e[kN];
        Vec<T>::split(part[v], e);
#pragma unroll
        for (int j = 0; j < kN; ++j) most = fmaxf(most, e[j]);
    }
    uint32_t my_top = key_of(most);
    const uint32_t want = k != 0xffffffffu ? k : (uint32_t)kList / 2;  // tokens that the bound has to let through
    // so many of each warp that the cluster's are a few times as many as wanted; a place for each of a block's threads
    const uint32_t places = kThreads / (kWarps * blocks);
    const uint32_t show = min(places, (3 * min(want, (uint32_t)kThreads) + kWarps * blocks - 1) / (kWarps * blocks));
    {
        uint32_t left = my_top, mine = 0;  // lane i: the i-th largest
        for (uint32_t i = 0; i < show; ++i) {
            const uint32_t m = __reduce_max_sync(~0u, left);
            if (lane == (int)i) mine = m;
            if (lane == __ffs(__ballot_sync(~0u, left == m)) - 1) left = 0;
        }
        // (a wait that ran out shows as a key that no logit has)
        if (!fine) mine = 0xffffffffu;
        for (uint32_t i = lane; i < places * blocks; i += 32) {
            const uint32_t v = __shfl_sync(~0u, mine, i / blocks);
            remote_store32(remote(smem_u32(&sm.shown[(rank * kWarps + wid) * places + i / blocks]), i % blocks), v);
        }
    }
    __syncwarp();
    if (blocks > 1) cluster_sync();
    else __syncthreads();
    const uint32_t shown = sm.shown[tid];
    uint32_t top_key = __reduce_max_sync(~0u, shown);
    if (lane == 0) sm.warp_words[wid].top = top_key;
    __syncthreads();
    top_key = __reduce_max_sync(~0u, sm.warp_words[lane & (kWarps - 1)].top);

    // sums and maxima over the cluster
    int turn = 0;
    auto exchange = [&](Sums v, Sums* before) {  // the blocks' before this one into `before`
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            v.a += __shfl_xor_sync(~0u, v.a, off);
            v.b += __shfl_xor_sync(~0u, v.b, off);
            v.c += __shfl_xor_sync(~0u, v.c, off);
        }
        v.n = __reduce_add_sync(~0u, v.n);
        if (lane == 0) sm.warp[wid] = v;
        __syncthreads();
        Sums mine = {0, 0, 0, 0};
#pragma unroll 4
        for (int i = 0; i < kWarps; ++i) {
            const Sums w = sm.warp[i];
            mine = Sums{mine.a + w.a, mine.b + w.b, mine.c + w.c, mine.n + w.n};
        }
        if (tid < (int)blocks) {  // to every block of the cluster
            const uint32_t to = remote(smem_u32(&sm.peers[turn][rank]), tid);
            remote_store(to, mine.a);
            remote_store(to + 8, mine.b);
            remote_store(to + 16, mine.c);
            remote_store(to + 24, mine.n);
        }
        __syncwarp();
        if (blocks > 1) cluster_sync();
        else __syncthreads();
        Sums all = {0, 0, 0, 0};
        for (uint32_t i = 0; i < blocks; ++i) {
            if (before && i == rank) *before = all;
            const Sums w = sm.peers[turn][i];
            all = Sums{all.a + w.a, all.b + w.b, all.c + w.c, all.n + w.n};
        }
        turn ^= 1;
        return all;
    };
    auto exchange_words = [&](Words v) {
        v.top = __reduce_max_sync(~0u, v.top);
        v.high = __reduce_max_sync(~0u, v.high);
        v.n = __reduce_add_sync(~0u, v.n);
        if (lane == 0) sm.warp_words[wid] = v;
        __syncthreads();
        const Words w = sm.warp_words[lane & (kWarps - 1)];
        v.top = __reduce_max_sync(~0u, w.top);
        v.high = __reduce_max_sync(~0u, w.high);
        v.n = __reduce_add_sync(~0u, lane < kWarps ? w.n : 0u);
        if (tid < (int)blocks) {
            const uint32_t to = remote(smem_u32(&sm.peer_words[turn][rank]), tid);
            remote_store32(to, v.top);
            remote_store32(to + 4, v.high);
            remote_store32(to + 8, v.n);
        }
        __syncwarp();
        if (blocks > 1) cluster_sync();
        else __syncthreads();
        v = Words{0, 0, 0};
        for (uint32_t i = 0; i < blocks; ++i) {
            const Words p = sm.peer_words[turn][i];
            v = Words{max(v.top, p.top), max(v.high, p.high), v.n + p.n};
        }
        turn ^= 1;
        return v;
    };
    auto answer = [&](int token, uint32_t w, uint64_t mass, uint32_t kept) {
        P.token[row] = token;
        if (P.logprob) P.logprob[row] = w == 0 ? (mass == 0 ? NAN : -INFINITY) : log_share(w, mass);
        if (P.n_kept) P.n_kept[row] = (int32_t)kept;
    };
    if (top_key == kEmptyKey || top_key == 0xffffffffu) {  // nothing to draw, or (never expected) a wait that ran out
        if (rank == 0 && tid == 0) answer(-1, 0, top_key == kEmptyKey ? 1 : 0, 0);
        return;
    }
    const bool infinite = top_key == key_of(INFINITY);
    if (infinite) {  // only the infinite logits have a weight: as zeros, the others as -inf
        for (int i = run0 * kN + lane; i < run1 * kN; i += 32) {
            T* at = reinterpret_cast<T*>(part) + i;
            *at = from_float<T>(to_float(*at) == INFINITY ? 0.f : -INFINITY);
        }
        __syncwarp();
        most = -INFINITY;
        for (int v = run0 + lane; v < run1; v += 32) {
            float e[kN];
            Vec<T>::split(part[v], e);
#pragma unroll
            for (int j = 0; j < kN; ++j) most = fmaxf(most, e[j]);
        }
        my_top = key_of(most);
        top_key = key_of(0.f);
    }
    // A key that at least `want` logits of the row reach: the want-th largest of the shown; 1 where not so many are.
    uint32_t bound = top_key;
    if (k > 1 && !infinite) {
        // from the warps' own maxima, if they are enough, to an eighth more than wanted or keys 2^12 near (2^-11 of a
        // logit)
        uint32_t low = __reduce_min_sync(~0u, tid % places == 0 ? shown : 0xffffffffu), hi = top_key;
        if (lane == 0) sm.warp_words[wid].high = low;
        __syncthreads();
        low = __reduce_min_sync(~0u, sm.warp_words[lane & (kWarps - 1)].high);
        bound = (uint32_t)__syncthreads_count(shown >= low) >= want ? max(low, 1u) : 1u;
        while (hi - bound >= 1u << 12) {
            const uint32_t mid = hi - (hi - bound) / 2;
            const uint32_t n = __syncthreads_count(shown >= mid);
            if (n >= want) bound = mid;
            else hi = mid - 1;
            if (n >= want && n <= want + want / 8) break;
        }
    }
    Scale s;
    s.top = value_of(top_key);
    s.rate = greedy ? 1.f : fminf(__fdiv_rn(0x1.715476p+0f, temperature), 3e38f);
    s.mz = P.minus_zeros;

    // f(two logits, their exponents, index of the first) over this warp's run
    auto each_pair = [&](auto&& f) {
        for (int v = run0 + lane; v < run1; v += 32) {
            float e[kN];
            Vec<T>::split(part[v], e);
#pragma unroll
            for (int j = 0; j < kN; j += 2) {
                float y0, y1;
                exponents(s, e[j], e[j + 1], y0, y1);
                f(e[j], e[j + 1], y0, y1, base + v * kN + j);
            }
        }
    };

    // ---- without top-k: the row's mass, what min-p keeps of it, and what may stand before that in the order
    bool cut = k != 0xffffffffu || p_part < 0x80000000u;
    uint64_t mass = 0;
    Sums kept = {0, 0, 0, 0}, kept_before = {0, 0, 0, 0};  // c: mass kept, n: tokens kept
    if (k == 0xffffffffu) {
        Sums v = {0, 0, 0, 0};
        if (least == 1) {
            each_pair([&](float, float, float y0, float y1, int) {
                uint32_t w0, w1;
                weights(s, y0, y1, w0, w1);
                v.a += (uint64_t)w0 + w1;
                v.n += min(w0, 1u) + min(w1, 1u);
            });
            v.c = v.a;
        } else {
            // Weights fall with the logits but for the rounding of the polynomial: `loose` is below every weight that
            // can stand before one of `least` in the order.
            const uint32_t loose = least - min(least, (least >> 20) + 1u);
            each_pair([&](float, float, float y0, float y1, int) {
                uint32_t w0, w1;
                weights(s, y0, y1, w0, w1);
                v.a += (uint64_t)w0 + w1;
                if (max(w0, w1) < loose) return;
                v.b += (uint64_t)(w0 >= loose ? w0 : 0u) + (w1 >= loose ? w1 : 0u);
                v.c += (uint64_t)(w0 >= least ? w0 : 0u) + (w1 >= least ? w1 : 0u);
                v.n += (w0 >= least) + (w1 >= least);
            });
        }
        kept = exchange(v, &kept_before);
        if (lane == 0) sm.warp_mass[wid] = sm.warp[wid].c;
        mass = kept.a;
        // every token that min-p keeps comes before the nucleus ends
        if (cut && least > 1 && kept.b <= share_of(mass, p_part)) cut = false;
    }

    // ---- few tokens: candidates to the first block
    if (cut && want <= (uint32_t)kList) {
        const uint32_t share = kGather / blocks, to = remote(smem_u32(sm.gather), 0) + 8 * rank * share;
        for (uint32_t m = __ballot_sync(~0u, my_top >= bound); m; m &= m - 1) {  // the logits of a lane that reaches it
            const int of = __ffs(m) - 1, n = (run1 - run0 - of + 31) / 32 * kN;
            for (int i = lane; i < n; i += 32) {
                const int at = (run0 + of + i / kN * 32) * kN + i % kN;
                const uint32_t key = key_of(to_float(reinterpret_cast<const T*>(part)[at]));
                if (key >= bound) {
                    const uint32_t slot = atomicAdd(&sm.n_mine, 1u);
                    if (slot < share) remote_store(to + 8 * slot, (uint64_t)key << 32 | (uint32_t)~(base + at));
                }
            }
            __syncwarp();
        }
        __syncthreads();
        if (tid < (int)blocks) remote_store32(remote(smem_u32(&sm.counts[rank]), tid), sm.n_mine);
        __syncwarp();
        if (blocks > 1) cluster_sync();
        else __syncthreads();
        bool fits = true;
        for (uint32_t i = 0; i < blocks; ++i) fits = fits && sm.counts[i] <= share;
        if (fits && k != 0xffffffffu && rank != 0) return;
        bool done = false;  // the first block has the token
        if (fits && rank == 0) {
            for (uint32_t i = tid; i < blocks * share; i += kThreads)
                if (i % share < sm.counts[i / share]) sm.list[atomicAdd(&sm.n_list, 1u)] = sm.gather[i];
            __syncthreads();
            // `team` threads a candidate, in no order: ranks and sums by comparison with every other
            const uint32_t n = sm.n_list;
            for (uint32_t i = tid; i < n; i += kThreads) sm.weight[i] = weight_of(s, value_of((uint32_t)(sm.list[i] >> 32)));
            int team_log2 = 0;
            while (team_log2 < 5 && (n << (team_log2 + 1)) <= kThreads) ++team_log2;
            const uint32_t team = 1u << team_log2, me0 = (uint32_t)tid >> team_log2, j0 = (uint32_t)tid & (team - 1);
            constexpr int kRounds = kGather / kThreads;  // candidates of a thread, where they are many
            uint64_t above[kRounds];
            uint32_t rank_of[kRounds];
            __syncthreads();
            uint64_t total = 0;
#pragma unroll
            for (int q = 0; q < kRounds; ++q) {
                const uint32_t i = me0 + q * kThreads;
                above[q] = 0;
                rank_of[q] = 0;
                if (q > 0 && n <= (uint32_t)(q * kThreads)) break;
                const uint64_t me = i < n ? sm.list[i] : ~0ull;
#pragma unroll 4
                for (uint32_t j = j0; j < n; j += team)
                    if (sm.list[j] > me) {
                        above[q] += sm.weight[j];
                        ++rank_of[q];
                    }
                for (uint32_t off = 1; off < team; off <<= 1) {
                    above[q] += __shfl_xor_sync(~0u, above[q], off);
                    rank_of[q] += __shfl_xor_sync(~0u, rank_of[q], off);
                }
                if (i < n && rank_of[q] < want) total = max(total, above[q] + sm.weight[i]);
            }
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) total = max(total, __shfl_xor_sync(~0u, total, off));
            if (lane == 0) sm.warp[wid].a = total;
            __syncthreads();
            for (int i = 0; i < kWarps; ++i) total = max(total, sm.warp[i].a);
            // the nucleus ends among the first `want`, or they are all there is
            const uint64_t goal = p_part < 0x80000000u ? share_of(k != 0xffffffffu ? total : mass, p_part) : ~0ull;
            const bool enough = k != 0xffffffffu || n < want || total >= goal;
            uint32_t n_kept = 0;
#pragma unroll
            for (int q = 0; q < kRounds; ++q) {
                const uint32_t i = me0 + q * kThreads;
                bool in = false;
                if (i < n && j0 == 0) {
                    const uint32_t w = sm.weight[i];
                    in = rank_of[q] < want && (above[q] < goal || rank_of[q] == 0) && w >= least;
                    sm.kept[i] = in ? w : 0u;
                }
                n_kept += __syncthreads_count(in);
            }
            if (enough) {
#pragma unroll
                for (int q = 0; q < kRounds; ++q) {
                    const uint32_t i = me0 + q * kThreads;
                    if (q > 0 && n <= (uint32_t)(q * kThreads)) break;
                    const uint32_t index = i < n ? ~(uint32_t)sm.list[i] : 0u;
                    uint64_t before = 0, sum = 0;
#pragma unroll 4
                    for (uint32_t j = j0; j < n; j += team) {
                        const uint32_t wj = sm.kept[j];
                        sum += wj;
                        before += ~(uint32_t)sm.list[j] < index ? wj : 0u;
                    }
                    for (uint32_t off = 1; off < team; off <<= 1) {
                        sum += __shfl_xor_sync(~0u, sum, off);
                        before += __shfl_xor_sync(~0u, before, off);
                    }
                    const uint64_t at_mass = share_of(sum, u_part);
                    const uint32_t w = i < n ? sm.kept[i] : 0u;
                    if (j0 == 0 && before <= at_mass && at_mass < before + w) answer((int)index, w, sum, n_kept);
                }
                done = true;
            }
        }
        if (fits && (k != 0xffffffffu || exchange_words(Words{done ? 1u : 0u, 0, 0}).top)) return;
    }

    // ---- the cut: keys above cut_key, and those equal to it up to cut_index
    uint32_t cut_key = 1;
    int cut_index = P.vocab;
    auto in_cut = [&](uint32_t key, int i) { return key > cut_key || (key == cut_key && i <= cut_index); };
    // moves the cut to the first tokens of the order that reach `n_goal` tokens or the mass `goal`, all of whose keys
    // are at least `floor`
    auto cut_at = [&](uint32_t n_goal, uint64_t goal, uint32_t floor) {
        uint64_t over = 0;      // mass and count above the part of a bin that the cut lies in
        uint32_t n_over = 0;
        int from = 0;           // the part, in units of the level
        for (int level = 0; level < 2; ++level) {
            const float unit = level == 0 ? 16.f : 16.f * kBins;  // bins of y a unit
            for (int i = tid; i < 3 * kBins; i += kThreads) (&sm.bins[0][0])[i] = 0;
            __syncthreads();
            each_pair([&](float x0, float x1, float y0, float y1, int at) {
                const float y[2] = {y0, y1}, e[2] = {x0, x1};
                uint32_t w[2];
                int bin[2];
                bool in[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    bin[j] = (int)(-y[j] * unit) - from;
                    const uint32_t key = key_of(e[j]);
                    in[j] = key >= floor && in_cut(key, at + j) && bin[j] >= 0 && (level == 0 || bin[j] < kBins || from == (kBins - 1) * kBins);
                    bin[j] = min(bin[j], kBins - 1);
                }
                if (!in[0] && !in[1]) return;
                weights(s, y0, y1, w[0], w[1]);
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (in[j]) {
                        atomicAdd(&sm.bins[0][bin[j]], w[j] & 0xffffu);
                        atomicAdd(&sm.bins[1][bin[j]], w[j] >> 16);
                        atomicAdd(&sm.bins[2][bin[j]], 1u);
                    }
            });
            if (blocks > 1) cluster_sync();
            else __syncthreads();
            // a bin a thread: its sums over the cluster, then over the bins before it
            uint64_t m = 0;
            uint32_t c = 0;
            for (uint32_t b = 0; b < blocks; ++b) {
                const uint32_t at = remote(smem_u32(&sm.bins[0][tid]), b);
                m += (uint64_t)remote_load(at) + ((uint64_t)remote_load(at + 4 * kBins) << 16);
                c += remote_load(at + 8 * kBins);
            }
            uint64_t ms = m;
            uint32_t cs = c;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const uint64_t a = __shfl_up_sync(~0u, ms, off);
                const uint32_t b = __shfl_up_sync(~0u, cs, off);
                if (lane >= off) ms += a, cs += b;
            }
            if (lane == 31) {
                sm.warp[wid].a = ms;
                sm.warp[wid].n = cs;
            }
            if (tid == 0) sm.found[0] = ~0ull;
            __syncthreads();
            ms += over;
            cs += n_over;
            for (int i = 0; i < wid; ++i) ms += sm.warp[i].a, cs += sm.warp[i].n;
            const bool at_goal = cs >= n_goal || ms >= goal, before = cs - c >= n_goal || ms - m >= goal;
            if (at_goal && !before) {
                sm.found[0] = tid;
                sm.found[1] = ms - m;
                sm.found[2] = cs - c;
            }
            if (blocks > 1) cluster_sync();  // no block clears its bins while another reads them
            else __syncthreads();
            if (sm.found[0] == ~0ull) return;  // the goal is beyond all of them
            over = sm.found[1];
            n_over = (uint32_t)sm.found[2];
            from = level == 0 ? (int)sm.found[0] * kBins : from + (int)sm.found[0];
            __syncthreads();
        }
        const bool last_bin = from == kBins * kBins - 1;  // open to below
        auto in_part = [&](float y) {
            const int b = (int)(-y * (16.f * kBins));
            return last_bin ? b >= from : b == from;
        };
        // the part's largest and smallest key
        uint32_t low = 0xffffffffu, high = 0;
        each_pair([&](float x0, float x1, float y0, float y1, int at) {
            const float y[2] = {y0, y1}, e[2] = {x0, x1};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (!in_part(y[j])) continue;
                const uint32_t key = key_of(e[j]);
                if (key >= floor && in_cut(key, at + j)) {
                    low = min(low, key);
                    high = max(high, key);
                }
            }
        });
        const Words ends = exchange_words(Words{high, ~low, 0});
        uint32_t hi_key = ends.top, lo_key = ~ends.high;
        Sums v = {0, 0, 0, 0};
        auto tally_part = [&](uint32_t from_key) {  // the part's keys >= from_key
            Sums t = {0, 0, 0, 0};
            each_pair([&](float x0, float x1, float y0, float y1, int at) {
                const float y[2] = {y0, y1}, e[2] = {x0, x1};
                if (!in_part(y0) && !in_part(y1)) return;
                uint32_t w[2];
                weights(s, y0, y1, w[0], w[1]);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t key = key_of(e[j]);
                    if (key >= from_key && key >= floor && in_part(y[j]) && in_cut(key, at + j)) {
                        t.a += w[j];
                        t.n += 1;
                    }
                }
            });
            return exchange(t, nullptr);
        };
        if (lo_key < hi_key) {
            while (lo_key < hi_key) {
                const uint32_t mid = hi_key - (hi_key - lo_key) / 2;
                v = tally_part(mid);
                if (n_over + v.n >= n_goal || over + v.a >= goal) lo_key = mid;
                else hi_key = mid - 1;
            }
            v = tally_part(lo_key + 1);
        }
        // of the tokens equal to it, those still needed, by index
        const uint32_t w = weight_of(s, value_of(lo_key));
        uint64_t need = n_goal - n_over - v.n;
        if (goal != ~0ull) {
            const uint64_t by_mass = w > 0 ? (goal - over - v.a + w - 1) / w : ~0ull;
            need = by_mass < need ? by_mass : need;
        }
        uint32_t c = 0;
        each_pair([&](float x0, float x1, float, float, int at) {
            c += (key_of(x0) == lo_key && in_cut(lo_key, at)) + (key_of(x1) == lo_key && in_cut(lo_key, at + 1));
        });
        c = __reduce_add_sync(~0u, c);
        Sums before;
        exchange(Sums{0, 0, 0, lane == 0 ? c : 0u}, &before);
        uint64_t seen = before.n;  // by the warps before this one
        for (int i = 0; i < wid; ++i) seen += sm.warp[i].n;
        uint32_t index = 0;
        if (seen < need && need <= seen + c) {  // in this warp's run: 32 logits at a time
            for (int i = run0 * kN; i < run1 * kN; i += 32) {
                const uint32_t key = i + lane < run1 * kN ? key_of(to_float(reinterpret_cast<const T*>(part)[i + lane])) : 0;
                uint32_t m = __ballot_sync(~0u, key == lo_key && in_cut(key, base + i + lane));
                if (seen + __popc(m) < need) {
                    seen += __popc(m);
                    continue;
                }
                for (; seen + 1 < need; ++seen) m &= m - 1;
                index = (uint32_t)(base + i + __ffs(m));  // one past it
                break;
            }
        }
        cut_index = (int)exchange_words(Words{index, 0, 0}).top - 1;  // the goal is reached, so that there is one
        cut_key = lo_key;
    };
    if (cut) {
        if (k != 0xffffffffu) cut_at(k, ~0ull, bound);
        if (p_part < 0x80000000u) {
            if (k != 0xffffffffu) {
                Sums v = {0, 0, 0, 0};
                each_pair([&](float x0, float x1, float y0, float y1, int at) {
                    const bool in0 = in_cut(key_of(x0), at), in1 = in_cut(key_of(x1), at + 1);
                    if (!in0 && !in1) return;
                    uint32_t w0, w1;
                    weights(s, y0, y1, w0, w1);
                    v.a += (uint64_t)(in0 ? w0 : 0u) + (in1 ? w1 : 0u);
                });
                mass = exchange(v, nullptr).a;
            }
            const uint64_t goal = share_of(mass, p_part);
            cut_at(0xffffffffu, goal > 0 ? goal : 1, cut_key);
        }
        Sums v = {0, 0, 0, 0};
        each_pair([&](float x0, float x1, float y0, float y1, int at) {
            const bool in0 = in_cut(key_of(x0), at), in1 = in_cut(key_of(x1), at + 1);
            if (!in0 && !in1) return;
            uint32_t w0, w1;
            weights(s, y0, y1, w0, w1);
            if (!in0 || w0 < least) w0 = 0;
            if (!in1 || w1 < least) w1 = 0;
            v.c += (uint64_t)w0 + w1;
            v.n += min(w0, 1u) + min(w1, 1u);
        });
        kept = exchange(v, &kept_before);
        if (lane == 0) sm.warp_mass[wid] = sm.warp[wid].c;
    }

    // ---- the draw: the warp's run that holds it, shared out over the block
    const uint64_t goal = share_of(kept.c, u_part);
    __syncthreads();
    uint64_t run_begin = kept_before.c;
    int run = 0;
    if (goal < run_begin) return;
    for (; run < kWarps && goal >= run_begin + sm.warp_mass[run]; ++run) run_begin += sm.warp_mass[run];
    if (run == kWarps) return;  // in a later block's part
    const int e0 = run * chunk * kN, e1 = min((run + 1) * chunk, count) * kN;
    const int each = (chunk * kN + kThreads - 1) / kThreads, a0 = min(e0 + tid * each, e1), a1 = min(a0 + each, e1);
    auto kept_weight = [&](int i) {
        const float v = to_float(reinterpret_cast<const T*>(part)[i]);
        if (cut && !in_cut(key_of(v), base + i)) return 0u;
        const uint32_t w = weight_of(s, v);
        return w >= least ? w : 0u;
    };
    uint64_t sum = 0;
    for (int i = a0; i < a1; ++i) sum += kept_weight(i);
    uint64_t upto = sum;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint64_t v = __shfl_up_sync(~0u, upto, off);
        if (lane >= off) upto += v;
    }
    if (lane == 31) sm.warp[wid].a = upto;
    __syncthreads();
    for (int i = 0; i < wid; ++i) upto += sm.warp[i].a;
    uint64_t at_mass = run_begin + upto - sum;
    if (at_mass <= goal && goal < at_mass + sum) {
        for (int i = a0; i < a1; ++i) {
            const uint32_t w = kept_weight(i);
            if (goal < at_mass + w) {
                answer(base + i, w, kept.c, kept.n);
                break;
            }
            at_mass += w;
        }
    }
}

template <typename T>
cudaError_t launch_typed(const SampleParams& p, cudaStream_t stream)
{
    constexpr int kN = Vec<T>::kN;
    const int n_vec = (p.vocab + 2 * kN - 2) / kN;  // at the worst alignment
    // as many blocks a row as keep the GPU's two an SM busy, and as its shared memory needs
    int blocks = 1;
    while (blocks < kMaxCluster && ((int64_t)p.n_rows * blocks < 304 || (n_vec + blocks - 1) / blocks * 16 > 72 * 1024)) blocks *= 2;
    while (blocks > 1 && n_vec / blocks < 64) blocks /= 2;
    const size_t bytes = (size_t)(n_vec + blocks - 1) / blocks * 16;
    auto kernel = sample_kernel<T>;
    cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (err != cudaSuccess) return err;
    return launch_dependent(kernel, dim3((unsigned)(p.n_rows * blocks)), dim3(kThreads), bytes, blocks, stream, p);
}

}  // namespace

cudaError_t launch_sample(const SampleParams& p, cudaStream_t stream)
{
    if (p.dtype == CTR_BF16) return launch_typed<__nv_bfloat16>(p, stream);
    if (p.dtype == CTR_F16) return launch_typed<__half>(p, stream);
    return launch_typed<float>(p, stream);
}

}  // namespace ctr
