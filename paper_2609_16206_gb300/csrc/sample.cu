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
//   * few of them (top-k up to kList, or a nucleus that is): the k-th largest
//     of the threads' own maxima is a bound that at least k logits reach and
//     not many more do; those go to the first block's list, which ranks them;
//   * a nucleus cut off by min-p anyway needs no cut: the mass of what min-p
//     keeps, summed with the whole row's, shows it;
//   * else the cut is found from the mass (or count) in 512 bins of y, then in
//     512 parts of the bin that holds it, then by bisection over the part's
//     keys, and over equal keys by index.
// The drawn token's block is known from the blocks' sums and finds it in a
// pass of its own.
#include "decode_internal.cuh"

namespace ctr {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kList = 128;          // tokens that the first block ranks
constexpr int kMine = 512;          // candidates of a block
constexpr int kGather = 1536;       // of the cluster
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
    if (s.top == INFINITY) {  // only the infinite ones have a weight
        y0 = x0 == INFINITY ? 0.f : -64.f;
        y1 = x1 == INFINITY ? 0.f : -64.f;
    }
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
struct Tally {
    uint64_t a, b;
    uint32_t n, top;
};
__device__ __forceinline__ Tally join(const Tally& x, const Tally& y)
{
    return Tally{x.a + y.a, x.b + y.b, x.n + y.n, x.top > y.top ? x.top : y.top};
}
__device__ __forceinline__ Tally shuffled(const Tally& v, int off)
{
    return Tally{__shfl_xor_sync(~0u, v.a, off), __shfl_xor_sync(~0u, v.b, off), __shfl_xor_sync(~0u, v.n, off),
                 __shfl_xor_sync(~0u, v.top, off)};
}

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
__device__ __forceinline__ uint32_t remote_load(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
struct __align__(16) Shared {
    uint64_t gather[kGather];       // first block: (key, ~index) of the candidates
    uint64_t mine[kMine];           // this block's; later the ranked ones' weights
    uint32_t bins[3][kBins];        // low and high halves of the masses, counts
    Tally warp[kWarps];
    Tally peers[2][kMaxCluster];    // exchanges alternate between the two
    uint64_t prefix[kWarps];
    uint64_t found[4];
    uint32_t n_mine;
    uint64_t bar[kPieces];
};

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
        sm.n_mine = 0;
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
    const int piece = ((per + kPieces - 1) / kPieces + kThreads - 1) / kThreads * kThreads;
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

    // ---- the row's maximum, and this thread's
    auto wait_piece = [&](int i) {
        uint32_t done = 0;
        for (unsigned it = 0; it < kWaitLimit && !done; ++it)
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], 0;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                         : "=r"(done)
                         : "r"(smem_u32(&sm.bar[i]))
                         : "memory");
        return done != 0;
    };
    float most = -INFINITY;
    bool fine = true;
    for (int i = 0; i < kPieces; ++i) {
        fine = wait_piece(i) && fine;
        for (int v = i * piece + tid; v < min((i + 1) * piece, count); v += kThreads) {
            float e[kN];
            Vec<T>::split(part[v], e);
#pragma unroll
            for (int j = 0; j < kN; ++j) most = fmaxf(most, e[j]);
        }
    }
    if (!fine)  // never expected: a second bounded wait, so that no copy outlives the block's shared memory
        for (int i = 0; i < kPieces; ++i) wait_piece(i);
    const uint32_t my_top = key_of(most);

    // sums over the cluster; the calling block's predecessors' into `before`
    int turn = 0;
    auto exchange = [&](Tally v, Tally* before) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) v = join(v, shuffled(v, off));
        if (lane == 0) sm.warp[wid] = v;
        __syncthreads();
        v = sm.warp[lane & (kWarps - 1)];
#pragma unroll
        for (int off = kWarps / 2; off > 0; off >>= 1) v = join(v, shuffled(v, off));
        if (blocks == 1) {
            if (before) *before = Tally{0, 0, 0, 0};
            __syncthreads();
            return v;
        }
        if (tid < (int)blocks) {  // to every block of the cluster
            const uint32_t to = remote(smem_u32(&sm.peers[turn][rank]), tid);
            remote_store(to, v.a);
            remote_store(to + 8, v.b);
            remote_store(to + 16, (uint64_t)v.top << 32 | v.n);
        }
        __syncwarp();
        cluster_sync();
        Tally all = {0, 0, 0, 0}, b = {0, 0, 0, 0};
        for (uint32_t i = 0; i < blocks; ++i) {
            if (i == rank) b = all;
            all = join(all, sm.peers[turn][i]);
        }
        if (before) *before = b;
        turn ^= 1;
        return all;
    };
    const Tally first = exchange(Tally{0, 0, fine ? 0u : 1u, my_top}, nullptr);
    const uint32_t top_key = first.top;
    auto answer = [&](int token, uint32_t w, uint64_t mass, uint32_t kept) {
        P.token[row] = token;
        if (P.logprob) P.logprob[row] = w == 0 ? (mass == 0 ? NAN : -INFINITY) : (float)log((double)w / (double)mass);
        if (P.n_kept) P.n_kept[row] = (int32_t)kept;
    };
    if (top_key == kEmptyKey || first.n > 0) {  // nothing to draw, or (never expected) a wait that ran out
        if (rank == 0 && tid == 0) answer(-1, 0, first.n > 0 ? 0 : 1, 0);
        return;
    }
    Scale s;
    s.top = value_of(top_key);
    s.rate = greedy ? 1.f : fminf(__fdiv_rn(0x1.715476p+0f, temperature), 3e38f);
    s.mz = P.minus_zeros;

    // f(two logits, their weights, index of the first) over this block's part; a part's vectors go round the threads
    auto each_pair = [&](auto&& f) {
        for (int v = tid; v < count; v += kThreads) {
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

    // ---- the whole row's mass, and what min-p keeps of it, where no small top-k makes them needless
    const bool by_list = k <= (uint32_t)kList;
    uint64_t mass = 0;
    bool cut = k != 0xffffffffu || p_part < 0x80000000u;
    if (!by_list && k == 0xffffffffu && cut) {
        // Weights fall with the logits but for the rounding of the polynomial: `loose` is below every weight that can
        // stand before one of `least` in the order.
        const uint32_t loose = least - min(least, (least >> 20) + 1u);
        Tally v = {0, 0, 0, 0};
        each_pair([&](float, float, float y0, float y1, int) {
            uint32_t w0, w1;
            weights(s, y0, y1, w0, w1);
            v.a += (uint64_t)w0 + w1;
            v.b += (uint64_t)(w0 >= loose ? w0 : 0u) + (w1 >= loose ? w1 : 0u);
        });
        v = exchange(v, nullptr);
        mass = v.a;
        // every token that min-p keeps comes before the nucleus ends
        if (least > 1 && v.b <= share_of(mass, p_part)) cut = false;
    }

    // ---- few tokens: candidates to the first block
    if (cut && (by_list || k == 0xffffffffu)) {
        const uint32_t want = by_list ? k : (uint32_t)kList;
        // the largest bound (of the upper key bits) that `want` threads' maxima reach; 1 where there are not so many
        uint32_t lo = 0, hi = top_key >> 16;
        while (lo < hi) {
            const uint32_t mid = hi - (hi - lo) / 2;
            if ((uint32_t)__syncthreads_count(my_top >> 16 >= mid) >= want) lo = mid;
            else hi = mid - 1;
        }
        const uint32_t bound = max(lo << 16, 1u);
        if (my_top >= bound) {
            for (int v = tid; v < count; v += kThreads) {
                float e[kN];
                Vec<T>::split(part[v], e);
#pragma unroll
                for (int j = 0; j < kN; ++j) {
                    const uint32_t key = key_of(e[j]);
                    if (key >= bound) {
                        const uint32_t at = atomicAdd(&sm.n_mine, 1u);
                        if (at < kMine) sm.mine[at] = (uint64_t)key << 32 | (uint32_t)~(base + v * kN + j);
                    }
                }
            }
        }
        __syncthreads();
        const uint32_t n_mine = sm.n_mine;
        Tally before;
        const uint32_t n = exchange(Tally{0, 0, tid > 0 ? 0 : n_mine <= kMine ? n_mine : kGather + 1, 0}, &before).n;
        const bool fits = n <= kGather;  // known to every block
        if (fits) {
            const uint32_t to = remote(smem_u32(sm.gather), 0) + 8 * before.n;
            for (uint32_t i = tid; i < n_mine; i += kThreads) remote_store(to + 8 * i, sm.mine[i]);
            __syncwarp();
            cluster_sync();
            if (by_list && rank != 0) return;
        }
        uint32_t done = 0;  // 1: the first block has the token
        if (rank == 0 && fits) {
            // the first `want` of them: those not below the want-th
            uint64_t mine[kGather / kThreads];
#pragma unroll
            for (int i = 0; i < kGather / kThreads; ++i) mine[i] = tid + i * kThreads < (int)n ? sm.gather[tid + i * kThreads] : 0;
            uint64_t last = 1;
            if (n > want) {
                uint64_t a = 1, b = (uint64_t)top_key << 32 | 0xffffffffu;
                while (a < b) {
                    const uint64_t mid = b - (b - a) / 2;
                    int c = 0;
#pragma unroll
                    for (int i = 0; i < kGather / kThreads; ++i) c += mine[i] >= mid;
                    // a count of threads is at most the count; more than one of a thread's are counted one by one
                    uint32_t total = __syncthreads_count(c > 0);
#pragma unroll
                    for (int i = 1; i < kGather / kThreads; ++i)
                        if (n > (uint32_t)(i * kThreads)) total += __syncthreads_count(c > i);
                    if (total >= want) a = mid;
                    else b = mid - 1;
                    if (total == want) b = a;
                }
                last = a;
            }
            __syncthreads();
            if (tid == 0) sm.n_mine = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kGather / kThreads; ++i)
                if (mine[i] >= last) sm.mine[atomicAdd(&sm.n_mine, 1u) & (kMine - 1)] = mine[i];
            __syncthreads();
            const uint32_t m = min(sm.n_mine, (uint32_t)kList);
            // a thread a token, in no order: ranks and sums by comparison with every other
            uint64_t* ws = reinterpret_cast<uint64_t*>(sm.bins);
            const uint64_t me = tid < (int)m ? sm.mine[tid] : 0;
            const uint32_t index = ~(uint32_t)me;
            uint32_t w = tid < (int)m ? weight_of(s, value_of((uint32_t)(me >> 32))) : 0;
            if (tid < kList) ws[tid] = w;
            __syncthreads();
            uint64_t above = 0, sum = 0;
            if (tid < (int)m)
                for (uint32_t j = 0; j < m; ++j) {
                    const uint64_t wj = ws[j];
                    sum += wj;
                    above += sm.mine[j] > me ? wj : 0;
                }
            const uint64_t goal = p_part < 0x80000000u ? share_of(by_list ? sum : mass, p_part) : ~0ull;
            // the nucleus ends among them, or they are all there is
            const bool enough = by_list || n < want || __syncthreads_or(tid < (int)m && above + w >= goal);
            if (!(above < goal || above == 0) || w < least) w = 0;
            __syncthreads();
            if (tid < kList) ws[tid] = w;
            const uint32_t kept = __syncthreads_count(w > 0);
            if (enough) {
                uint64_t before = 0;
                sum = 0;
                if (w > 0)
                    for (uint32_t j = 0; j < m; ++j) {
                        const uint64_t wj = ws[j];
                        sum += wj;
                        before += ~(uint32_t)sm.mine[j] < index ? wj : 0;
                    }
                const uint64_t at_mass = share_of(sum, u_part);
                if (w > 0 && before <= at_mass && at_mass < before + w) answer((int)index, w, sum, kept);
                done = 1;
            }
        }
        if (by_list && fits) return;
        if (fits && exchange(Tally{0, 0, 0, done}, nullptr).top) return;
    }

    // ---- the cut: keys above cut_key, and those equal to it up to cut_index
    uint32_t cut_key = 1;
    int cut_index = P.vocab;
    auto in_cut = [&](uint32_t key, int i) { return key > cut_key || (key == cut_key && i <= cut_index); };
    // moves the cut to the first tokens of the order that reach `count` tokens or `goal`
    auto cut_at = [&](uint32_t n_goal, uint64_t goal) {
        uint64_t over = 0;      // mass and count above the part of a bin that the cut lies in
        uint32_t n_over = 0;
        uint32_t lo_key = cut_key, hi_key = top_key;
        int from = 0;           // in units of the level
        bool reached = true;
        for (int level = 0; level < 2 && reached; ++level) {
            const float unit = level == 0 ? 16.f : 16.f * kBins;  // bins of y a unit
            for (int i = tid; i < 3 * kBins; i += kThreads) (&sm.bins[0][0])[i] = 0;
            __syncthreads();
            each_pair([&](float x0, float x1, float y0, float y1, int at) {
                uint32_t w[2];
                const float y[2] = {y0, y1}, e[2] = {x0, x1};
                int bin[2];
                bool in[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    bin[j] = (int)(-y[j] * unit) - from;
                    const uint32_t key = key_of(e[j]);
                    in[j] = key != kEmptyKey && in_cut(key, at + j) && bin[j] >= 0 && (level == 0 || bin[j] < kBins || from == (kBins - 1) * kBins);
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
            if (lane == 31) sm.warp[wid] = Tally{ms, 0, cs, 0};
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
            reached = sm.found[0] != ~0ull;
            if (reached) {
                over = sm.found[1];
                n_over = (uint32_t)sm.found[2];
                from = level == 0 ? (int)sm.found[0] * kBins : from + (int)sm.found[0];
            }
            __syncthreads();
        }
        if (!reached) return;  // the goal is beyond all of them
        const bool last_bin = from == kBins * kBins - 1;  // open to below
        auto in_part = [&](float y) {
            const int b = (int)(-y * (16.f * kBins));
            return last_bin ? b >= from : b == from;
        };
        auto tally_part = [&](uint32_t from_key) {  // the part's keys >= from_key
            Tally v = {0, 0, 0, 0};
            each_pair([&](float x0, float x1, float y0, float y1, int at) {
                const float y[2] = {y0, y1}, e[2] = {x0, x1};
                if (!in_part(y0) && !in_part(y1)) return;
                uint32_t w[2];
                weights(s, y0, y1, w[0], w[1]);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t key = key_of(e[j]);
                    if (key != kEmptyKey && key >= from_key && in_part(y[j]) && in_cut(key, at + j))
                        v = join(v, Tally{w[j], 0, 1, key});
                }
            });
            return v;
        };
        // the part's largest and smallest key
        Tally v = tally_part(1);
        uint32_t low = 0xffffffffu;
        each_pair([&](float x0, float x1, float y0, float y1, int at) {
            const float y[2] = {y0, y1}, e[2] = {x0, x1};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t key = key_of(e[j]);
                if (key != kEmptyKey && in_part(y[j]) && in_cut(key, at + j)) low = min(low, key);
            }
        });
        hi_key = exchange(Tally{0, 0, 0, v.top}, nullptr).top;
        lo_key = ~exchange(Tally{0, 0, 0, ~low}, nullptr).top;
        while (lo_key < hi_key) {
            const uint32_t mid = hi_key - (hi_key - lo_key) / 2;
            v = exchange(tally_part(mid), nullptr);
            if (n_over + v.n >= n_goal || over + v.a >= goal) lo_key = mid;
            else hi_key = mid - 1;
        }
        // of the tokens equal to it, those still needed, by index
        v = lo_key == 0xffffffffu ? Tally{0, 0, 0, 0} : exchange(tally_part(lo_key + 1), nullptr);
        const uint32_t w = weight_of(s, value_of(lo_key));
        uint64_t need = n_goal - n_over - v.n;
        if (goal != ~0ull) {
            const uint64_t by_mass = w > 0 ? (goal - over - v.a + w - 1) / w : ~0ull;
            need = by_mass < need ? by_mass : need;
        }
        // a contiguous run of vectors to a thread
        const int run = (count + kThreads - 1) / kThreads, a0 = min(tid * run, count), a1 = min(a0 + run, count);
        uint32_t c = 0;
        for (int i = a0 * kN; i < a1 * kN; ++i) {
            const uint32_t key = key_of(to_float(reinterpret_cast<const T*>(part)[i]));
            c += key == lo_key && in_cut(key, base + i);
        }
        Tally before;
        exchange(Tally{0, 0, c, 0}, &before);
        uint32_t cs = c;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const uint32_t b = __shfl_up_sync(~0u, cs, off);
            if (lane >= off) cs += b;
        }
        if (lane == 31) sm.warp[wid].n = cs;
        __syncthreads();
        for (int i = 0; i < wid; ++i) cs += sm.warp[i].n;
        cs += before.n;
        uint32_t index = 0;
        if (cs - c < need && need <= cs) {
            uint64_t left = need - (cs - c);
            for (int i = a0 * kN; i < a1 * kN; ++i) {
                const uint32_t key = key_of(to_float(reinterpret_cast<const T*>(part)[i]));
                if (key == lo_key && in_cut(key, base + i) && --left == 0) {
                    index = (uint32_t)(base + i) + 1u;
                    break;
                }
            }
        }
        __syncthreads();
        index = exchange(Tally{0, 0, 0, index}, nullptr).top;
        cut_key = lo_key;
        cut_index = (int)index - 1;  // the goal is reached, so that there is one
    };
    if (cut) {
        if (k != 0xffffffffu) {
            cut_at(k, ~0ull);
            if (p_part < 0x80000000u) {
                Tally v = {0, 0, 0, 0};
                each_pair([&](float x0, float x1, float y0, float y1, int at) {
                    uint32_t w0, w1;
                    weights(s, y0, y1, w0, w1);
                    v.a += (uint64_t)(in_cut(key_of(x0), at) ? w0 : 0u) + (in_cut(key_of(x1), at + 1) ? w1 : 0u);
                });
                mass = exchange(v, nullptr).a;
            }
        }
        if (p_part < 0x80000000u) {
            const uint64_t goal = share_of(mass, p_part);
            cut_at(0xffffffffu, goal > 0 ? goal : 1);
        }
    }

    // ---- the draw: every block's kept mass, then the token in the block that holds it
    auto kept_weights = [&](float x0, float x1, int at, uint32_t& w0, uint32_t& w1) {
        float y0, y1;
        exponents(s, x0, x1, y0, y1);
        weights(s, y0, y1, w0, w1);
        if (w0 < least || (cut && !in_cut(key_of(x0), at))) w0 = 0;
        if (w1 < least || (cut && !in_cut(key_of(x1), at + 1))) w1 = 0;
    };
    Tally mine = {0, 0, 0, 0};
    for (int v = tid; v < count; v += kThreads) {
        float e[kN];
        Vec<T>::split(part[v], e);
#pragma unroll
        for (int j = 0; j < kN; j += 2) {
            uint32_t w0, w1;
            kept_weights(e[j], e[j + 1], base + v * kN + j, w0, w1);
            mine.a += (uint64_t)w0 + w1;
            mine.n += (w0 > 0) + (w1 > 0);
        }
    }
    Tally before;
    const uint64_t my_mass = [&] {  // of the block
        Tally v = mine;
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) v = join(v, shuffled(v, off));
        if (lane == 0) sm.prefix[wid] = v.a;
        __syncthreads();
        uint64_t m = 0;
        for (int i = 0; i < kWarps; ++i) m += sm.prefix[i];
        __syncthreads();
        return m;
    }();
    const Tally all = exchange(mine, &before);
    const uint64_t goal = share_of(all.a, u_part);
    if (goal < before.a || goal >= before.a + my_mass) return;
    const int run = (count + kThreads - 1) / kThreads, a0 = min(tid * run, count), a1 = min(a0 + run, count);
    uint64_t sum = 0;
    for (int v = a0; v < a1; ++v) {
        float e[kN];
        Vec<T>::split(part[v], e);
#pragma unroll
        for (int j = 0; j < kN; j += 2) {
            uint32_t w0, w1;
            kept_weights(e[j], e[j + 1], base + v * kN + j, w0, w1);
            sum += (uint64_t)w0 + w1;
        }
    }
    uint64_t upto = sum;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint64_t v = __shfl_up_sync(~0u, upto, off);
        if (lane >= off) upto += v;
    }
    if (lane == 31) sm.prefix[wid] = upto;
    __syncthreads();
    for (int i = 0; i < wid; ++i) upto += sm.prefix[i];
    uint64_t at_mass = before.a + upto - sum;
    if (at_mass <= goal && goal < at_mass + sum) {
        for (int v = a0; v < a1; ++v) {
            float e[kN];
            Vec<T>::split(part[v], e);
#pragma unroll
            for (int j = 0; j < kN; j += 2) {
                uint32_t w0, w1;
                kept_weights(e[j], e[j + 1], base + v * kN + j, w0, w1);
                if (at_mass <= goal && goal < at_mass + w0) answer(base + v * kN + j, w0, all.a, all.n);
                at_mass += w0;
                if (at_mass <= goal && goal < at_mass + w1) answer(base + v * kN + j + 1, w1, all.a, all.n);
                at_mass += w1;
            }
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
