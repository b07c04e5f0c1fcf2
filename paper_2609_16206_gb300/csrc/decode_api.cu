// decode_api.cu -- the extern "C" entry points of include/ctr_decode.h:
// host-side validation, parameter packing and kernel launches.  Nothing here
// allocates device memory or synchronises.
#include <cmath>
#include <cstring>

#include "decode_internal.cuh"

using namespace ctr;

namespace {

bool in_range(int64_t v, int64_t lo, int64_t hi) { return v >= lo && v <= hi; }

int cuda_status(cudaError_t e) { return e == cudaSuccess ? CTR_OK : CTR_ECUDA; }

constexpr int64_t kStrideMax = 1LL << 44;  // elements: every offset a kernel forms stays below 2^63

int log2_of(int32_t v)
{
    int l = 0;
    while ((1 << l) < v) ++l;
    return l;
}

bool valid_cache(const ctr_kv_cache* c)
{
    if (!c || !c->k || !c->v) return false;
    if (c->dtype != CTR_BF16 && c->dtype != CTR_F16) return false;
    if (!in_range(c->n_kv_heads, 1, 1024) || !in_range(c->head_dim, 8, 256) || c->head_dim % 8 != 0) return false;
    if (!in_range(c->page_tokens, 16, 1024) || (c->page_tokens & (c->page_tokens - 1)) != 0) return false;
    if (!in_range(c->n_pages, 1, 2147483647LL)) return false;
    if (!in_range(c->page_stride, 0, kStrideMax) || !in_range(c->head_stride, 0, kStrideMax) ||
        !in_range(c->token_stride, 0, kStrideMax))
        return false;
    return c->page_stride <= (1LL << 59) / c->n_pages;  // with the heads' and tokens' 2^54 each, offsets stay below 2^60
}

bool valid_rows(const ctr_rows& r, int64_t n_tokens, int32_t n_heads, bool may_be_null)
{
    if (!r.ptr) return may_be_null;
    if ((uintptr_t)r.ptr % 2u != 0) return false;
    if (!in_range(r.token_stride, 0, kStrideMax) || !in_range(r.head_stride, 0, kStrideMax)) return false;
    if (n_tokens > 0 && r.token_stride > (1LL << 59) / n_tokens) return false;
    return n_heads <= 0 || r.head_stride <= (1LL << 59) / n_heads;
}

bool aligned16(const void* p, int64_t a, int64_t b) { return (uintptr_t)p % 16u == 0 && a % 8 == 0 && b % 8 == 0; }

bool valid_attention_sizes(const ctr_kv_cache* c, int32_t n_q_heads, int32_t n_seqs, int32_t max_nodes)
{
    if (!valid_cache(c) || (c->head_dim != 64 && c->head_dim != 128)) return false;
    if (!in_range(n_q_heads, 1, 65536) || n_q_heads % c->n_kv_heads != 0 || n_q_heads / c->n_kv_heads > 64) return false;
    return in_range(n_seqs, 0, CTR_MAX_SEQS) && in_range(max_nodes, 1, CTR_MAX_NODES);
}

}  // namespace

extern "C" {

int ctr_kv_append(const ctr_kv_cache* cache, const ctr_rope* rope, ctr_rows q, ctr_rows k, ctr_rows v, ctr_rows q_out,
                  int64_t n_tokens, int32_t n_q_heads, const int64_t* positions, const int64_t* slots, void* stream)
{
    if (!valid_cache(cache) || !rope) return CTR_EINVAL;
    if (!in_range(n_tokens, 0, 2147483647LL) || !in_range(n_q_heads, 0, 4096)) return CTR_EINVAL;
    if (!in_range(rope->rot_dim, 0, cache->head_dim) || rope->rot_dim % 2 != 0) return CTR_EINVAL;
    if (rope->interleaved != 0 && rope->interleaved != 1) return CTR_EINVAL;
    if (!std::isfinite(rope->scale) || rope->reserved0 != 0) return CTR_EINVAL;
    if (n_tokens == 0) return CTR_OK;
    if (rope->rot_dim > 0 && (!rope->turns || !positions)) return CTR_EINVAL;
    if (!slots) return CTR_EINVAL;
    if (!valid_rows(k, n_tokens, cache->n_kv_heads, false) || !valid_rows(v, n_tokens, cache->n_kv_heads, false))
        return CTR_EINVAL;
    if (n_q_heads > 0 &&
        (!valid_rows(q, n_tokens, n_q_heads, false) || !valid_rows(q_out, n_tokens, n_q_heads, false)))
        return CTR_EINVAL;
    if (((uintptr_t)cache->k | (uintptr_t)cache->v) % 2u != 0) return CTR_EINVAL;
    AppendParams p;
    std::memset(&p, 0, sizeof(p));
    p.cache = *cache;
    p.rope = *rope;
    p.q = q;
    p.k = k;
    p.v = v;
    p.q_out = q_out;
    p.n_tokens = n_tokens;
    p.n_q_heads = n_q_heads;
    p.page_log2 = log2_of(cache->page_tokens);
    p.positions = positions;
    p.slots = slots;
    return cuda_status(launch_append(p, (cudaStream_t)stream));
}

size_t ctr_attention_workspace_bytes(const ctr_kv_cache* cache, int32_t n_q_heads, int32_t n_seqs, int32_t max_nodes)
{
    if (!valid_attention_sizes(cache, n_q_heads, n_seqs, max_nodes)) return 0;
    return attention_workspace(*cache, n_q_heads, n_seqs, max_nodes);
}

int ctr_tree_attention(const ctr_kv_cache* cache, ctr_rows q, ctr_rows out, int64_t n_rows, int32_t n_q_heads,
                       int32_t n_seqs, int32_t max_nodes, const int32_t* q_start, const int32_t* kv_len,
                       const int32_t* page_table, int32_t table_stride, const uint64_t* tree_mask, float scale,
                       float* lse, int32_t* status, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!valid_attention_sizes(cache, n_q_heads, n_seqs, max_nodes)) return CTR_EINVAL;
    if (!in_range(n_rows, 0, 2147483647LL) || !std::isfinite(scale)) return CTR_EINVAL;
    if (n_rows == 0 || n_seqs == 0) return CTR_OK;
    if (!q_start || !kv_len || !page_table || table_stride < 1) return CTR_EINVAL;
    if ((int64_t)table_stride > 2147483647LL / cache->page_tokens) return CTR_EINVAL;  // lengths are 32-bit
    if (!valid_rows(q, n_rows, n_q_heads, false) || !valid_rows(out, n_rows, n_q_heads, false)) return CTR_EINVAL;
    if (!aligned16(q.ptr, q.token_stride, q.head_stride) || !aligned16(out.ptr, out.token_stride, out.head_stride))
        return CTR_EINVAL;
    if (!aligned16(cache->k, cache->token_stride, cache->head_stride) || !aligned16(cache->v, cache->page_stride, 0))
        return CTR_EINVAL;
    if (!workspace || (uintptr_t)workspace % 256u != 0 ||
        workspace_bytes < attention_workspace(*cache, n_q_heads, n_seqs, max_nodes))
        return CTR_EINVAL;
    AttentionParams p;
    std::memset(&p, 0, sizeof(p));
    p.cache = *cache;
    p.q = q;
    p.out = out;
    p.n_rows = n_rows;
    p.n_q_heads = n_q_heads;
    p.group = n_q_heads / cache->n_kv_heads;
    p.n_seqs = n_seqs;
    p.max_nodes = max_nodes;
    p.table_stride = table_stride;
    p.page_log2 = log2_of(cache->page_tokens);
    p.q_start = q_start;
    p.kv_len = kv_len;
    p.page_table = page_table;
    p.tree_mask = tree_mask;
    p.scale_log2 = (float)((double)scale * 1.4426950408889634);
    p.group_magic = ((1u << 20) + (uint32_t)p.group - 1) / (uint32_t)p.group;
    p.lse = lse;
    p.status = status;
    p.ws = static_cast<unsigned char*>(workspace);
    return cuda_status(launch_attention(p, (cudaStream_t)stream));
}

int ctr_sample(const void* logits, int32_t dtype, int64_t row_stride, int64_t n_rows, int32_t vocab,
               const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, const float* u,
               int32_t* token, float* logprob, int32_t* n_kept, void* stream)
{
    if (dtype != CTR_BF16 && dtype != CTR_F16 && dtype != CTR_F32) return CTR_EINVAL;
    if (!in_range(n_rows, 0, 2147483647LL) || !in_range(vocab, 1, CTR_MAX_VOCAB)) return CTR_EINVAL;
    if (!in_range(row_stride, vocab, kStrideMax)) return CTR_EINVAL;
    if (n_rows == 0) return CTR_OK;
    if (row_stride > (1LL << 59) / n_rows) return CTR_EINVAL;
    if (!logits || !temperature || !u || !token) return CTR_EINVAL;
    if ((uintptr_t)logits % (dtype == CTR_F32 ? 4u : 2u) != 0) return CTR_EINVAL;
    SampleParams p;
    std::memset(&p, 0, sizeof(p));
    p.logits = logits;
    p.dtype = dtype;
    p.vocab = vocab;
    p.row_stride = row_stride;
    p.n_rows = n_rows;
    p.temperature = temperature;
    p.top_k = top_k;
    p.top_p = top_p;
    p.min_p = min_p;
    p.u = u;
    p.token = token;
    p.logprob = logprob;
    p.n_kept = n_kept;
    p.minus_zeros = 0x8000000080000000ull;
    return cuda_status(launch_sample(p, (cudaStream_t)stream));
}

}  // extern "C"
