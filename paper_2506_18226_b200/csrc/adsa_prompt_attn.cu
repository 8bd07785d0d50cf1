// Attention of many query rows per sequence: whole prompts laid end to end (adsa_packed_attn), and a chunk of new tokens over a
// paged cache with a prefix that sequences share (adsa_chunk_attn).
#include <math.h>

#include "adsa_prompt.cuh"

namespace adsa {

constexpr int kPromptMaxBatch = 4000;        // the list of their work lies in shared memory, beside the tiles
// Tokens of a call, packed rows of a call, rows a table and a prefix's have room for: numbers of tokens and rows stay in 32 bits past the last tile, and past the
// last item too, where a warp looks at 32 items of up to 256 tokens at a time.
constexpr long long kPromptMaxRows = 0x7fffffffLL - 32 * 256 - 256;
constexpr int kPromptMaxPerKv = 64;

namespace {

int g_polls = -1;                            // of a wait inside the kernels; below 0: by the rows a sequence can have

// A poll waits for 4 us itself.  A second, and 50 us a tile for what waits while the five items before it run (2 us a tile, 20 by row copies).
int polls_for(long long rows)
{
    const int polls = __atomic_load_n(&g_polls, __ATOMIC_RELAXED);
    return polls >= 0 ? polls : (1 << 18) + 64 * (int)(rows / kTileRows + 2);
}

int sm_count()
{
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return 148;
    }
    return n;
}

bool heads_ok(int n_heads, int n_kv_heads, int head_dim)
{
    return n_kv_heads >= 1 && n_heads >= n_kv_heads && n_heads % n_kv_heads == 0 && n_heads / n_kv_heads <= kPromptMaxPerKv && head_dim >= 2 &&
           head_dim % 2 == 0 && head_dim <= ADSA_MAX_HEAD_DIM;
}

// what both calls ask of q, the outputs and the workspace
bool rows_ok(const void *q, long long q_token, long long q_head, int batch, long long n_q, int n_heads, float softmax_scale, const void *out,
             const float *out_f32, const float *lse, const int32_t *cu_q, const void *workspace)
{
    if (!q || batch < 1 || batch > kPromptMaxBatch || n_q > kPromptMaxRows || n_q * n_heads > 0x7fffffffLL || (!cu_q && n_q % batch)) return false;
    if ((!out && !out_f32) || !(softmax_scale >= 0.f) || !workspace) return false;
    if (((uintptr_t)q & 3) || q_token % 2 || q_head % 2 || ((uintptr_t)workspace & 255) || ((uintptr_t)out & 3) || ((uintptr_t)out_f32 & 7)) return false;
    return (((uintptr_t)lse | (uintptr_t)cu_q) & 3) == 0;
}

}  // namespace
}  // namespace adsa

using namespace adsa;

extern "C" {

int adsa_prompt_workspace_bytes(int batch, int n_heads, int n_kv_heads, int head_dim, size_t *out_bytes)
{
    if (!out_bytes || batch < 1 || batch > kPromptMaxBatch || !heads_ok(n_heads, n_kv_heads, head_dim)) return ADSA_EINVAL;
    *out_bytes = prompt_workspace(head_dim, sm_count(), nullptr, nullptr);
    return ADSA_OK;
}

int adsa_prompt_wait_polls(int polls) { return __atomic_exchange_n(&g_polls, polls < 0 ? -1 : polls, __ATOMIC_RELAXED); }

int adsa_packed_attn(int dtype, const void *q, long long q_token, long long q_head, const void *k, long long k_token, long long k_head,
                     const void *v, long long v_token, long long v_head, const int32_t *cu_q, const int32_t *cu_k, int batch, long long n_q,
                     long long n_k, int n_heads, int n_kv_heads, int head_dim, int causal, float softmax_scale, void *out, float *out_f32,
                     float *lse, void *workspace, size_t workspace_bytes, adsa_stream_t stream)
{
    return adsa_packed_attn_status(dtype, q, q_token, q_head, k, k_token, k_head, v, v_token, v_head, cu_q, cu_k, batch, n_q, n_k, n_heads, n_kv_heads, head_dim,
                                   causal, softmax_scale, out, out_f32, lse, workspace, workspace_bytes, nullptr, stream);
}

int adsa_packed_attn_status(int dtype, const void *q, long long q_token, long long q_head, const void *k, long long k_token, long long k_head,
                            const void *v, long long v_token, long long v_head, const int32_t *cu_q, const int32_t *cu_k, int batch, long long n_q,
                            long long n_k, int n_heads, int n_kv_heads, int head_dim, int causal, float softmax_scale, void *out, float *out_f32,
                            float *lse, void *workspace, size_t workspace_bytes, uint32_t *status, adsa_stream_t stream)
{
    size_t bytes = 0;
    if ((dtype != ADSA_BF16 && dtype != ADSA_F16) || !heads_ok(n_heads, n_kv_heads, head_dim) || n_q < 0 || n_k < 0) return ADSA_EINVAL;
    if (n_q == 0) return ADSA_OK;
    if (!rows_ok(q, q_token, q_head, batch, n_q, n_heads, softmax_scale, out, out_f32, lse, cu_q, workspace)) return ADSA_EINVAL;
    if ((n_k && (!k || !v)) || n_k > kPromptMaxRows || (!cu_k && n_k % batch)) return ADSA_EINVAL;
    if (((uintptr_t)k & 3) || k_token % 2 || k_head % 2 || ((uintptr_t)v & 3) || v_token % 2 || v_head % 2 || (((uintptr_t)cu_k | (uintptr_t)status) & 3))
        return ADSA_EINVAL;
    if (adsa_prompt_workspace_bytes(batch, n_heads, n_kv_heads, head_dim, &bytes) != ADSA_OK) return ADSA_EINVAL;
    if (workspace_bytes < bytes) return ADSA_ENOMEM;
    PromptArgs a = {};
    a.q = q; a.q_token = q_token; a.q_head = q_head;
    a.k = k; a.k_token = k_token; a.k_head = k_head;
    a.v = v; a.v_token = v_token; a.v_head = v_head;
    a.cu_q = cu_q; a.cu_k = cu_k; a.batch = batch; a.n_q = n_q; a.n_k = n_k;
    a.kv_heads = n_kv_heads; a.per_kv = n_heads / n_kv_heads; a.d = head_dim; a.causal = causal != 0;
    a.scale_log2e = (softmax_scale == 0.f ? 1.0f / sqrtf((float)head_dim) : softmax_scale) * 1.44269504088896341f;
    a.out = out; a.out_f32 = out_f32; a.lse = lse; a.status = status;
    a.polls = polls_for(n_k);
    const int sms = sm_count();
    prompt_workspace(head_dim, sms, &a, workspace);
    return launch_prompt_tiles(dtype, a, sms, (cudaStream_t)stream) == cudaSuccess ? ADSA_OK : ADSA_ECUDA;
}

int adsa_chunk_attn(const adsa_paged_kv *kv, const void *q, long long q_token, long long q_head, const int32_t *cu_tokens, int batch,
                    long long n_tokens, int n_heads, const int32_t *page_table, int max_pages, const int32_t *n_rows,
                    const int32_t *prefix_table, int max_prefix_pages, const int32_t *prefix_rows, const int32_t *group_start, int n_groups,
                    float softmax_scale, void *out, float *out_f32, float *lse, void *workspace, size_t workspace_bytes, uint32_t *status,
                    adsa_stream_t stream)
{
    size_t bytes = 0;
    if (!paged_kv_ok(kv) || !heads_ok(n_heads, kv->n_kv_heads, kv->head_dim) || n_tokens < 0 || n_groups < 0 || max_pages < 1) return ADSA_EINVAL;
    if (n_tokens == 0) return ADSA_OK;
    if (!rows_ok(q, q_token, q_head, batch, n_tokens, n_heads, softmax_scale, out, out_f32, lse, cu_tokens, workspace)) return ADSA_EINVAL;
    if (!page_table || !n_rows || n_groups > kPromptMaxBatch) return ADSA_EINVAL;
    if (n_groups && (!prefix_table || !prefix_rows || !group_start || max_prefix_pages < 1)) return ADSA_EINVAL;
    if (((uintptr_t)page_table | (uintptr_t)n_rows | (uintptr_t)prefix_table | (uintptr_t)prefix_rows | (uintptr_t)group_start | (uintptr_t)status) & 3)
        return ADSA_EINVAL;
    if (((long long)max_pages + (n_groups ? max_prefix_pages : 0)) * kv->page_rows > kPromptMaxRows) return ADSA_EINVAL;   // (rows of both are added up)
    if (adsa_prompt_workspace_bytes(batch, n_heads, kv->n_kv_heads, kv->head_dim, &bytes) != ADSA_OK) return ADSA_EINVAL;
    if (workspace_bytes < bytes) return ADSA_ENOMEM;
    PromptArgs a = {};
    a.q = q; a.q_token = q_token; a.q_head = q_head;
    a.k = kv->k_pool; a.v = kv->v_pool;
    a.cu_q = cu_tokens; a.batch = batch; a.n_q = n_tokens;
    a.table = page_table; a.max_pages = max_pages; a.n_rows = n_rows;
    a.p_table = prefix_table; a.max_p_pages = max_prefix_pages; a.p_rows = prefix_rows; a.start = group_start; a.groups = n_groups;
    a.page_rows = kv->page_rows; a.n_pages = kv->n_pages; a.row_stride = kv->row_stride; a.status = status;
    a.kv_heads = kv->n_kv_heads; a.per_kv = n_heads / kv->n_kv_heads; a.d = kv->head_dim; a.causal = 1;
    a.scale_log2e = (softmax_scale == 0.f ? 1.0f / sqrtf((float)kv->head_dim) : softmax_scale) * 1.44269504088896341f;
    a.out = out; a.out_f32 = out_f32; a.lse = lse;
    a.polls = polls_for(((long long)max_pages + (n_groups ? max_prefix_pages : 0)) * kv->page_rows);
    const int sms = sm_count();
    prompt_workspace(kv->head_dim, sms, &a, workspace);
    return launch_prompt_tiles(kv->dtype, a, sms, (cudaStream_t)stream) == cudaSuccess ? ADSA_OK : ADSA_ECUDA;
}

}  // extern "C"
