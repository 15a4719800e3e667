// Shared by the attention kernels (include/nq.h: nq_head_norm, nq_cache_read, nq_attention_prompt, nq_attention_token): a cache
// descriptor as a kernel takes it, and the host-side checks.
#pragma once
#include "nq_fp8.h"

namespace nq {

// nq_kv_cache by value, with what finds a token's page.
struct CacheView {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    int64_t page_step, token_step, head_step, scale_page_step, scale_token_step, scale_head_step;
    int64_t slots;
    Divider by_page;
    int32_t pages, type;
};

struct Place {
    int64_t page;
    int64_t token;
};
// (slots past 2^31 take the long division: some hundred instructions, for a token's whole row)
__device__ __forceinline__ Place place_of(const CacheView &c, int64_t slot)
{
    const int64_t page = slot < (int64_t(1) << 31) ? (int64_t)divide((uint32_t)slot, c.by_page) : (int64_t)((uint64_t)slot / c.by_page.d);
    return Place{page, slot - page * c.by_page.d};
}

// Sum over the lanes before this one, and over all.
__device__ __forceinline__ int before(int v, int *all)
{
    int x = v;
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);      // one, two, four and eight lanes on in the row of sixteen
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // the row before's last to the second and fourth row
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);      // the half's last to the other half
    *all = __builtin_amdgcn_readlane(x, 63);
    return x - v;
}
// ---- host ------------------------------------------------------------------------------------------------------

// (a row of heads of floats is at most 2^32 elements away from the next, as check_matrix has it)
constexpr int64_t KV_MAX_STEP = int64_t(1) << 26, KV_MAX_PAGE_STEP = int64_t(1) << 40, ATT_MAX_ROWS = (int64_t(1) << 30) - 4096;     // (two of them and a tile fit 31 bits)

inline nq_status check_heads(int q_heads, int kv_heads, int head_dim)
{
    if (q_heads < 1 || kv_heads < 1 || head_dim < 1) return NQ_ERR_INVALID_ARG;
    if (q_heads > NQ_MAX_HEADS || kv_heads > NQ_MAX_HEADS || head_dim > NQ_HEAD_MAX_DIM || head_dim % 8) return NQ_ERR_SHAPE;
    return NQ_OK;
}

inline nq_status check_cache(const nq_kv_cache *c)
{
    if (!c || c->pages < 0 || c->page_tokens < 1) return NQ_ERR_INVALID_ARG;
    if (c->type < NQ_KV_F16 || c->type > NQ_KV_E4M3) return NQ_ERR_INVALID_ARG;
    nq_status st = check_heads(c->heads, c->heads, c->head_dim);
    if (st != NQ_OK) return st;
    if (c->page_step < 0 || c->token_step < 0 || c->head_step < 0) return NQ_ERR_INVALID_ARG;
    if (c->pages > INT32_MAX || c->page_tokens > (1 << 20)) return NQ_ERR_SHAPE;
    if (c->page_step > KV_MAX_PAGE_STEP || c->token_step > KV_MAX_STEP || c->head_step > KV_MAX_STEP) return NQ_ERR_SHAPE;
    if (c->type == NQ_KV_E4M3) {
        if (c->scale_page_step < 0 || c->scale_token_step < 0 || c->scale_head_step < 0) return NQ_ERR_INVALID_ARG;
        if (c->scale_page_step > KV_MAX_PAGE_STEP || c->scale_token_step > KV_MAX_STEP || c->scale_head_step > KV_MAX_STEP) return NQ_ERR_SHAPE;
    }
    if (c->pages == 0) return NQ_OK;
    if (!c->d_k || !c->d_v) return NQ_ERR_INVALID_ARG;
    if (c->type != NQ_KV_E4M3) return aligned_to(c->d_k, 2) && aligned_to(c->d_v, 2) ? NQ_OK : NQ_ERR_ALIGN;
    if (!c->d_k_scale || !c->d_v_scale) return NQ_ERR_INVALID_ARG;
    return aligned_to(c->d_k_scale, 4) && aligned_to(c->d_v_scale, 4) ? NQ_OK : NQ_ERR_ALIGN;
}

inline CacheView view_of(const nq_kv_cache &c)
{
    CacheView v;
    v.k = static_cast<uint8_t *>(c.d_k);
    v.v = static_cast<uint8_t *>(c.d_v);
    v.k_scale = c.d_k_scale;
    v.v_scale = c.d_v_scale;
    v.page_step = c.page_step;
    v.token_step = c.token_step;
    v.head_step = c.head_step;
    v.scale_page_step = c.scale_page_step;
    v.scale_token_step = c.scale_token_step;
    v.scale_head_step = c.scale_head_step;
    v.slots = c.pages * c.page_tokens;
    v.by_page = make_divider((uint32_t)c.page_tokens);
    v.pages = (int32_t)c.pages;
    v.type = c.type;
    return v;
}

}  // namespace nq
