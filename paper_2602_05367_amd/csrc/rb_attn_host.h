// Argument checks shared by the attention and cache entry points.
#pragma once
#include <initializer_list>

#include "rabit.h"
#include "rb_attn.h"

namespace rb {
namespace attn {

// the 64 rows of a tile are addressed by 32 bits, everything above them by 64
constexpr long long MAX_STRIDE = 1ll << 23, MAX_PAGE_STRIDE = 1ll << 40;
// products of a token and a group, and the positions of a cache, stay within 31 bits
constexpr int MAX_SEQS = 1 << 20, MAX_TOKENS = 1 << 24, MAX_PAGE = 1 << 16;

int check_heads(const rb_heads *H);
int check_scale(float scale);

inline int check_cache(const rb_cache *C)
{
    if (!C || !C->k || !C->v) return RB_ERR_NULL;
    if (C->pages < 1 || C->kv_heads < 1 || C->kv_heads > 65536 || C->dim < 8 || C->dim % 8 != 0) return RB_ERR_SHAPE;
    if (C->page_tokens < 8 || C->page_tokens > MAX_PAGE || (C->page_tokens & (C->page_tokens - 1)) != 0) return RB_ERR_SHAPE;
    if (C->dim > 128 || (C->dtype != RB_F16 && C->dtype != RB_BF16)) return RB_ERR_UNSUPPORTED;
    if (C->page_stride < 0 || C->page_stride > MAX_PAGE_STRIDE) return RB_ERR_SHAPE;
    for (const long long s : {C->token_stride, C->head_stride})
        if (s < 0 || s > MAX_STRIDE) return RB_ERR_SHAPE;
    if ((C->page_stride | C->token_stride | C->head_stride) % 8 != 0) return RB_ERR_ALIGN;
    if (((uintptr_t)C->k | (uintptr_t)C->v) & 15) return RB_ERR_ALIGN;
    return RB_OK;
}

inline int check_cache8(const rb_cache8 *C)
{
    if (!C || !C->k || !C->v || !C->k_exp || !C->v_exp) return RB_ERR_NULL;
    const rb_cache pages = {C->k, C->v, C->pages, C->page_tokens, C->kv_heads, C->dim, C->dtype, C->page_stride, C->token_stride, C->head_stride};
    const int rc = check_cache(&pages);
    if (rc != RB_OK) return rc;
    if (C->token_stride < C->dim) return RB_ERR_SHAPE;      // (rows past a sequence's end are told by where they lie)
    if (C->dim % 16 != 0) return RB_ERR_UNSUPPORTED;
    if ((C->page_stride | C->token_stride | C->head_stride) % 16 != 0 || ((uintptr_t)C->k_exp | (uintptr_t)C->v_exp) & 7) return RB_ERR_ALIGN;
    return RB_OK;
}

// Rows that a workgroup joins the parts of, where `jobs` have up to `rows` of them: two where that is few workgroups, else eight, since many of the workgroups find
// no work (130 decoding sequences of 8 heads 61 us with two everywhere and 41 so, 512 new tokens 31 and 23; one sequence of 32 heads 0.5 us less with two).
inline int rows_joined(long long jobs, long long rows) { return jobs * rows <= 2048 ? 2 : 8; }

// paged calls with few rows per sequence (rb_attn_few.hip), of sequences of up to `positions` positions
bool few_applies(int tokens, int n_seqs, int group, long long positions);
size_t few_workspace_bytes(int kv_heads, int dim, int compute_units);
int launch_few(const Args &A, int dtype, int compute_units, hipStream_t stream);
// the same over a cache in 8 bits (rb_attn_few8.hip)
size_t few8_workspace_bytes(int kv_heads, int dim, int compute_units);
int launch_few8(const Args &A, int dtype, int compute_units, hipStream_t stream);

inline Side side(const void *p, long long token, long long head) { return {rb::address_of(p), token * 2, head * 2}; }

}  // namespace attn
}  // namespace rb
