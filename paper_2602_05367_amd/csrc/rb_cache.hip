// Tokens enter a paged cache, their rotary embedding on the way: bytes in, bytes out.
#include <hip/hip_runtime.h>

#include "rabit.h"
#include "rb_attn.h"
#include "rb_attn_host.h"

namespace rb {
namespace attn {
namespace {

struct AppendArgs {
    Side q, k, v;
    Address k_to, v_to, q_to, cos, sin, first, lengths, table;
    long long page, token_stride, head_stride;      // of the cache, in bytes
    int n_seqs, tokens, heads, kv_heads, dim, rotary, table_rows, pages, page_shift, width, blocks;
};

// Element pairs (x, y) of a head become (x cos - y sin, y cos + x sin), products and sum in fp32 and rounded once.  Eight elements per thread, so loads and stores are
// of eight bytes or sixteen: four of either half of a head, or eight in a row where pairs are neighbours or nothing is turned.  A workgroup has elements of one token and finds its sequence itself.
// Bound: bytes (sixteen prompts of 6000 tokens in all, 64 and 8 heads of 128, bf16: 42 us, 5.8 TB/s); one token: latencies, 3 us.  The elements are
// on their way while the place is looked up (after it: 44 us).
template <class T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void append_kernel(const AppendArgs A)
{
    const int token = workgroup() / A.blocks, part = workgroup() % A.blocks, lane = threadIdx.x & 63;
    if (token >= A.tokens) return;
    const int pieces = A.dim / 8, unit = part * 256 + threadIdx.x, head = unit / pieces, piece = unit % pieces;
    const bool there = head < A.heads + 2 * A.kv_heads;
    const bool is_q = head < A.heads, is_v = head >= A.heads + A.kv_heads, turned = !is_v && piece * 8 < A.rotary;
    const int kvh = is_q ? head : head - A.heads - (is_v ? A.kv_heads : 0);
    const int at_x = piece * (INTERLEAVED || !turned ? 16 : 8), at_y = INTERLEAVED || !turned ? at_x + 8 : at_x + A.rotary;      // bytes
    Four a = {}, b = {};
    if (there) {      // on the way while the place is looked up
        const Side &from_side = is_q ? A.q : is_v ? A.v : A.k;
        const uint8_t *from = global_at<const uint8_t>(from_side.at) + token * from_side.token + kvh * from_side.head;
        a.w = *(const v2u *)(from + at_x);
        b.w = *(const v2u *)(from + at_y);
    }
    const int *first = global_at<const int>(A.first), *lengths = global_at<const int>(A.lengths);
    int s, end, length;
    sequence_of_token(first, lengths, A.n_seqs, token, lane, s, end, length);
    const long long position = (long long)length - end + token;
    const bool inside = position >= 0 && position < (long long)A.width << A.page_shift;
    if (!there || token >= end) return;      // behind the last sequence's end (padding): nobody's
    uint8_t *to;
    if (is_q) {
        to = global_at<uint8_t>(A.q_to) + ((long long)token * A.heads + head) * (A.dim * 2);
    } else {
        if (!inside) return;
        const int p = (int)position, page = global_at<const int>(A.table)[(long long)s * A.width + (p >> A.page_shift)];
        if (page < 0 || page >= A.pages) return;      // (another's page is not written over)
        to = global_at<uint8_t>(is_v ? A.v_to : A.k_to) + (long long)page * A.page + (p & ((1 << A.page_shift) - 1)) * A.token_stride + kvh * A.head_stride;
    }
    if (!turned) {
        *(v4u *)(to + at_x) = (v4u){a.w.x, a.w.y, b.w.x, b.w.y};
        return;
    }
    const long long row = min(max(position, 0ll), (long long)A.table_rows - 1) * (A.rotary / 2) + piece * 4;
    const v4f c = *(const v4f *)(global_at<const float>(A.cos) + row), sn = *(const v4f *)(global_at<const float>(A.sin) + row);
    float x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float u = T::widen(INTERLEAVED ? (i < 2 ? a.h[2 * i] : b.h[2 * i - 4]) : a.h[i]);
        const float w = T::widen(INTERLEAVED ? (i < 2 ? a.h[2 * i + 1] : b.h[2 * i - 3]) : b.h[i]);
        x[i] = u * c[i] - w * sn[i];
        y[i] = w * c[i] + u * sn[i];
    }
    if (INTERLEAVED) {
        a.w = (v2u){T::pack(x[0], y[0]), T::pack(x[1], y[1])};
        b.w = (v2u){T::pack(x[2], y[2]), T::pack(x[3], y[3])};
    } else {
        a.w = (v2u){T::pack(x[0], x[1]), T::pack(x[2], x[3])};
        b.w = (v2u){T::pack(y[0], y[1]), T::pack(y[2], y[3])};
    }
    *(v2u *)(to + at_x) = a.w;
    *(v2u *)(to + at_y) = b.w;
}

}  // namespace
}  // namespace attn
}  // namespace rb

using namespace rb::attn;

extern "C" int rb_cache_append(const rb_cache *C, const rb_heads *H, const void *q, const void *k, const void *v, const float *cos, const float *sin, int table_rows,
                               int rotary, int interleaved, const int32_t *first, const int32_t *lengths, const int32_t *table, int width, int n_seqs, int tokens,
                               void *q_out, void *stream)
{
    int rc = check_cache(C);
    if (rc != RB_OK) return rc;
    rc = check_heads(H);
    if (rc != RB_OK) return rc;
    if (!k || !v || !first || !lengths || !table || !q != !q_out || !cos != !sin) return RB_ERR_NULL;
    if (H->kv_heads != C->kv_heads || H->dim != C->dim || H->dtype != C->dtype) return RB_ERR_SHAPE;
    if (n_seqs < 1 || n_seqs > MAX_SEQS || tokens < 1 || tokens > MAX_TOKENS || width < 1) return RB_ERR_SHAPE;
    if (cos && (table_rows < 1 || rotary < 8 || rotary % 8 != 0 || rotary > C->dim)) return RB_ERR_SHAPE;
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out | (uintptr_t)cos | (uintptr_t)sin) & 15) return RB_ERR_ALIGN;
    if (((uintptr_t)first | (uintptr_t)lengths | (uintptr_t)table) & 3) return RB_ERR_ALIGN;
    AppendArgs A = {};
    A.q = side(q, H->q_token, H->q_head), A.k = side(k, H->k_token, H->k_head), A.v = side(v, H->v_token, H->v_head);
    A.k_to = rb::address_of(C->k), A.v_to = rb::address_of(C->v), A.q_to = rb::address_of(q_out);
    A.cos = rb::address_of(cos), A.sin = rb::address_of(sin);
    A.first = rb::address_of(first), A.lengths = rb::address_of(lengths), A.table = rb::address_of(table);
    A.page = C->page_stride * 2, A.token_stride = C->token_stride * 2, A.head_stride = C->head_stride * 2;
    A.n_seqs = n_seqs, A.tokens = tokens, A.heads = q ? H->heads : 0, A.kv_heads = H->kv_heads, A.dim = H->dim;
    A.rotary = cos ? rotary : 0, A.table_rows = table_rows, A.pages = C->pages, A.page_shift = __builtin_ctz((unsigned)C->page_tokens), A.width = width;
    A.blocks = (int)(((long long)(A.heads + 2 * A.kv_heads) * (A.dim / 8) + 255) / 256);
    const long long n = (long long)tokens * A.blocks;
    if (n > 0x7fffffffll) return RB_ERR_SHAPE;
    const dim3 grid = workgroups(n), threads(256);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (H->dtype == RB_F16) {
        if (interleaved)
            hipLaunchKernelGGL((append_kernel<F16, true>), grid, threads, 0, st, A);
        else
            hipLaunchKernelGGL((append_kernel<F16, false>), grid, threads, 0, st, A);
    } else {
        if (interleaved)
            hipLaunchKernelGGL((append_kernel<BF16, true>), grid, threads, 0, st, A);
        else
            hipLaunchKernelGGL((append_kernel<BF16, false>), grid, threads, 0, st, A);
    }
    return hipGetLastError() == hipSuccess ? RB_OK : RB_ERR_HIP;
}
