// Tokens enter a paged cache in 8 bits, their rotary embedding on the way, and come back out of it: bytes in, bytes out.
#include <hip/hip_runtime.h>

#include "rabit.h"
#include "rb_attn.h"
#include "rb_attn8.h"
#include "rb_attn_host.h"

namespace rb {
namespace attn {
namespace {

struct Cache8Args {
    Address k, v, k_exp, v_exp, first, lengths, table;
    long long page, token_stride, head_stride;      // of k and v, in bytes
    int n_seqs, tokens, kv_heads, dim, pages, page_shift, width;
};
Cache8Args cache8_args(const rb_cache8 *C, const int32_t *first, const int32_t *lengths, const int32_t *table, int width, int n_seqs, int tokens)
{
    return {rb::address_of(C->k), rb::address_of(C->v), rb::address_of(C->k_exp), rb::address_of(C->v_exp), rb::address_of(first), rb::address_of(lengths), rb::address_of(table),
            C->page_stride, C->token_stride, C->head_stride, n_seqs, tokens, C->kv_heads, C->dim, C->pages, __builtin_ctz((unsigned)C->page_tokens), width};
}
struct Append8Args {
    Cache8Args c;
    Side q, k_from, v_from;
    Address q_to, cos, sin;
    int heads, rotary, table_rows, blocks, lanes_shift, query_units;      // lanes of a head: the power of two that holds its pieces; threads of a token for its queries
};

// Where a position lies in the cache, behind the first head's elements and exponents; false: nowhere
__device__ __forceinline__ bool place_of(const Cache8Args &C, int s, long long position, long long &elements, long long &exponents)
{
    if (position < 0 || position >= (long long)C.width << C.page_shift) return false;
    const int p = (int)position, page = global_at<const int>(C.table)[(long long)s * C.width + (p >> C.page_shift)], row = p & ((1 << C.page_shift) - 1);
    if (page < 0 || page >= C.pages) return false;
    elements = page * C.page + row * C.token_stride;
    exponents = (((long long)page * C.kv_heads) << C.page_shift) + row;
    return true;
}

// Element pairs are turned as in append_kernel (rb_cache.hip), eight elements per thread: four of either half of a head, or eight in a row.  Keys and values are then held in
// units of a power of two of the head's own, so x / unit is exact and the one rounding is that to e4m3: the largest |x| of the head is found
// among its lanes, a power of two of them.  A workgroup has elements of one token and finds its sequence itself; a wavefront has queries, two heads to a thread, or keys and values.
//
// Bound: bytes, and for a single token the launch (one token, 40 heads of 128: 3.8 us).  16 prompts of 5992 tokens together, 64 heads of 128 over 8 of keys, interleaved (233 MB): 41 us,
// 5.6 TB/s, a copy of as many bytes 36; 47 with one head of queries to a thread or four, 57 with these in pieces of 8 bytes and loads that lanes without a head branch around.
constexpr int QUERIES = 2;
template <class T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void append8_kernel(const Append8Args A)
{
    const Cache8Args &C = A.c;
    const int token = workgroup() / A.blocks, part = workgroup() % A.blocks, lane = threadIdx.x & 63;
    if (token >= C.tokens) return;
    const int first_unit = __builtin_amdgcn_readfirstlane(part * 256 + (threadIdx.x & 192)), unit = first_unit + lane;
    const bool queries = first_unit < A.query_units;      // (whole wavefronts)
    const int piece = unit & ((1 << A.lanes_shift) - 1), head = queries ? (unit >> A.lanes_shift) * QUERIES : (unit - A.query_units) >> A.lanes_shift;
    const bool is_v = !queries && head >= C.kv_heads, turned = !is_v && piece * 8 < A.rotary;
    const int heads = queries ? A.heads : 2 * C.kv_heads, mine = piece * 8 < C.dim ? min(heads - head, queries ? QUERIES : 1) : 0, kvh = is_v ? head - C.kv_heads : head;
    const int at_x = piece * (INTERLEAVED || !turned ? 8 : 4), at_y = INTERLEAVED || !turned ? at_x + 4 : at_x + A.rotary / 2;      // elements
    Four a[QUERIES] = {}, b[QUERIES] = {};
    {      // on the way while the place is looked up; lanes without a head, or with fewer, load others again
        const bool there = mine > 0;
        const Address side_at = queries ? A.q.at : is_v ? A.v_from.at : A.k_from.at;
        const long long token_step = queries ? A.q.token : is_v ? A.v_from.token : A.k_from.token, head_step = queries ? A.q.head : is_v ? A.v_from.head : A.k_from.head;
        const uint8_t *from = global_at<const uint8_t>(side_at) + token * token_step + (there ? kvh * head_step : 0);
        const int x = there ? at_x * 2 : 0;
        [[maybe_unused]] const int y = there ? at_y * 2 : 0;
#pragma unroll
        for (int i = 0; i < QUERIES; ++i)
            if (i == 0 || queries) {
                const uint8_t *head_from = from + min(i, max(mine - 1, 0)) * head_step;
                if constexpr (INTERLEAVED) {
                    const v4u w = *(const v4u *)(head_from + x);
                    a[i].w = (v2u){w.x, w.y}, b[i].w = (v2u){w.z, w.w};
                } else {
                    a[i].w = *(const v2u *)(head_from + x), b[i].w = *(const v2u *)(head_from + y);
                }
            }
    }
    int s, end, length;
    sequence_of_token(global_at<const int>(C.first), global_at<const int>(C.lengths), C.n_seqs, token, lane, s, end, length);
    if (token >= end) return;      // behind the last sequence's end (padding): nobody's
    const long long position = (long long)length - end + token;
    v4f c = {}, sn = {};
    if (turned && mine > 0) {
        const long long row = min(max(position, 0ll), (long long)A.table_rows - 1) * (A.rotary / 2) + piece * 4;
        c = *(const v4f *)(global_at<const float>(A.cos) + row), sn = *(const v4f *)(global_at<const float>(A.sin) + row);
    }
    float x[4], y[4];      // the elements from at_x and at_y on
    auto turn = [&](const Four &u, const Four &w) RB_INLINE {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = T::widen(u.h[i]), y[i] = T::widen(w.h[i]);
        if (!turned) return;
        auto pair = [&](float &f, float &g, int i) RB_INLINE {
            const float t = f * c[i] - g * sn[i];
            g = g * c[i] + f * sn[i];
            f = t;
        };
        if constexpr (INTERLEAVED) {
            pair(x[0], x[1], 0), pair(x[2], x[3], 1), pair(y[0], y[1], 2), pair(y[2], y[3], 3);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) pair(x[i], y[i], i);
        }
    };
    if (queries) {
        uint8_t *to = global_at<uint8_t>(A.q_to) + ((long long)token * A.heads + head) * (C.dim * 2);
#pragma unroll
        for (int i = 0; i < QUERIES; ++i)
            if (i < mine) {
                turn(a[i], b[i]);
                const v4u w = turned ? (v4u){T::pack(x[0], x[1]), T::pack(x[2], x[3]), T::pack(y[0], y[1]), T::pack(y[2], y[3])} : (v4u){a[i].w.x, a[i].w.y, b[i].w.x, b[i].w.y};
                uint8_t *const head_to = to + i * C.dim * 2;
                if (INTERLEAVED || !turned) {      // 16 bytes in a row
                    *(v4u *)(head_to + at_x * 2) = w;
                } else {
                    *(v2u *)(head_to + at_x * 2) = (v2u){w.x, w.y};
                    *(v2u *)(head_to + at_y * 2) = (v2u){w.z, w.w};
                }
            }
        return;
    }
    long long elements, exponents;
    if (!place_of(C, s, position, elements, exponents)) return;      // (another's page is not written over)
    turn(a[0], b[0]);
    // the head's exponent, in every lane of it
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = fmaxf(most, fmaxf(bounded8<T>(x[i]), bounded8<T>(y[i])));
    if (mine <= 0) most = 0.f;
    for (int d = 1; d < 1 << A.lanes_shift; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
    if (mine <= 0) return;
    const int exponent = exponent8(most);
    const Address to_at = is_v ? C.v : C.k, exponents_at = is_v ? C.v_exp : C.k_exp;
    uint8_t *to = global_at<uint8_t>(to_at) + elements + kvh * C.head_stride;
    *(uint32_t *)(to + at_x) = narrow8<T>(x, exponent);
    *(uint32_t *)(to + at_y) = narrow8<T>(y, exponent);
    if (piece == 0) global_at<uint8_t>(exponents_at)[exponents + ((long long)kvh << C.page_shift)] = (uint8_t)exponent;
}

// Sixteen elements of a key and of its value per thread: two loads, four stores.  A wavefront has elements of one token.
// Bound: bytes.  16 sequences of 8 heads of 128, 100000 positions together (616 MB): 116 us, a copy of as many bytes 114; with loads that the caches keep 120, with stores that they do not 187; 333 tokens of 12 heads of 80: 3.4 us, the launch.
template <class T>
__global__ __launch_bounds__(256) void read8_kernel(const Cache8Args C, Address k_to, Address v_to, int waves)      // wavefronts of a token
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(workgroup() * 4 + (threadIdx.x >> 6)), token = wave / waves;
    if (token >= C.tokens) return;
    const int pieces = C.dim / 16, unit = wave % waves * 64 + lane, head = unit / pieces, piece = unit % pieces;
    int s, end, length;
    sequence_of_token(global_at<const int>(C.first), global_at<const int>(C.lengths), C.n_seqs, token, lane, s, end, length);
    if (token >= end || head >= C.kv_heads) return;
    long long elements, exponents;
    v4u w[2] = {};
    uint32_t exponent[2] = {};
    if (place_of(C, s, (long long)length - end + token, elements, exponents)) {
        elements += head * C.head_stride + piece * 16, exponents += (long long)head << C.page_shift;
        w[0] = __builtin_nontemporal_load((const v4u *)(global_at<const uint8_t>(C.k) + elements)), w[1] = __builtin_nontemporal_load((const v4u *)(global_at<const uint8_t>(C.v) + elements));
        exponent[0] = global_at<const uint8_t>(C.k_exp)[exponents], exponent[1] = global_at<const uint8_t>(C.v_exp)[exponents];
    }
    const long long at = (((long long)token * C.kv_heads + head) * C.dim + piece * 16) * 2;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint8_t *to = global_at<uint8_t>(i ? v_to : k_to) + at;
        *(v4u *)to = widen8<T>((v2u){w[i].x, w[i].y}, unit8(exponent[i]));
        *(v4u *)(to + 16) = widen8<T>((v2u){w[i].z, w[i].w}, unit8(exponent[i]));
    }
}

}  // namespace
}  // namespace attn
}  // namespace rb

using namespace rb::attn;

extern "C" int rb_cache8_append(const rb_cache8 *C, const rb_heads *H, const void *q, const void *k, const void *v, const float *cos, const float *sin, int table_rows,
                                int rotary, int interleaved, const int32_t *first, const int32_t *lengths, const int32_t *table, int width, int n_seqs, int tokens,
                                void *q_out, void *stream)
{
    int rc = check_cache8(C);
    if (rc != RB_OK) return rc;
    rc = check_heads(H);
    if (rc != RB_OK) return rc;
    if (!k || !v || !first || !lengths || !table || !q != !q_out || !cos != !sin) return RB_ERR_NULL;
    if (H->kv_heads != C->kv_heads || H->dim != C->dim || H->dtype != C->dtype) return RB_ERR_SHAPE;
    if (n_seqs < 1 || n_seqs > MAX_SEQS || tokens < 1 || tokens > MAX_TOKENS || width < 1) return RB_ERR_SHAPE;
    if (cos && (table_rows < 1 || rotary < 8 || rotary % 8 != 0 || rotary > C->dim)) return RB_ERR_SHAPE;
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out | (uintptr_t)cos | (uintptr_t)sin) & 15) return RB_ERR_ALIGN;
    if (((uintptr_t)first | (uintptr_t)lengths | (uintptr_t)table) & 3) return RB_ERR_ALIGN;
    Append8Args A = {};
    A.c = cache8_args(C, first, lengths, table, width, n_seqs, tokens);
    A.q = side(q, H->q_token, H->q_head), A.k_from = side(k, H->k_token, H->k_head), A.v_from = side(v, H->v_token, H->v_head);
    A.q_to = rb::address_of(q_out), A.cos = rb::address_of(cos), A.sin = rb::address_of(sin);
    A.heads = q ? H->heads : 0, A.rotary = cos ? rotary : 0, A.table_rows = table_rows;
    while (8 << A.lanes_shift < C->dim) ++A.lanes_shift;
    const long long query_units = (((long long)((A.heads + QUERIES - 1) / QUERIES) << A.lanes_shift) + 63) / 64 * 64;
    A.query_units = (int)query_units;
    A.blocks = (int)((query_units + ((long long)2 * C->kv_heads << A.lanes_shift) + 255) / 256);
    const long long n = (long long)tokens * A.blocks;
    if (n > 0x7fffffffll) return RB_ERR_SHAPE;
    const dim3 grid = workgroups(n), threads(256);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (H->dtype == RB_F16) {
        if (interleaved)
            hipLaunchKernelGGL((append8_kernel<F16, true>), grid, threads, 0, st, A);
        else
            hipLaunchKernelGGL((append8_kernel<F16, false>), grid, threads, 0, st, A);
    } else {
        if (interleaved)
            hipLaunchKernelGGL((append8_kernel<BF16, true>), grid, threads, 0, st, A);
        else
            hipLaunchKernelGGL((append8_kernel<BF16, false>), grid, threads, 0, st, A);
    }
    return hipGetLastError() == hipSuccess ? RB_OK : RB_ERR_HIP;
}

extern "C" int rb_cache8_read(const rb_cache8 *C, const int32_t *first, const int32_t *lengths, const int32_t *table, int width, int n_seqs, int tokens, void *k, void *v,
                              void *stream)
{
    const int rc = check_cache8(C);
    if (rc != RB_OK) return rc;
    if (!first || !lengths || !table || !k || !v) return RB_ERR_NULL;
    if (n_seqs < 1 || n_seqs > MAX_SEQS || tokens < 1 || tokens > MAX_TOKENS || width < 1) return RB_ERR_SHAPE;
    if (((uintptr_t)k | (uintptr_t)v) & 15) return RB_ERR_ALIGN;
    if (((uintptr_t)first | (uintptr_t)lengths | (uintptr_t)table) & 3) return RB_ERR_ALIGN;
    const Cache8Args A = cache8_args(C, first, lengths, table, width, n_seqs, tokens);
    const int waves = (int)(((long long)C->kv_heads * (C->dim / 16) + 63) / 64);
    const long long n = ((long long)tokens * waves + 3) / 4;
    if (n > 0x1fffffffll) return RB_ERR_SHAPE;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (C->dtype == RB_F16)
        hipLaunchKernelGGL((read8_kernel<F16>), workgroups(n), dim3(256), 0, st, A, rb::address_of(k), rb::address_of(v), waves);
    else
        hipLaunchKernelGGL((read8_kernel<BF16>), workgroups(n), dim3(256), 0, st, A, rb::address_of(k), rb::address_of(v), waves);
    return hipGetLastError() == hipSuccess ? RB_OK : RB_ERR_HIP;
}
