// Attention of few new tokens per sequence over a paged cache (a decoding batch, drafts to verify): the time is that of reading the cache once.
//
// A job is up to 32 rows (tokens times the heads of a group) of one sequence and key head; its work is a row of tiles of 32 keys.  The tiles of
// all jobs of a key head, one after the other, are cut into equal shares, one per wavefront, wherever that falls: contexts of any mix of lengths load every
// compute unit alike.  A wavefront keeps two tiles of keys and values on their way into LDS of its own, across jobs, and meets nobody.  What it has
// of a job that it does not have all of goes to the workspace, unnormalised, and a second launch joins the parts in a fixed order.
//
// Bound: bytes, where there are enough of them (48 sequences of 250000 positions in all, 64 query and 8 key heads of 128, bf16: 180 to 184 us and 6 for the join, 5.6 to 5.7 TB/s;
// six sequences of 3 to 5 drafts on 8500 positions, 40 heads: 35 and 5); else a chain of latencies, the arrays, the table, the keys, their scores, and a launch
// for the join (one token on 2000 positions, 32 heads, fp16: 11 and 5 us).
#include <hip/hip_runtime.h>
#include <algorithm>

#include "rabit.h"
#include "rb_attn.h"
#include "rb_attn_host.h"
#include "rb_attn_shares.h"

namespace rb {
namespace attn {
namespace {

using few::Cursor, few::KEYS, few::ROWS, few::Shape, few::Shares;
constexpr int WAVES = 4;

// the part that share w has of a job of which it does not have all: its first job (0) or its last (1)
template <int D> __device__ __forceinline__ PartOfRows<D, ROWS> part_of(Address workspace, int kvh, int wavefronts, int w, int which)
{
    return PartOfRows<D, ROWS>(workspace, ((size_t)kvh * wavefronts + w) * 2 + which);
}

template <class T, int D>
__global__ __launch_bounds__(64 * WAVES, 1) void few_kernel(const Args A)
{
    using L = Tile<D>;
    __shared__ __attribute__((aligned(16))) uint8_t keys_a[WAVES * L::bytes(KEYS)], values_a[WAVES * L::bytes(KEYS)], keys_b[WAVES * L::bytes(KEYS)], values_b[WAVES * L::bytes(KEYS)];
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kvh = blockIdx.x % A.kv_heads, wavefronts = (int)(gridDim.x / A.kv_heads) * WAVES, w = (int)(blockIdx.x / A.kv_heads) * WAVES + wave;
    const int *first = global_at<const int>(A.first_q), *lengths = global_at<const int>(A.first_k);
    typedef const __attribute__((address_space(4))) int *Uniform;
    const Uniform table_u = (Uniform)global_at<const int>(A.table);
    const Sums<Shape> sums_of(A, first, lengths, lane);
    const Shares shares(sums_of.before(A.n_seqs), wavefronts);
    if (w >= shares.n) return;
    int begin = shares.start(w);
    const int n = shares.start(w + 1) - begin;
    if (n <= 0) return;

    auto entries = [&](int s, int &q0, int &q1, int &length) RB_INLINE { sums_of.entries(s, q0, q1, length); };
    Cursor at = {}, ahead = {};      // the tile at hand, and the next to be asked for
    at.s = __builtin_amdgcn_readfirstlane(sums_of.locate(begin));
    if (!at.stand(A, begin, entries)) return;
    at.block = __builtin_amdgcn_readfirstlane(at.block), at.t = __builtin_amdgcn_readfirstlane(at.t);
    ahead = at;

    constexpr int LOADS = Part<D, KEYS, 1>::LOADS;
    const Part<D, KEYS, 1> part(A.k.token, A.dim, 0, lane);
    const uint8_t *k_base = global_at<const uint8_t>(A.k.at) + kvh * A.k.head, *v_base = global_at<const uint8_t>(A.v.at) + kvh * A.v.head;
    auto place = [&](int page, int r) RB_INLINE { return min(max(page, 0), A.pages - 1) * A.page + (r & ((1 << A.page_shift) - 1)) * A.k.token; };
    int pages[4] = {};      // of the tile to be asked for next
    auto ask_pages = [&](const Cursor &c) RB_INLINE {
        const Uniform row = table_u + (long long)min(c.s, A.n_seqs - 1) * A.width;
        if (A.page_shift >= 5) {
            pages[0] = row[min((c.t * KEYS) >> A.page_shift, A.width - 1)];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) pages[i] = row[min((c.t * KEYS + i * 8) >> A.page_shift, A.width - 1)];
        }
    };
    // tile number i of the share, which `ahead` stands at; past the share's end loads count, but fetch nothing
    auto load = [&](int i, const uint8_t *base, uint8_t *tile) RB_INLINE {
        const int r = ahead.t * KEYS, len = i < n ? ahead.n_k - r : 0;
        if (A.page_shift >= 5) {
            part.template load<0, LOADS>(rows_buffer(base + place(pages[0], r), A.k.token, len, KEYS, A.dim), tile, 0);
        } else {
            constexpr int P = LOADS / 4;      // a load's offsets count from the tile's first row
            part.template load<0, P>(rows_buffer(base + place(pages[0], r), A.k.token, len, 8, A.dim), tile, 0);
            part.template load<P, P>(rows_buffer(base + place(pages[1], r + 8) - 8 * A.k.token, A.k.token, len, 16, A.dim), tile, 0);
            part.template load<2 * P, P>(rows_buffer(base + place(pages[2], r + 16) - 16 * A.k.token, A.k.token, len, 24, A.dim), tile, 0);
            part.template load<3 * P, P>(rows_buffer(base + place(pages[3], r + 24) - 24 * A.k.token, A.k.token, len, 32, A.dim), tile, 0);
        }
    };
    auto next_ahead = [&]() RB_INLINE {
        ahead.advance(A, entries);
        ask_pages(ahead);
    };

    const Rows<D> rows(lane);
    const Columns<D> columns(lane);
    constexpr int B = D / 32;
    v4u q[D / 16];
    v16f sums[B];
    float top, total;
    int limit, least, from_t, token, head;
    bool real, found;
    auto start = [&]() RB_INLINE {
        const int n_q = at.shape.rows / A.group, row0 = at.block * ROWS;
        const int row = min(row0 + (lane & 31), at.shape.rows - 1);
        real = row0 + (lane & 31) < at.shape.rows;
        token = at.q0 + row / A.group;
        head = kvh * A.group + row % A.group;
        limit = at.n_k - n_q + row / A.group;
        least = at.n_k - n_q + row0 / A.group;
        from_t = at.t;
        const uint8_t *from = global_at<const uint8_t>(A.q.at) + token * A.q.token + head * A.q.head;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) q[k] = k * 16 + h * 8 < A.dim ? *(const v4u *)(from + k * 32 + h * 16) : (v4u)(0u);
#pragma unroll
        for (int b = 0; b < B; ++b) sums[b] = (v16f)(0.f);
        top = RB_NEG_INF;
        total = 0.f;
        found = false;
    };
    // Waited for once a job: where the rows are used, the compiler would wait for all loads at every tile
    auto rows_arrived = [&]() RB_INLINE {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) asm volatile("" : "+v"(q[k]));
    };
    bool first_job = true;
    auto finish = [&]() RB_INLINE {      // with tile at.t
        if (found)
            for (int r = max(max(least + 1, 0) / KEYS, from_t) * KEYS; r < min((at.t + 1) * KEYS, at.n_k); ++r) {
                const int page = table_u[(long long)at.s * A.width + (r >> A.page_shift)];
                add_not_finite<T, D>(sums, v_base + place(page, r), A.dim, h, r <= limit);
            }
        total = over_halves_sum(total);
        if (from_t == 0 && at.t == at.shape.tiles - 1) {
            const bool empty = limit < 0;
            store_columns<T, D>(sums, empty ? 0.f : 1.f / total, global_at<uint8_t>(A.o) + ((long long)token * A.heads + head) * (A.dim * 2), A.dim, h, real, empty);
        } else if (real) {
            part_of<D>(A.parts, kvh, wavefronts, w, first_job ? 0 : 1).store(sums, top, total, lane & 31, h);
        }
        first_job = false;
    };

    auto step = [&](int i, uint8_t *keys, uint8_t *values) RB_INLINE {
        if (i > 0 && at.t == 0) {
            start();
            rows_arrived();
        }
        loads_arrived<3 * LOADS>();
        v16f x = {};
        stream_operands<D / 16, 4>([&](int k) RB_INLINE { return rows.read(keys, 0, k); }, [&](int k, v4u a) RB_INLINE { x = T::mfma(a, q[k], x); });
        load(i + 2, k_base, keys);
        const int first_key = at.t * KEYS;
        if (first_key + KEYS - 1 > least) {
            const int seen = limit - first_key - 4 * h;
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (8 * (e / 4) + e % 4 > seen) x[e] = RB_NEG_INF;
        }
        float most = x[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) most = fmaxf(most, x[e]);
        most = over_halves_max(most) * A.c;
        if (__ballot(most > top + SLACK)) {
            const float now = fmaxf(top, most), shrink = now == RB_NEG_INF ? 1.f : __builtin_amdgcn_exp2f(top - now);
            top = now;
            total *= shrink;
#pragma unroll
            for (int b = 0; b < B; ++b) sums[b] *= shrink;
        }
        const float zero_at = (top == RB_NEG_INF ? 0.f : top) - T::BIAS;
        // Each weight in two parts of 16 bits, what the first leaves out being the second: as good as 32 bits, since a row of few keys has few weights for roundings to average out over
        // (one token on 2000 positions: error 1.5 times that of 32-bit weights without, the same with), and the matrix units have time (15.4 and 15.7 us).
        uint32_t wt[8], rest[8];
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const float a = __builtin_amdgcn_exp2f(fmaf(x[e], A.c, -zero_at)), z = __builtin_amdgcn_exp2f(fmaf(x[e + 1], A.c, -zero_at));
            total += a + z;
            wt[e / 2] = T::pack(a, z);
            rest[e / 2] = T::pack(a - T::widen(wt[e / 2] & 0xffffu), z - T::widen(wt[e / 2] >> 16));
        }
        const v4u p[2] = {{wt[0], wt[1], wt[2], wt[3]}, {wt[4], wt[5], wt[6], wt[7]}}, p_rest[2] = {{rest[0], rest[1], rest[2], rest[3]}, {rest[4], rest[5], rest[6], rest[7]}};
        loads_arrived<3 * LOADS>();
        if (least < min(first_key + KEYS, at.n_k) - 1) {      // some row does not see all of the tile's keys: see make_finite
            bool any = false;
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                lds_v4u *v = (lds_v4u *)(lds_byte *)(values + j * L::GROUP + lane * 16);
                const v4u was = *v, is = finite_part<T>(was);
                if (was.x != is.x || was.y != is.y || was.z != is.z || was.w != is.w) {
                    any = true;
                    *v = is;
                }
            }
            found |= __ballot(any) != 0;
        }
        stream_operands<2 * B, 4>([&](int k) RB_INLINE { return columns.read(values, k % B, k / B); }, [&](int k, v4u a) RB_INLINE {
            sums[k % B] = T::mfma(a, p[k / B], sums[k % B]);
            sums[k % B] = T::mfma(a, p_rest[k / B], sums[k % B]);
        });
        load(i + 2, v_base, values);
        next_ahead();
        if (i == n - 1 || at.t == at.shape.tiles - 1) finish();
        at.advance(A, entries);
    };

    uint8_t *const ka = keys_a + wave * L::bytes(KEYS), *const va = values_a + wave * L::bytes(KEYS), *const kb = keys_b + wave * L::bytes(KEYS), *const vb = values_b + wave * L::bytes(KEYS);
    ask_pages(ahead);
    start();
    load(0, k_base, ka);
    load(0, v_base, va);
    next_ahead();
    load(1, k_base, kb);
    load(1, v_base, vb);
    next_ahead();
    rows_arrived();
    for (int i = 0; i < n && at.there(A); i += 2) {      // (past the last sequence only where the arrays are not in order)
        step(i, ka, va);
        if (i + 1 < n && at.there(A)) step(i + 1, kb, vb);
    }
    loads_arrived();
}

// A job that several wavefronts had parts of
template <class T, int D> __global__ __launch_bounds__(256) void join_kernel(const Args A, int wavefronts, int joined)
{
    const int lane = threadIdx.x & 63, kvh = blockIdx.x % A.kv_heads, block = blockIdx.x / A.kv_heads, row0 = blockIdx.y * joined;
    const int *first = global_at<const int>(A.first_q), *lengths = global_at<const int>(A.first_k);
    const Sums<Shape> sums_of(A, first, lengths, lane);
    const int s = __builtin_amdgcn_readfirstlane(sums_of.of_block(block));
    int q0, q1, length;
    sums_of.entries(s, q0, q1, length);
    const Shape shape = Shape::of(A, q0, q1, length);
    const int b = block - block_start(q0, s, A.group, ROWS);
    if (b < 0 || b >= shape.blocks || b * ROWS + row0 >= shape.rows) return;
    const Shares shares(sums_of.before(A.n_seqs), wavefronts);
    const int from = sums_of.before(s) + b * shape.tiles;
    int w0, w1;
    if (!shares.of_job(from, shape.tiles, w0, w1) || w0 == w1) return;      // (one: it has stored the result)
    const bool starts_inside = shares.start(w0) < from;      // the first part is that share's last, all others are their shares' first
    const int n_q = shape.rows / A.group, n_k = positions(length, A.width, A.page_shift);
    q0 = min(max(q0, 0), A.tokens_q);
    auto token = [&](int r) { return (b * ROWS + r) / A.group; };
    join_rows<T, D>(
        joined, w1 - w0 + 1, row0, min(shape.rows - b * ROWS - row0, joined), A.dim,
        [&](int i) { return part_of<D>(A.parts, kvh, wavefronts, w0 + i, i == 0 && starts_inside ? 1 : 0); },
        [&](int r) { return global_at<uint8_t>(A.o) + ((long long)(q0 + token(r)) * A.heads + kvh * A.group + (b * ROWS + r) % A.group) * (A.dim * 2); },
        [&](int r) { return n_k - n_q + token(r) < 0; });
}

// one workgroup per compute unit, shared out over the key heads
int groups_per_head(const Args &A, int compute_units) { return compute_units > A.kv_heads ? compute_units / A.kv_heads : 1; }

template <class T, int D> int launch(const Args &A, int compute_units, hipStream_t stream)
{
    const int groups = groups_per_head(A, compute_units);
    const long long jobs = block_numbers(A.tokens_q, A.n_seqs, A.group, ROWS) * A.kv_heads;
    if (jobs > 0x7fffffffll) return RB_ERR_SHAPE;
    hipLaunchKernelGGL((few_kernel<T, D>), dim3((unsigned)(groups * A.kv_heads)), dim3(64 * WAVES), 0, stream, A);
    const int rows = (int)std::min((long long)ROWS, (long long)A.tokens_q * A.group), joined = rows_joined(jobs, rows);      // rows of one job, at most
    hipLaunchKernelGGL((join_kernel<T, D>), dim3((unsigned)jobs, (rows + joined - 1) / joined), dim3(256), 0, stream, A, groups * WAVES, joined);
    return hipGetLastError() == hipSuccess ? RB_OK : RB_ERR_HIP;
}

}  // namespace

// Up to 32 rows per sequence and key head on average: few_kernel reads a sequence's positions once per 32 rows, rows_kernel once per 128, with more to start and to join.  (fp16, 32 query and
// 8 key heads of 128, calls in us by few_kernel and by rows_kernel: sixteen sequences of 1, 4, 8, 12 and 16 tokens on 2000 31 and 35, 34 and 36, 36.6 and 37.1, 43 and 39, 46 and 41; one of 1, 8 and 16 on
// 8000 18 and 22, 23.3 and 23.0, 28 and 24; 128 tokens on 2000 beside 15, 32, 64 and 256 single ones on 1000 41 and 35, 48 and 56, 65 and 84, 240 and 239.  What an average costs: 512 tokens on 7700 beside
// 64, 128 and 256 single ones 274 and 166, 314 and 260, 388 and 346, of which the last two are few_kernel's by it.  32 key heads, sixteen of 8, 16 and 32 tokens 107 and 112, 113 and 108, 120 and 111.)
bool few_applies(int tokens, int n_seqs, int group, long long positions)
{
    const long long tiles = block_numbers(tokens, n_seqs, group, ROWS) * (std::min(positions, 0x7fffffffll) / KEYS + 1);
    return (long long)tokens * group <= (long long)ROWS * n_seqs && tiles < 0x7fffffffll;
}

size_t few_workspace_bytes(int kv_heads, int dim, int compute_units)
{
    Args A = {};
    A.kv_heads = kv_heads;
    return (size_t)kv_heads * groups_per_head(A, compute_units) * WAVES * 2 * (dim <= 64 ? PartOfRows<64, ROWS>::FLOATS : PartOfRows<128, ROWS>::FLOATS) * 4;
}

int launch_few(const Args &A, int dtype, int compute_units, hipStream_t stream)
{
    if (dtype == RB_F16) return A.dim <= 64 ? launch<F16, 64>(A, compute_units, stream) : launch<F16, 128>(A, compute_units, stream);
    return A.dim <= 64 ? launch<BF16, 64>(A, compute_units, stream) : launch<BF16, 128>(A, compute_units, stream);
}

}  // namespace attn
}  // namespace rb
