// Attention over packed prompts and over a paged cache: o_i = sum_j p_ij v_j with
// p_ij = exp(c q_i . k_j - lse_i), lse_i = log sum_j exp(c q_i . k_j) over the keys j that row i sees.
#include <hip/hip_runtime.h>
#include <algorithm>

#include "rabit.h"
#include "rb_attn.h"
#include "rb_attn8.h"
#include "rb_attn_host.h"
#include "rb_internal.h"

namespace rb {
namespace attn {
namespace {

constexpr int BM = 128, KEYS = 64;

// A cache is shared out to workgroups by what the lengths ask for: a block of rows has as many, each with a part of the keys, as it takes for none to have more than some number
// of tiles.  That is the smallest of some numbers, from the tiles per workgroup wanted up to twice those, for which no more workgroups start than run at once, and where the blocks
// are too many for any, or the sequences too many to try, the first: workgroups then take turns.  (fp16, against the same number of parts for every block: 700, 64, 33 and 200 new tokens
// on 100, 4000, 9000 and 2000, 64 query and 8 key heads of 128, 181 -> 82 us; 128 tokens on 30000, 8 heads, 53 -> 39; 512 tokens on 7500, 32 and 8 heads, where all parts are alike,
// 85 -> 88.  Sharing the tiles out exactly, workgroups going on from one block to the next, took 121, 40 and 98: every start of a block costs some 4 us.)
constexpr float LEAST = 8.f;               // tiles of a part (512 new tokens: 23 us, with 4 26)
constexpr long long GROUPS = 2, MANY = 4;  // workgroups per compute unit: wanted, and those of whole blocks that need no sharing
constexpr long long JOINING = 2048;        // workgroups that join: all at once (8192, most of which find no work, 10 us more)
struct Blocks {
    static constexpr int JOB = BM;
    int blocks, tiles, parts;      // (tiles of a block on average)
    static __device__ __forceinline__ Blocks of(const Args &A, int q0, int q1, int length)
    {
        q0 = min(max(q0, 0), A.tokens_q);
        q1 = min(max(q1, q0), A.tokens_q);
        const int n_q = q1 - q0, n_k = positions(length, A.width, A.page_shift);
        const int first = max((n_k - n_q) / KEYS, 0) + 1, last = n_k / KEYS + 1, tiles = first + (last - first) / 2;
        return {(n_q * A.group + BM - 1) / BM, tiles, max((int)(tiles * A.per_tile + 0.98f), 1)};
    }
};
struct Groups : Blocks {
    __device__ __forceinline__ Groups(const Blocks &b) : Blocks(b) {}
    __device__ __forceinline__ int count() const { return blocks * parts; }
    static __device__ __forceinline__ Groups of(const Args &A, int q0, int q1, int length) { return Blocks::of(A, q0, q1, length); }
};
struct Tiles : Blocks {
    __device__ __forceinline__ Tiles(const Blocks &b) : Blocks(b) {}
    __device__ __forceinline__ int count() const { return blocks * tiles; }
    static __device__ __forceinline__ Tiles of(const Args &A, int q0, int q1, int length) { return Blocks::of(A, q0, q1, length); }
};
struct Slots : Blocks {      // of the workspace: one for each workgroup that has a part
    __device__ __forceinline__ Slots(const Blocks &b) : Blocks(b) {}
    __device__ __forceinline__ int count() const { return parts > 1 ? blocks * parts : 0; }
    static __device__ __forceinline__ Slots of(const Args &A, int q0, int q1, int length) { return Blocks::of(A, q0, q1, length); }
};
__device__ __forceinline__ Args with_shares(Args A, const Sums<Tiles> &tiles)
{
    const float share = max(tiles.before(A.n_seqs) / (float)A.wanted, LEAST);
    float times = 1.f;
    if (A.n_seqs <= 32) {      // each group of lanes tries another number
        const int pad = A.n_seqs > 1 ? padded(A.n_seqs) : 1, s = tiles.lane & (pad - 1);
        const int q0 = __shfl(tiles.q0, s), q1 = __shfl(tiles.q1, s), length = __shfl(tiles.length, s);
        const float mine = 1.f + (float)(tiles.lane / pad) * pad / 64.f;
        A.per_tile = 1.f / (share * mine);
        int groups = s < A.n_seqs ? Groups::of(A, q0, q1, length).count() : 0;
        for (int d = 1; d < pad; d <<= 1) groups += __shfl_xor(groups, d);
        const unsigned long long fits = __ballot(groups <= A.wanted);
        if (fits) times = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), __builtin_ctzll(fits)));
    }
    A.per_tile = 1.f / (share * times);
    return A;
}

// One workgroup does 128 rows of one key head, 32 per wavefront, over all keys that they see, KEYS at a time; the next tile of keys and values
// is on its way into LDS while one is used.  Bound: matrix and vector instructions, which two wavefronts per SIMD overlap in part (one long
// prompt of 8192 tokens, 64 query and 8 key heads of 128, causal, bf16: 1.00 to 1.14 ms, 0.97 to 1.10 PFLOP/s, by the card and by how long it has been at work).  What was tried beside it: 32 keys at a time and
// three wavefronts per SIMD, the same on long prompts and a fifth slower on short ones; a pipeline within a wavefront, scores of one half of a tile
// beside the weights of the other, 1.08 ms; eight wavefronts and three tiles ahead, 1.09 ms; operand reads left to the compiler, 1.11 ms.
//
// HALVES = 2: eight wavefronts, four of them with the first 32 keys of every tile and four with the second, joined at the end.  For calls of no more workgroups than compute units, and
// of one sequence up to twice as many: a step takes less time where a workgroup has a compute unit to itself, and the longest blocks of one long sequence decide its time (fp16, causal,
// heads of 128: 64 tokens of 8 heads 12.4 -> 9.9 us, 512 of 32 16.3 -> 15.3, 1200 of 32 and 8 28.6 -> 25.3, 8192 of one head 141 -> 111, 6000 of 8 116 -> 96; heads of 64 3 to 10 %).
// Beyond, two workgroups fill a compute unit as well as one of twice the size, without the join (2600 tokens of 32 and 8 heads, 656 workgroups, 67 and 78 us; eight sequences of 1000
// tokens in all, 312 workgroups, 11.5 and 16.8).
//
// Of a cache in 8 bits, elements come into registers, are widened to T in their units there, and stored into the tile that the rest of the kernel knows (512 and seven new tokens on 21513 positions,
// 32 and 8 heads: 115 us and 14 for the join; of 16 bits, where tiles go into LDS past the registers, 90 to 100 and 14).
enum From { PACKED, PAGES, PAGES8 };      // where keys and values are: packed, in a cache, in a cache in 8 bits
template <class T, int D, From FROM, int HALVES>
__global__ __launch_bounds__(256 * HALVES, 2) void rows_kernel(const Args A)
{
    using L = Tile<D>;
    constexpr int WAVES = 4 * HALVES;
    constexpr bool PAGED = FROM != PACKED, IN8 = FROM == PAGES8;
    // tiles as variables of their own: the compiler then knows that loads into one do not concern reads of another
    __shared__ __attribute__((aligned(16))) uint8_t keys_a[L::bytes(KEYS)], values_a[L::bytes(KEYS)], keys_b[L::bytes(KEYS)], values_b[L::bytes(KEYS)];
    __shared__ int found;
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), quarter = wave & 3, half = wave >> 2;
    const int kvh = blockIdx.x % A.kv_heads, number = blockIdx.x / A.kv_heads, numbers = (int)gridDim.x / A.kv_heads;      // the workgroups of a head go to the same XCDs
    const int *first_q = global_at<const int>(A.first_q), *first_k = global_at<const int>(A.first_k);
    int s, of_sequence, split = 0, splits = 1;
    [[maybe_unused]] int slot = 0;      // of this workgroup's part
    if constexpr (!PAGED) {
        if (!rows_of_workgroup<BM>(first_q, first_k, A.n_seqs, A.ordered, A.tokens_q, A.tokens_k, A.group, A.causal, number, numbers, lane, s, of_sequence)) return;
    } else if (!A.wanted) {
        const int block = numbers - 1 - number;      // the longest first
        s = sequence_of_block(first_q, A.n_seqs, A.group, BM, block, lane);
        of_sequence = block - block_start(first_q[s], s, A.group, BM);
    } else {
        const Sums<Tiles> tiles_of(A, first_q, first_k, lane);
        const Args B = with_shares(A, tiles_of);
        const Sums<Groups> groups(B, tiles_of);
        int at = groups.before(A.n_seqs) - 1 - number;
        if (at < 0) return;
        s = __builtin_amdgcn_readfirstlane(groups.locate(at));
        if (s >= A.n_seqs) return;
        int q0, q1, length;
        groups.entries(s, q0, q1, length);
        splits = __builtin_amdgcn_readfirstlane(Blocks::of(B, q0, q1, length).parts);
        of_sequence = __builtin_amdgcn_readfirstlane((int)((unsigned)at / (unsigned)splits));
        split = __builtin_amdgcn_readfirstlane((int)((unsigned)at % (unsigned)splits));
        if (splits > 1) {
            slot = Sums<Slots>(B, tiles_of).before(s) + at;
            if (slot < 0 || slot >= 2 * A.wanted) return;      // (arrays that are not in order)
        }
    }
    Sequence S = sequence_at(first_q, PAGED ? first_q : first_k, s, A.tokens_q, PAGED ? A.tokens_q : A.tokens_k);
    if (PAGED) {
        S.k0 = 0;
        S.n_k = positions(__builtin_amdgcn_readfirstlane(first_k[s]), A.width, A.page_shift);
    }
    const int row0 = of_sequence * BM, n_rows = S.n_q * A.group;
    if (row0 < 0 || row0 >= n_rows) return;

    const int my_row = row0 + quarter * 32 + (lane & 31);
    const bool real = my_row < n_rows;
    const int row = min(my_row, n_rows - 1), token = row / A.group, head = kvh * A.group + row % A.group;
    // the last key that a row sees; -1 or less: none
    const int ahead = S.n_k - S.n_q;
    auto last_key = [&](int r) { return A.causal ? min(ahead + min(r, n_rows - 1) / A.group, S.n_k - 1) : S.n_k - 1; };
    const int limit = A.causal ? ahead + token : S.n_k - 1;
    const int block_least = last_key(row0), block_most = last_key(row0 + BM - 1);
    const int wave_least = __builtin_amdgcn_readfirstlane(last_key(row0 + quarter * 32)), wave_most = __builtin_amdgcn_readfirstlane(last_key(row0 + quarter * 32 + 31));
    const int tiles = __builtin_amdgcn_readfirstlane(max(block_most + 1, 0) + KEYS - 1) / KEYS, parts = PAGED ? splits_of(tiles, splits) : 1;
    if (split >= parts) return;
    const int first_tile = tiles * split / parts, n_tiles = tiles * (split + 1) / parts;      // (the end of this workgroup's)

    v4u q[D / 16];
    {
        const uint8_t *from = global_at<const uint8_t>(A.q.at) + (S.q0 + token) * A.q.token + head * A.q.head;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) q[k] = k * 16 + h * 8 < A.dim ? *(const v4u *)(from + k * 32 + h * 16) : (v4u)(0u);
    }

    // rows of a page are counted from the first that the wavefront needs, others from the tile's
    constexpr int MINE = KEYS / WAVES, LOADS = Part<D, KEYS, WAVES>::LOADS;
    const Part<D, KEYS, WAVES> k_part(A.k.token, A.dim, PAGED ? 0 : wave * MINE, lane), v_part(A.v.token, A.dim, PAGED ? 0 : wave * MINE, lane);
    const uint8_t *k_base = global_at<const uint8_t>(A.k.at) + S.k0 * A.k.token + kvh * A.k.head;
    const uint8_t *v_base = global_at<const uint8_t>(A.v.at) + S.k0 * A.v.token + kvh * A.v.head;
    const int *table = PAGED ? global_at<const int>(A.table) + (long long)s * A.width : nullptr;
    auto place = [&](int page, int r) RB_INLINE {      // of row r, behind the first page
        return min(max(page, 0), A.pages - 1) * A.page + (r & ((1 << A.page_shift) - 1)) * A.k.token;
    };
    // A wavefront's part of a tile lies in one page, or, 16 rows in pages of eight, in two.  Pages are asked for one step before the rows are.
    constexpr int PARTS = MINE / 8, PART_LOADS = LOADS / PARTS;
    const __attribute__((address_space(4))) int *pages_at = (const __attribute__((address_space(4))) int *)table;
    int pages[PARTS] = {};
    auto ask_pages = [&](int t) RB_INLINE {
#pragma unroll
        for (int i = 0; i < PARTS; ++i) pages[i] = pages_at[min((t * KEYS + wave * MINE + i * 8) >> A.page_shift, A.width - 1)];
    };
    auto load_one = [&](int t, const uint8_t *base, long long stride, const Part<D, KEYS, WAVES> &part, uint8_t *tile) RB_INLINE {
        if constexpr (!PAGED) {
            part.template load<0, LOADS>(rows_buffer(base + (long long)t * KEYS * stride, stride, S.n_k - t * KEYS, KEYS, A.dim), tile, wave);
        } else {
            const int r = t * KEYS + wave * MINE;
            part.template load<0, PART_LOADS>(rows_buffer(base + place(pages[0], r), stride, S.n_k - r, 8, A.dim), tile, wave);
            if constexpr (PARTS == 2)      // (its offsets are eight rows on)
                part.template load<PART_LOADS, PART_LOADS>(rows_buffer(base + place(pages[1], r + 8) - 8 * stride, stride, S.n_k - r, 16, A.dim), tile, wave);
        }
    };
    // of 8 bits, by way of registers
    const uint32_t at8 = Rows8<D, MINE>::at(A.k.token, A.dim, lane);
    auto exponents_at = [&](Address exponents, int page, int r) RB_INLINE {
        return global_at<const uint8_t>(exponents) + (((long long)min(max(page, 0), A.pages - 1) * A.kv_heads + kvh) << A.page_shift) + (r & ((1 << A.page_shift) - 1));
    };
    [[maybe_unused]] Rows8<D, MINE> raw_k, raw_v;
    [[maybe_unused]] auto load8 = [&](int t) RB_INLINE {
        const int r = t * KEYS + wave * MINE;
#pragma unroll
        for (int i = 0; i < PARTS; ++i) raw_k.load(i, k_base + place(pages[i], r + i * 8), exponents_at(A.k_exp, pages[i], r + i * 8), A.k.token, S.n_k - r - i * 8, A.dim, at8, lane);
#pragma unroll
        for (int i = 0; i < PARTS; ++i) raw_v.load(i, v_base + place(pages[i], r + i * 8), exponents_at(A.v_exp, pages[i], r + i * 8), A.v.token, S.n_k - r - i * 8, A.dim, at8, lane);
        ask_pages(t + 1);
    };
    auto write8 = [&](uint8_t *keys, uint8_t *values) RB_INLINE {
        raw_k.template write<T>(keys, wave * MINE, lane);
        raw_v.template write<T>(values, wave * MINE, lane);
    };
    auto load = [&](int t, uint8_t *keys, uint8_t *values) RB_INLINE {
        load_one(t, k_base, A.k.token, k_part, keys);
        load_one(t, v_base, A.v.token, v_part, values);
        if constexpr (PAGED) ask_pages(t + 1);
    };

    // A tile's rows past the sequence's end are zeros, but where one value stands for all (a stride of zero) they are that value again, which no row sees
    const int rows_end = !PAGED && A.v.token < A.dim * 2 ? 0x7fffffff : S.n_k;
    const Rows<D> rows(lane);
    const Columns<D> columns(lane);
    constexpr int B = D / 32, H = KEYS / 32 / HALVES;      // 32s of elements, and of keys of a tile
    v16f sums[B] = {};
    float top = RB_NEG_INF, total = 0.f;
    auto step = [&](int t, uint8_t *keys, uint8_t *values, uint8_t *next_keys, uint8_t *next_values) RB_INLINE {
        if constexpr (IN8) {
            meet();
            if (t + 1 < n_tiles) write8(next_keys, next_values);
            if (t + 2 < n_tiles) load8(t + 2);
        } else {
            loads_arrived();
            __syncthreads();      // tile t is there, everybody has done with tile t - 1
            if (t + 1 < n_tiles) load(t + 1, next_keys, next_values);
        }
        if (block_least < min(t * KEYS + KEYS, rows_end) - 1) {      // some row of the workgroup does not see all of the tile's keys
            make_finite<T, D, KEYS, WAVES>(values, &found, tid);
            __syncthreads();
        }
        const int first_key = t * KEYS + half * 32;
        if (first_key > wave_most) return;
        v16f x[H] = {};
        stream_operands<H * D / 16, 6>([&](int i) RB_INLINE { return rows.read(keys, half * H + i % H, i / H); }, [&](int i, v4u a) RB_INLINE { x[i % H] = T::mfma(a, q[i / H], x[i % H]); });
        if (first_key + 32 * H - 1 > wave_least) {
            const int seen = limit - first_key - 4 * h;
#pragma unroll
            for (int b = 0; b < H; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (b * 32 + 8 * (i / 4) + i % 4 > seen) x[b][i] = RB_NEG_INF;
        }
        float most = x[0][0];
#pragma unroll
        for (int i = 1; i < 16 * H; ++i) most = fmaxf(most, x[i / 16][i % 16]);
        most = over_halves_max(most) * A.c;
        if (__ballot(most > top + SLACK)) {
            const float now = fmaxf(top, most);
            const float shrink = now == RB_NEG_INF ? 1.f : __builtin_amdgcn_exp2f(top - now);
            top = now;
            total *= shrink;
#pragma unroll
            for (int b = 0; b < B; ++b) sums[b] *= shrink;
        }
        const float zero_at = (top == RB_NEG_INF ? 0.f : top) - T::BIAS;
        v4u p[2 * H];
#pragma unroll
        for (int b = 0; b < H; ++b) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float a = __builtin_amdgcn_exp2f(fmaf(x[b][i], A.c, -zero_at)), z = __builtin_amdgcn_exp2f(fmaf(x[b][i + 1], A.c, -zero_at));
                total += a + z;
                w[i / 2] = T::pack(a, z);
            }
            p[2 * b] = (v4u){w[0], w[1], w[2], w[3]};
            p[2 * b + 1] = (v4u){w[4], w[5], w[6], w[7]};
        }
        stream_operands<2 * H * B, 4>([&](int i) RB_INLINE { return columns.read(values, i % B, 2 * half * H + i / B); }, [&](int i, v4u a) RB_INLINE { sums[i % B] = T::mfma(a, p[i / B], sums[i % B]); });
    };
    if (tid == 0) found = 0;
    if (first_tile < n_tiles) {
        if constexpr (PAGED) ask_pages(first_tile);
        if constexpr (IN8) {
            load8(first_tile);
            write8(keys_a, values_a);
            load8(first_tile + 1);
        } else {
            load(first_tile, keys_a, values_a);
        }
    }
    for (int t = first_tile; t < n_tiles; t += 2) {
        step(t, keys_a, values_a, keys_b, values_b);
        if (t + 1 < n_tiles) step(t + 1, keys_b, values_b, keys_a, values_a);
    }

    __syncthreads();
    if constexpr (HALVES == 2) {      // the second half's sums to the first, in units of the larger maximum
        __shared__ float tops[BM], totals[BM];
        static_assert(B * 4096 <= L::bytes(KEYS), "sums of 32 rows");
        uint8_t *const by = quarter == 0 ? keys_a : quarter == 1 ? keys_b : quarter == 2 ? values_a : values_b;
        const int r = quarter * 32 + (lane & 31);
        total = over_halves_sum(total);
        if (half == 1) {
            if (h == 0) tops[r] = top, totals[r] = total;
#pragma unroll
            for (int b = 0; b < B; ++b)
#pragma unroll
                for (int i = 0; i < 16; i += 4) *(v4f *)(by + (b * 4 + i / 4) * 1024 + lane * 16) = (v4f){sums[b][i], sums[b][i + 1], sums[b][i + 2], sums[b][i + 3]};
        }
        __syncthreads();
        if (half == 1) return;
        const float now = fmaxf(top, tops[r]), mine = now == RB_NEG_INF ? 1.f : __builtin_amdgcn_exp2f(top - now), theirs = now == RB_NEG_INF ? 1.f : __builtin_amdgcn_exp2f(tops[r] - now);
        top = now;
        total = 0.5f * (total * mine + totals[r] * theirs);      // (both halves of the wavefront have all of it, and are added below)
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) sums[b][i] = sums[b][i] * mine + ((const v4f *)(by + (b * 4 + i / 4) * 1024 + lane * 16))[0][i % 4] * theirs;
    }
    if (__builtin_amdgcn_readfirstlane(found)) {
        for (int r = max(max(block_least + 1, 0) / KEYS, first_tile) * KEYS; r <= min(wave_most, n_tiles * KEYS - 1); ++r) {
            if constexpr (IN8) {
                const int page = __builtin_amdgcn_readfirstlane(table[r >> A.page_shift]);
                add_not_finite8<T, D>(sums, v_base + place(page, r), *exponents_at(A.v_exp, page, r), A.dim, h, r <= limit);
            } else {
                add_not_finite<T, D>(sums, v_base + (PAGED ? place(__builtin_amdgcn_readfirstlane(table[r >> A.page_shift]), r) : r * A.v.token), A.dim, h, r <= limit);
            }
        }
    }

    total = over_halves_sum(total);
    const bool empty = limit < 0;
    if (parts > 1) {
        if (real) PartOfRows<D, BM>(A.parts, (size_t)slot * A.kv_heads + kvh).store(sums, top, total, quarter * 32 + (lane & 31), h);
        return;
    }
    if (A.lse && real && h == 0)
        global_at<float>(A.lse)[(long long)(S.q0 + token) * A.heads + head] = empty ? RB_NEG_INF : (top - T::BIAS + __builtin_amdgcn_logf(total)) * LN2;
    uint8_t *to = global_at<uint8_t>(A.o) + ((long long)(S.q0 + token) * A.heads + head) * (A.dim * 2);
    store_columns<T, D>(sums, empty ? 0.f : 1.f / total, to, A.dim, h, real, empty);
}

// What several workgroups had parts of
template <class T, int D> __global__ __launch_bounds__(256) void join_kernel(const Args A, int joined)
{
    const int lane = threadIdx.x & 63, kvh = blockIdx.x % A.kv_heads, block = blockIdx.x / A.kv_heads;
    const int *first = global_at<const int>(A.first_q), *lengths = global_at<const int>(A.first_k);
    const Sums<Tiles> tiles_of(A, first, lengths, lane);
    const Args B = with_shares(A, tiles_of);
    const Sums<Slots> slots(B, tiles_of);
    const int s = __builtin_amdgcn_readfirstlane(slots.of_block(block));
    int q0, q1, length;
    slots.entries(s, q0, q1, length);
    const Blocks shape = Blocks::of(B, q0, q1, length);
    const int b = block - block_start(q0, s, A.group, BM);
    if (b < 0 || b >= shape.blocks || shape.parts == 1) return;
    q0 = min(max(q0, 0), A.tokens_q);
    const int n_q = min(max(q1, q0), A.tokens_q) - q0, before = b * BM, n_rows = n_q * A.group - before, ahead = positions(length, A.width, A.page_shift) - n_q;
    const int most = ahead + (before + min(n_rows, BM) - 1) / A.group, parts = splits_of((max(most + 1, 0) + KEYS - 1) / KEYS, shape.parts);
    if (parts == 1) return;
    const int slot = slots.before(s) + b * shape.parts;
    if (slot < 0 || slot > 2 * A.wanted - parts) return;
    for (int row0 = blockIdx.y * joined; row0 < min(n_rows, BM); row0 += gridDim.y * joined) {
        join_rows<T, D>(
            joined, parts, row0, min(n_rows - row0, joined), A.dim, [&](int i) { return PartOfRows<D, BM>(A.parts, (size_t)(slot + i) * A.kv_heads + kvh); },
            [&](int r) { return global_at<uint8_t>(A.o) + ((long long)(q0 + (before + r) / A.group) * A.heads + kvh * A.group + (before + r) % A.group) * (A.dim * 2); },
            [&](int r) { return ahead + (before + r) / A.group < 0; });
        __syncthreads();
    }
}

// Workgroups per key head that the work over a cache is shared out to; 0: one per block of rows, where those are many, or the tiles are not counted in 31 bits
int groups_wanted(int tokens, int n_seqs, int kv_heads, int group, long long most_positions, int compute_units)
{
    const long long blocks = block_numbers(tokens, n_seqs, group, BM);
    if (blocks * kv_heads >= MANY * compute_units || blocks * (most_positions / KEYS + 2) >= 0x7fffffffll) return 0;
    return (int)std::max(GROUPS * compute_units / kv_heads, 1ll);
}
// Blocks of more than one part have at most twice the workgroups wanted: a block that x > 1 would do for has less than x + 1.  (As much for any number of tokens, if for one.)
size_t parts_workspace_bytes(int kv_heads, int group, int dim, int compute_units)
{
    const size_t slots = (size_t)groups_wanted(1, 1, kv_heads, group, 0, compute_units) * 2;
    return slots * kv_heads * (dim <= 64 ? PartOfRows<64, BM>::FLOATS : PartOfRows<128, BM>::FLOATS) * 4;
}

template <class T, int D> int launch_rows(Args A, bool paged, int compute_units, hipStream_t stream)
{
    const long long blocks = block_numbers(A.tokens_q, A.n_seqs, A.group, BM) * A.kv_heads, n = blocks + (long long)A.wanted * A.kv_heads;      // (a block that has a share of x has at most x + 1)
    if (!one_launch(n, 256) || (long long)A.tokens_q * A.group > 0x7fff0000ll) return RB_ERR_SHAPE;
    A.ordered = ordered_for(A.n_seqs, n, 2ll * compute_units);
    const dim3 grid((unsigned)n);
    if (paged) {
        if (A.k_exp)
            hipLaunchKernelGGL((rows_kernel<T, D, PAGES8, 1>), grid, dim3(256), 0, stream, A);
        else
            hipLaunchKernelGGL((rows_kernel<T, D, PAGES, 1>), grid, dim3(256), 0, stream, A);
        const int joined = rows_joined(blocks, BM);
        if (A.wanted) hipLaunchKernelGGL((join_kernel<T, D>), dim3((unsigned)blocks, (unsigned)std::min((long long)BM / joined, std::max(JOINING / blocks, 1ll))), dim3(256), 0, stream, A, joined);
    } else if (n <= (A.n_seqs == 1 ? 2 : 1) * compute_units) {
        hipLaunchKernelGGL((rows_kernel<T, D, PACKED, 2>), grid, dim3(512), 0, stream, A);
    } else {
        hipLaunchKernelGGL((rows_kernel<T, D, PACKED, 1>), grid, dim3(256), 0, stream, A);
    }
    return hipGetLastError() == hipSuccess ? RB_OK : RB_ERR_HIP;
}
int launch(const Args &A, int dtype, bool paged, int compute_units, hipStream_t stream)
{
    if (dtype == RB_F16) return A.dim <= 64 ? launch_rows<F16, 64>(A, paged, compute_units, stream) : launch_rows<F16, 128>(A, paged, compute_units, stream);
    return A.dim <= 64 ? launch_rows<BF16, 64>(A, paged, compute_units, stream) : launch_rows<BF16, 128>(A, paged, compute_units, stream);
}

}  // namespace

int check_heads(const rb_heads *H)
{
    if (!H) return RB_ERR_NULL;
    if (H->heads < 1 || H->kv_heads < 1 || H->heads % H->kv_heads != 0 || H->heads > 65536) return RB_ERR_SHAPE;
    if (H->dim < 8 || H->dim % 8 != 0) return RB_ERR_SHAPE;
    if (H->dim > 128 || (H->dtype != RB_F16 && H->dtype != RB_BF16)) return RB_ERR_UNSUPPORTED;
    for (const long long s : {H->q_token, H->q_head, H->k_token, H->k_head, H->v_token, H->v_head}) {
        if (s < 0 || s > MAX_STRIDE) return RB_ERR_SHAPE;
        if (s % 8 != 0) return RB_ERR_ALIGN;
    }
    return RB_OK;
}

int check_scale(float scale)
{
    return scale > 0.f && scale <= 2e38f ? RB_OK : RB_ERR_VALUE;      // (times log2(e) it is a number still)
}

}  // namespace attn
}  // namespace rb

using namespace rb::attn;

extern "C" int rb_attn_prompt(const rb_heads *H, const void *q, const void *k, const void *v, const int32_t *first_q, const int32_t *first_k, int n_seqs,
                              int tokens_q, int tokens_k, int causal, float scale, void *o, float *lse, void *stream)
{
    const int rc = check_heads(H);
    if (rc != RB_OK) return rc;
    if (!q || (tokens_k != 0 && (!k || !v)) || !first_q || !o) return RB_ERR_NULL;
    if (n_seqs < 1 || n_seqs > MAX_SEQS || tokens_q < 1 || tokens_k < 0 || tokens_q > MAX_TOKENS || tokens_k > MAX_TOKENS || (!first_k && tokens_k != tokens_q)) return RB_ERR_SHAPE;
    if (check_scale(scale) != RB_OK) return RB_ERR_VALUE;
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)o) & 15) return RB_ERR_ALIGN;
    if (((uintptr_t)first_q | (uintptr_t)first_k | (uintptr_t)lse) & 3) return RB_ERR_ALIGN;
    Args A = {};
    A.q = side(q, H->q_token, H->q_head), A.k = side(k, H->k_token, H->k_head), A.v = side(v, H->v_token, H->v_head);
    A.o = rb::address_of(o), A.lse = rb::address_of(lse), A.first_q = rb::address_of(first_q), A.first_k = rb::address_of(first_k ? first_k : first_q);
    A.n_seqs = n_seqs, A.tokens_q = tokens_q, A.tokens_k = tokens_k;
    A.heads = H->heads, A.kv_heads = H->kv_heads, A.group = H->heads / H->kv_heads, A.dim = H->dim, A.causal = causal != 0;
    A.c = scale * LOG2E;
    return launch(A, H->dtype, false, rb::mx::device_groups(), static_cast<hipStream_t>(stream));
}

namespace {

// Calls over a cache: `C` as one of 16 bits, its strides in elements of `size` bytes
size_t paged_workspace_bytes(const rb_cache &C, bool in8, int heads, int n_seqs, int tokens)
{
    if (heads < 1 || heads % C.kv_heads != 0 || n_seqs < 1 || tokens < 1) return 0;
    const int units = rb::mx::device_groups(), group = heads / C.kv_heads;
    // whichever kernel a call of up to so many tokens and sequences and its table's width will choose
    const size_t few = few_applies(1, n_seqs, group, 0) ? (in8 ? few8_workspace_bytes : few_workspace_bytes)(C.kv_heads, C.dim, units) : 0;
    return std::max(few, parts_workspace_bytes(C.kv_heads, group, C.dim, units));
}
int paged(const rb_cache &C, int size, const uint8_t *k_exp, const uint8_t *v_exp, const void *q, long long q_token, long long q_head, int heads, const int32_t *first,
          const int32_t *lengths, const int32_t *table, int width, int n_seqs, int tokens, float scale, void *o, void *workspace, size_t workspace_bytes, void *stream)
{
    const rb_heads H = {heads, C.kv_heads, C.dim, C.dtype, q_token, q_head, C.token_stride, C.head_stride, C.token_stride, C.head_stride};
    const int rc = check_heads(&H);
    if (rc != RB_OK) return rc;
    if (!q || !first || !lengths || !table || !o) return RB_ERR_NULL;
    if (n_seqs < 1 || n_seqs > MAX_SEQS || tokens < 1 || tokens > MAX_TOKENS || width < 1) return RB_ERR_SHAPE;
    if (check_scale(scale) != RB_OK) return RB_ERR_VALUE;
    if (((uintptr_t)q | (uintptr_t)o) & 15) return RB_ERR_ALIGN;
    if (((uintptr_t)first | (uintptr_t)lengths | (uintptr_t)table) & 3) return RB_ERR_ALIGN;
    if (workspace_bytes < paged_workspace_bytes(C, size == 1, heads, n_seqs, tokens) || (workspace_bytes && !workspace)) return RB_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 15) return RB_ERR_ALIGN;
    Args A = {};
    A.q = side(q, q_token, q_head);
    A.k = {rb::address_of(C.k), C.token_stride * size, C.head_stride * size}, A.v = {rb::address_of(C.v), C.token_stride * size, C.head_stride * size};
    A.k_exp = rb::address_of(k_exp), A.v_exp = rb::address_of(v_exp);
    A.o = rb::address_of(o), A.first_q = rb::address_of(first), A.first_k = rb::address_of(lengths), A.table = rb::address_of(table);
    A.page = C.page_stride * size, A.pages = C.pages, A.width = width, A.page_shift = __builtin_ctz((unsigned)C.page_tokens);
    A.n_seqs = n_seqs, A.tokens_q = tokens;
    A.heads = heads, A.kv_heads = C.kv_heads, A.group = heads / C.kv_heads, A.dim = C.dim, A.causal = 1;
    A.c = scale * LOG2E;
    A.parts = rb::address_of(workspace);
    const int units = rb::mx::device_groups();
    A.wanted = groups_wanted(tokens, n_seqs, A.kv_heads, A.group, std::min((long long)width * C.page_tokens, 0x7fffffffll), units);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (few_applies(tokens, n_seqs, A.group, (long long)width * C.page_tokens)) return (size == 1 ? launch_few8 : launch_few)(A, C.dtype, units, st);
    return launch(A, C.dtype, true, units, st);
}
rb_cache as16(const rb_cache8 &C) { return {C.k, C.v, C.pages, C.page_tokens, C.kv_heads, C.dim, C.dtype, C.page_stride, C.token_stride, C.head_stride}; }

}  // namespace

extern "C" size_t rb_attn_paged_workspace_bytes(const rb_cache *C, int heads, int n_seqs, int tokens)
{
    return check_cache(C) == RB_OK ? paged_workspace_bytes(*C, false, heads, n_seqs, tokens) : 0;
}

extern "C" int rb_attn_paged(const rb_cache *C, const void *q, long long q_token, long long q_head, int heads, const int32_t *first, const int32_t *lengths,
                             const int32_t *table, int width, int n_seqs, int tokens, float scale, void *o, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = check_cache(C);
    if (rc != RB_OK) return rc;
    return paged(*C, 2, nullptr, nullptr, q, q_token, q_head, heads, first, lengths, table, width, n_seqs, tokens, scale, o, workspace, workspace_bytes, stream);
}

extern "C" size_t rb_attn_cache8_workspace_bytes(const rb_cache8 *C, int heads, int n_seqs, int tokens)
{
    return check_cache8(C) == RB_OK ? paged_workspace_bytes(as16(*C), true, heads, n_seqs, tokens) : 0;
}

extern "C" int rb_attn_cache8(const rb_cache8 *C, const void *q, long long q_token, long long q_head, int heads, const int32_t *first, const int32_t *lengths,
                              const int32_t *table, int width, int n_seqs, int tokens, float scale, void *o, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = check_cache8(C);
    if (rc != RB_OK) return rc;
    return paged(as16(*C), 1, C->k_exp, C->v_exp, q, q_token, q_head, heads, first, lengths, table, width, n_seqs, tokens, scale, o, workspace, workspace_bytes, stream);
}
