// Attention of few new tokens per sequence over a paged cache in 8 bits: as rb_attn_few.hip, the time being that of reading the cache once.
//
// The same shares, one per wavefront.  Tiles of 32 keys go into LDS as they are, 8 bits an element, and are widened on their way to the matrix instructions: a key's elements
// in units of their own to the queries' type (exactly, but for fp16's last bits below 2^-24); a value's as they are, to bf16, their units going into the weights, which then have all the range of fp32
// and two parts of 16 bits, as good as 16 bits.  With half the bytes to a tile two of them per wavefront are asked for ahead, and two workgroups share a compute unit.  Once in two tiles the
// compiler waits for more than it has to: the loop may end between the two, and there it counts on the keys just asked for (heads of up to 64: on all loads, as half of the lanes make them).
//
// Bound: bytes of the cache that one long run of loads brings in, and that wait.  Kernels: 48 sequences of 250000 positions together, 8 key heads of 128 elements (518 MB, of which 521 are fetched): 103 us, 111 in
// another run (4.7 to 5.0 TB/s; a copy of 616 MB reaches 5.4), and 7.4 for joining; vector instructions are 43 % of its time.  8 heads of 64, half the bytes: 100 us for the call, 110 with 128.  Leaving out, for a
// measurement, the second part of the weights, the product with the values or the widening changed nothing; leaving out the units' bytes, lines of their own among the elements', with the wait for
// them, took off 4 %.  6 sequences of five drafted tokens, 40 heads (89 MB): 28.5 us and 6.6; one of 2000 tokens: 12.4 and 5.1, the chain of finding the share, its pages, its first tiles and the join.
#include <hip/hip_runtime.h>
#include <algorithm>

#include "rabit.h"
#include "rb_attn.h"
#include "rb_attn8.h"
#include "rb_attn_few.h"
#include "rb_attn_host.h"

namespace rb {
namespace attn {
namespace {

using few::Cursor, few::KEYS, few::part_of, few::ROWS, few::Shape, few::Shares, few::WAVES;

// A tile of 32 rows of D bytes (a head's elements and zeros after them) in LDS, 16-byte pieces of a row permuted: piece c of row r lies at c ^ spread(r).  Sixteen rows at one piece, and eight rows
// (four and four, eight apart) at one, then touch every bank once.
template <int D> struct Tile8 {
    static constexpr int BYTES = KEYS * D, PIECES = D / 16;
    static __device__ __forceinline__ int spread(int r) { return D == 128 ? (r >> 1) & 7 : (r >> 2) & 3; }
};

// Heads of a token lie next to each other where pages are [tokens][heads][elements]: a workgroup's four wavefronts then read 512 bytes in a row in place of four times 128 (calls: drafts over 40 heads 34 us,
// 45 with a head to a workgroup; 48 sequences 111 both, 119 with loads that the caches keep)
constexpr int XCDS = 8;
__host__ __device__ __forceinline__ int heads_together(int kv_heads) { return kv_heads % 4 == 0 ? 4 : kv_heads % 2 == 0 ? 2 : 1; }

template <class T, int D>
__global__ __launch_bounds__(64 * WAVES, 2) void few8_kernel(const Args A)
{
    using L = Tile8<D>;
    // tiles as variables of their own: the compiler then knows that loads into one do not concern reads of another
    __shared__ __attribute__((aligned(16))) uint8_t keys_a[WAVES * L::BYTES], values_a[WAVES * L::BYTES], keys_b[WAVES * L::BYTES], values_b[WAVES * L::BYTES];
    __shared__ __attribute__((aligned(16))) float units[WAVES * KEYS];
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // A workgroup's wavefronts have the same share of up to four heads: rows of these lie next to each other.  Those that have the same of the others are on the same XCD.
    const int wavefronts = A.wanted, together = heads_together(A.kv_heads), others = A.kv_heads / together;
    const int turn = (int)blockIdx.x / XCDS, kvh = turn % others * together + wave % together, w = (turn / others * XCDS + (int)blockIdx.x % XCDS) * (WAVES / together) + wave / together;
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

    const uint8_t *k_base = global_at<const uint8_t>(A.k.at) + kvh * A.k.head, *v_base = global_at<const uint8_t>(A.v.at) + kvh * A.v.head;
    auto in_range = [&](int page) RB_INLINE { return min(max(page, 0), A.pages - 1); };
    auto place = [&](int page, int r) RB_INLINE { return in_range(page) * A.page + (r & ((1 << A.page_shift) - 1)) * A.k.token; };
    auto exponent_place = [&](int page, int r) RB_INLINE { return (((long long)in_range(page) * A.kv_heads + kvh) << A.page_shift) + (r & ((1 << A.page_shift) - 1)); };
    int pages[4] = {};      // of the tile to be asked for next, per eight rows
    auto ask_pages = [&](const Cursor &c) RB_INLINE {
        const Uniform row = table_u + (long long)min(c.s, A.n_seqs - 1) * A.width;
        if (A.page_shift >= 5) {
            pages[0] = pages[1] = pages[2] = pages[3] = row[min((c.t * KEYS) >> A.page_shift, A.width - 1)];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) pages[i] = row[min((c.t * KEYS + i * 8) >> A.page_shift, A.width - 1)];
        }
    };
    // Eight rows a load, which lie in one page: 16 bytes per lane, of half the lanes where a row has but four pieces
    constexpr int LOADS = KEYS / 8;
    const int r8 = lane / L::PIECES;
    uint32_t offset[2];      // of this lane's piece of eight rows, where those are the tile's rows 0 .. 7 or 16 .. 23, and 8 .. 15 or 24 .. 31
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = (lane % L::PIECES) ^ L::spread(i * 8 + r8);
        offset[i] = c * 16 < A.dim ? (uint32_t)(r8 * A.k.token) + c * 16 : NOWHERE;
    }
    // tile number i of the share, which `ahead` stands at; past the share's end loads count, but fetch nothing
    auto load = [&](int i, const uint8_t *base, uint8_t *tile) RB_INLINE {
        const int r = ahead.t * KEYS, len = i < n ? ahead.n_k - r : 0;
        if (D == 128 || lane < 32) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int rows = min(len - j * 8, 8);
                load_to_lds(buffer(base + place(pages[j], r + j * 8), rows <= 0 ? 0u : (uint32_t)((rows - 1) * (int)A.k.token + A.dim)), tile + j * 8 * D, offset[j & 1]);
            }
        }
    };
    // its units' exponents: in the lower half of the lanes the keys', in the upper the values'
    const uint8_t *const exponents = global_at<const uint8_t>(h ? A.v_exp : A.k_exp);
    auto load_exponents = [&](int i) RB_INLINE {
        const int r = lane & 31, of[4] = {pages[0], pages[1], pages[2], pages[3]};
        const int low = r & 8 ? of[1] : of[0], high = r & 8 ? of[3] : of[2], page = r & 16 ? high : low;
        return (uint32_t)exponents[i < n && ahead.t * KEYS + r < ahead.n_k ? exponent_place(page, ahead.t * KEYS + r) : 0];
    };
    auto next_ahead = [&]() RB_INLINE {
        ahead.advance(A, entries);
        ask_pages(ahead);
    };

    // Keys as left operands: row lane % 32; the 16 bytes of a read are the operands of two instructions, so the elements of those are 32 (i / 2) + 16 h + 8 (i % 2) ..
    const int row_at = (lane & 31) * D, row_spread = L::spread(lane & 31);
    // Values, transposed on the way: eight rows of a column per lane, in the numbering of the weights
    const int v_row = 4 * h + (lane & 15) / 2 % 4 + (lane & 15) / 8 * 8, v_at = v_row * D + (lane & 1) * 8, v_spread = L::spread(v_row), v_piece = lane >> 4 & 1;
    typedef int v2i __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) v2i lds_v2i;
    auto value_operand = [&](const uint8_t *values, int b, int k) RB_INLINE {      // (16 rows on, the permutation is the same)
        const uint8_t *p = values + v_at + 16 * D * k + ((2 * b + v_piece) ^ v_spread) * 16;
        return widen8<BF16>(__builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i *)(lds_byte *)p)), 1.f);
    };

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
        for (int k = 0; k < D / 16; ++k) {
            const int e = k / 2 * 32 + h * 16 + k % 2 * 8;
            q[k] = e < A.dim ? *(const v4u *)(from + e * 2) : (v4u)(0u);
        }
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
                add_not_finite8<BF16, D>(sums, v_base + place(page, r), global_at<const uint8_t>(A.v_exp)[exponent_place(page, r)], A.dim, h, r <= limit);
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

    // Loads on their way behind the ones waited for: of a tile's keys, its exponents and values, and the next one's
    constexpr int LEFT = 3 * LOADS + 2;
    float *const units_w = units + wave * KEYS;
    auto step = [&](int i, uint8_t *keys, uint8_t *values, uint32_t &exponent) RB_INLINE {
        if (i > 0 && at.t == 0) {
            start();
            rows_arrived();
        }
        const uint32_t bits = max(exponent << 23, 0x400000u);      // (2^-127 is no normal number)
        const auto unit = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);      // of key lane % 32, and of its value
        const float key_unit = __uint_as_float(unit[0]);
        if (lane < 32) units_w[lane] = __uint_as_float(unit[1]);
        loads_arrived<LEFT>();
        v16f x = {};
        {
            v4u held[D / 32];
#pragma unroll
            for (int m = 0; m < D / 32; ++m) held[m] = *(const lds_v4u *)(lds_byte *)(keys + row_at + (((2 * m + h) ^ row_spread) * 16));
#pragma unroll
            for (int m = 0; m < D / 32; ++m) {
                x = T::mfma(widen8<T>((v2u){held[m].x, held[m].y}, key_unit), q[2 * m], x);
                x = T::mfma(widen8<T>((v2u){held[m].z, held[m].w}, key_unit), q[2 * m + 1], x);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        load(i + 2, k_base, keys);
        exponent = load_exponents(i + 2);
        const int first_key = at.t * KEYS;
        const bool cut = first_key + KEYS - 1 > least;      // some row does not see all of the tile's keys
        const int seen = limit - first_key - 4 * h;
        if (cut) {
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
        // Each weight times its value's unit in two parts of 16 bits, what the first leaves out being the second
        const float zero_at = top == RB_NEG_INF ? 0.f : top;
        uint32_t wt[8], rest[8];
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const v4f u = *(const __attribute__((address_space(3))) v4f *)(lds_byte *)(units_w + 2 * e + 4 * h);
            float p[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                p[j] = __builtin_amdgcn_exp2f(fmaf(x[e + j], A.c, -zero_at));
                total += p[j];
                p[j] *= u[j];
                if (cut && 8 * (e / 4) + j > seen) p[j] = 0.f;      // (whatever unit a value has that is not seen)
            }
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                const uint32_t both = wt[(e + j) / 2] = BF16::pack(p[j], p[j + 1]);
                rest[(e + j) / 2] = BF16::pack(p[j] - BF16::widen(both & 0xffffu), p[j + 1] - BF16::widen(both >> 16));
            }
        }
        const v4u p[2] = {{wt[0], wt[1], wt[2], wt[3]}, {wt[4], wt[5], wt[6], wt[7]}}, p_rest[2] = {{rest[0], rest[1], rest[2], rest[3]}, {rest[4], rest[5], rest[6], rest[7]}};
        loads_arrived<LEFT>();
        if (least < min(first_key + KEYS, at.n_k) - 1) {      // NaN in places that a row does not see: weight zero times such a value would be NaN
            bool any = false;
#pragma unroll
            for (int j = 0; j < L::BYTES / 1024; ++j) {
                lds_v4u *v = (lds_v4u *)(lds_byte *)(values + j * 1024 + lane * 16);
                const v4u was = *v;
                v4u is;
#pragma unroll
                for (int c = 0; c < 4; ++c) is[c] = without_nan8(was[c]);
                if (was.x != is.x || was.y != is.y || was.z != is.z || was.w != is.w) {
                    any = true;
                    *v = is;
                }
            }
            found |= __ballot(any) != 0;
        }
        {
            constexpr int AHEAD = 4;
            v4u held[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) held[k] = value_operand(values, k % B, k / B);
#pragma unroll
            for (int k = 0; k < 2 * B; ++k) {
                const v4u a = held[k % AHEAD];
                sums[k % B] = BF16::mfma(a, p[k / B], sums[k % B]);
                sums[k % B] = BF16::mfma(a, p_rest[k / B], sums[k % B]);
                if (k + AHEAD < 2 * B) held[k % AHEAD] = value_operand(values, (k + AHEAD) % B, (k + AHEAD) / B);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        load(i + 2, v_base, values);
        next_ahead();
        if (i == n - 1 || at.t == at.shape.tiles - 1) finish();
        at.advance(A, entries);
    };

    uint8_t *const ka = keys_a + wave * L::BYTES, *const va = values_a + wave * L::BYTES, *const kb = keys_b + wave * L::BYTES, *const vb = values_b + wave * L::BYTES;
    ask_pages(ahead);
    start();
    load(0, k_base, ka);
    uint32_t exponent_a = load_exponents(0);
    load(0, v_base, va);
    next_ahead();
    load(1, k_base, kb);
    uint32_t exponent_b = load_exponents(1);
    load(1, v_base, vb);
    next_ahead();
    rows_arrived();
    for (int i = 0; i < n && at.there(A); i += 2) {      // (past the last sequence only where the arrays are not in order)
        step(i, ka, va, exponent_a);
        if (i + 1 < n && at.there(A)) step(i + 1, kb, vb, exponent_b);
    }
    loads_arrived();
}

// two workgroups per compute unit, shared out over the key heads (calls with one each: 48 sequences 134 us in place of 111, drafts 38 in place of 34; a single sequence of 2000 tokens 16.9 in place of 17.3)
int groups_per_head(int kv_heads, int compute_units) { return std::max(2 * compute_units / kv_heads, 1); }

template <class T, int D> int launch(Args A, int compute_units, hipStream_t stream)
{
    const int groups = groups_per_head(A.kv_heads, compute_units), together = heads_together(A.kv_heads);
    A.wanted = groups * WAVES;
    const int shares = A.wanted / (WAVES / together), turns = (shares + XCDS - 1) / XCDS;      // workgroups of as many heads; those past the last share find no work
    return few::launch<T, D>(A, groups, stream, [&](dim3, dim3 threads) { hipLaunchKernelGGL((few8_kernel<T, D>), dim3((unsigned)(turns * XCDS * (A.kv_heads / together))), threads, 0, stream, A); });
}

}  // namespace

size_t few8_workspace_bytes(int kv_heads, int dim, int compute_units) { return few::workspace_bytes(kv_heads, dim, groups_per_head(kv_heads, compute_units)); }

int launch_few8(const Args &A, int dtype, int compute_units, hipStream_t stream)
{
    if (dtype == RB_F16) return A.dim <= 64 ? launch<F16, 64>(A, compute_units, stream) : launch<F16, 128>(A, compute_units, stream);
    return A.dim <= 64 ? launch<BF16, 64>(A, compute_units, stream) : launch<BF16, 128>(A, compute_units, stream);
}

}  // namespace attn
}  // namespace rb
