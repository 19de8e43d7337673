// What the attention kernels share: element types and their matrix instructions, tiles of keys and
// values in LDS, and the way from a workgroup's number to the rows it has to do.
//
// All products are v_mfma_f32_32x32x16.  Its operands hold, per lane, row (left) or column (right)
// lane % 32 and eight values along the contraction, of the half lane / 32; its result holds column
// lane % 32 and rows 8 (i / 4) + 4 (lane / 32) + i % 4 for i = 0..15.  Scores are computed transposed, keys
// by query rows: a lane then owns one query row, its softmax statistics are scalars of the lane, and
// the weights are already where the next product's right operand wants them, with the contraction
// index numbered 4 (lane / 32) + e % 4 + 8 (e / 4).  The left operand of that product, the transposed values,
// is read in the same numbering from the row-major tile by ds_read_b64_tr_b16 (four rows by
// sixteen columns per sixteen lanes, transposed on the way).
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

#include "rabit.h"
#include "rb_attn_shares.h"
#include "rb_device.h"

namespace rb {
namespace attn {

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
#define RB_NEG_INF (-__builtin_inff())
#define RB_INLINE __attribute__((always_inline))

// Weights are rounded to the inputs' type before they meet the values, each on its own and to
// nearest: one rounding of relative size 2^-11 (2^-8) per weight, which averages out over a row to what
// the rounding of the result costs.  fp16 reaches down to 2^-14 only at full precision, so its weights are
// kept 2^BIAS times as large as the softmax defines them.
struct F16 {
    static constexpr int BIAS = 6, GRAD_BIAS = 14;
    static constexpr uint32_t EXPONENT = 0x7c00u;
    static __device__ __forceinline__ v16f mfma(v4u a, v4u b, v16f c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){a, b}, v2h)); }
    static __device__ __forceinline__ float widen(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }
    // a packed pair's sum, in fp32, on top of another
    static __device__ __forceinline__ float sum(uint32_t w, float on) { return __builtin_amdgcn_fdot2(__builtin_bit_cast(v2h, w), (v2h){(_Float16)1.f, (_Float16)1.f}, on, false); }
};
struct BF16 {
    static constexpr int BIAS = 0, GRAD_BIAS = 0;
    static constexpr uint32_t EXPONENT = 0x7f80u;
    static __device__ __forceinline__ v16f mfma(v4u a, v4u b, v16f c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8b, a), __builtin_bit_cast(v8b, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){a, b}, v2b)); }
    static __device__ __forceinline__ float widen(uint32_t bits) { return __uint_as_float(bits << 16); }
    static __device__ __forceinline__ float sum(uint32_t w, float on) { return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2b, w), (v2b){(__bf16)1.f, (__bf16)1.f}, on, false); }
};

// an infinity or a NaN among the two 16-bit values of a word
template <class T> __device__ __forceinline__ bool not_finite(uint32_t w)
{
    constexpr uint32_t E = T::EXPONENT;
    return (w & E) == E || ((w >> 16) & E) == E;
}
template <class T> __device__ __forceinline__ uint32_t finite_part(uint32_t w)
{
    constexpr uint32_t E = T::EXPONENT;
    return ((w & E) == E ? 0 : w & 0xffffu) | (((w >> 16) & E) == E ? 0 : w & 0xffff0000u);
}

template <class T> __device__ __forceinline__ v4u finite_part(v4u w)
{
    return (v4u){finite_part<T>(w.x), finite_part<T>(w.y), finite_part<T>(w.z), finite_part<T>(w.w)};
}

// the sum or maximum of a lane's value and that of the lane 32 away, in both
__device__ __forceinline__ float over_halves_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float over_halves_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ------------------------------------------------------------------- tiles ---
// A tile is some rows of D elements (D = 64 or 128, a head's elements and zeros after them) in LDS, in groups of rows that
// one load of a wavefront fills (1 KB), 16 bytes between groups, 16-byte pieces of a row permuted: piece c of row r lies at c ^ spread(r).  So 32
// rows at one column and four rows at 32 columns both touch every bank once, and most of what varies in an address is a constant.
template <int D> struct Tile {
    static constexpr int ROW = D * 2, PIECES = D / 8, GROUP_ROWS = 1024 / ROW, GROUP = 1024 + 16;
    static __device__ __forceinline__ int spread(int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2 | ((r >> 2) & 1) << 1; }
    static constexpr int bytes(int rows) { return rows / GROUP_ROWS * GROUP; }
    static __device__ __forceinline__ int row_at(int r) { return r / GROUP_ROWS * GROUP + r % GROUP_ROWS * ROW; }
};

typedef __attribute__((address_space(3))) uint8_t lds_byte;
typedef __attribute__((address_space(3))) v4s lds_v4s;
typedef __attribute__((address_space(3))) v4u lds_v4u;

// Loads past the end of a buffer give zeros, in LDS too: rows past a sequence's end and elements past a
// head's last are zeros in every tile, whatever lies there in memory.
constexpr uint32_t NOWHERE = 0x7fffff00u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const uint8_t *p, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p), 0, (int)bytes, 0x00020000);
}

// W wavefronts load a tile, each some consecutive rows of it.  at[i]: where this lane's piece of load i lies behind the start of the buffer, whose row 0 is the row
// `first_row` rows before the wavefront's own
template <int D, int ROWS, int W> struct Part {
    using L = Tile<D>;
    static constexpr int LOADS = ROWS / L::GROUP_ROWS / W;
    uint32_t at[LOADS];
    __device__ __forceinline__ Part(long long stride, int dim, int first_row, int lane)
    {
        const int r = lane / L::PIECES, c = (lane % L::PIECES) ^ L::spread(r);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) at[i] = c * 8 < dim ? (uint32_t)((first_row + i * L::GROUP_ROWS + r) * stride) + c * 16 : NOWHERE;
    }
    // loads FROM .. FROM + N - 1 of the part, from a buffer
    template <int FROM, int N> __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t from, uint8_t *tile, int wave) const
    {
#pragma unroll
        for (int i = FROM; i < FROM + N; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)(tile + (wave * LOADS + i) * L::GROUP), 16, (int)at[i], 0, 0, 0);
    }
};
// `rows` rows of a head from `base` on, at most `most`; rows <= 0: nothing
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_buffer(const uint8_t *base, long long stride, int rows, int most, int dim)
{
    rows = min(rows, most);
    return buffer(base, rows <= 0 ? 0u : (uint32_t)((rows - 1) * (int)stride + dim * 2));
}

// Reads of a tile as left operands.  Rows: row 32 b + lane % 32, elements 16 k + 8 (lane / 32) ..; columns:
// element 32 b + lane % 32 of rows 16 k + the numbering above.
template <int D> struct Rows {
    int row, piece;
    __device__ __forceinline__ Rows(int lane) : row(Tile<D>::row_at(lane & 31)), piece(((lane >> 5) ^ Tile<D>::spread(lane & 31)) * 16) {}
    __device__ __forceinline__ void write(uint8_t *tile, int b, int k, v4u v) const
    {
        *(lds_v4u *)(lds_byte *)(tile + (row + (piece ^ (k * 32 & (D == 128 ? 192 : 96)))) + (k * 32 & (D == 128 ? ~192 : ~96)) + 32 / Tile<D>::GROUP_ROWS * Tile<D>::GROUP * b) = v;
    }
    __device__ __forceinline__ v4u read(const uint8_t *tile, int b, int k) const
    {
        constexpr int MOVED = D == 128 ? 192 : 96;      // bits of a piece's place that the permutation touches
        return *(const lds_v4u *)(lds_byte *)(tile + (row + (piece ^ (k * 32 & MOVED))) + (k * 32 & ~MOVED) + 32 / Tile<D>::GROUP_ROWS * Tile<D>::GROUP * b);
    }
};
template <int D> struct Columns {
    int row, piece;
    __device__ __forceinline__ Columns(int lane)
    {
        const int h = lane >> 5, i = lane & 15, r = 4 * h + i / 4, c = (lane >> 4 & 1) * 2 + (i & 3) / 2;
        row = Tile<D>::row_at(r) + (i & 1) * 8;
        piece = (c ^ Tile<D>::spread(r)) * 16;
    }
    __device__ __forceinline__ v4u read(const uint8_t *tile, int b, int k) const
    {
        constexpr int EIGHT = 8 / Tile<D>::GROUP_ROWS * Tile<D>::GROUP;      // the permutation is the same eight rows on
        const uint8_t *p = tile + (row + (piece ^ (b * 64))) + 2 * EIGHT * k;
        const v2u lo = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(lds_byte *)p));
        const v2u hi = __builtin_bit_cast(v2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(lds_byte *)(p + EIGHT)));
        return (v4u){lo.x, lo.y, hi.x, hi.y};
    }
};

// N matrix instructions, each with a left operand from LDS that is read AHEAD instructions before its use.  The order is held: left alone, the
// compiler puts every read right before its use and waits for it (see the figures at the kernels).
template <int N, int AHEAD, class Read, class Use> __device__ __forceinline__ void stream_operands(Read read, Use use)
{
    v4u held[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) held[i] = read(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        use(i, held[i % AHEAD]);
        if (i + AHEAD < N) held[i % AHEAD] = read(i + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Infinities and NaN in places that a row does not see: weight zero times such a value would be NaN.  Tiles of which some row of the
// workgroup sees only a part are looked through before use: what is not finite becomes zero, and `found` says that there was some.
template <class T, int D, int ROWS, int W> __device__ __forceinline__ void make_finite(uint8_t *tile, int *found, int tid)
{
    using L = Tile<D>;
#pragma unroll
    for (int i = 0; i < ROWS / L::GROUP_ROWS / W; ++i) {
        lds_v4u *at = (lds_v4u *)(lds_byte *)(tile + (i * W + (tid >> 6)) * L::GROUP + (tid & 63) * 16);
        const v4u w = *at;
        if (not_finite<T>(w.x) || not_finite<T>(w.y) || not_finite<T>(w.z) || not_finite<T>(w.w)) {
            *found = 1;
            *at = finite_part<T>(w);
        }
    }
}
// At the end, where something was found: sums [element][column of the lane] += what is not finite in row `from` (in memory), if the lane's
// column sees it.  Any weight gives the same.
template <class T, int D> __device__ __forceinline__ void add_not_finite(v16f (&sums)[D / 32], const uint8_t *from, int dim, int h, bool seen)
{
    const __amdgpu_buffer_rsrc_t row = buffer(from, dim * 2);
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const v2u w = __builtin_bit_cast(v2u, __builtin_amdgcn_raw_buffer_load_b64(row, h * 8, (b * 32 + 2 * i) * 2, 0));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t bits = (j < 2 ? w.x : w.y) >> (j % 2 * 16) & 0xffffu;
                if (seen && (bits & T::EXPONENT) == T::EXPONENT) sums[b][i + j] += T::widen(bits);
            }
        }
}
// sums [element][column], element 32 b + 8 (i / 4) + 4 h + i % 4, as a row of 16-bit values per column; `empty`: zeros whatever they are
template <class T, int D> __device__ __forceinline__ void store_columns(const v16f (&sums)[D / 32], float scale, uint8_t *to, int dim, int h, bool real, bool empty)
{
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 8) {
            // elements 0-3 and 8-11 of a run of 16 are in the lower half, the others in the upper: exchanged, each half stores eight in a row
            const auto lo = __builtin_amdgcn_permlane32_swap(T::pack(sums[b][i] * scale, sums[b][i + 1] * scale), T::pack(sums[b][i + 4] * scale, sums[b][i + 5] * scale), false, false);
            const auto hi = __builtin_amdgcn_permlane32_swap(T::pack(sums[b][i + 2] * scale, sums[b][i + 3] * scale), T::pack(sums[b][i + 6] * scale, sums[b][i + 7] * scale), false, false);
            const int e = b * 32 + i * 2 + h * 8;
            if (real && e < dim) *(v4u *)(to + e * 2) = empty ? (v4u)(0u) : (v4u){lo[0], hi[0], lo[1], hi[1]};
        }
}
// the loads into LDS that this wavefront has asked for have arrived, all but the last LEFT: a barrier alone does not wait for them
template <int LEFT = 0> __device__ __forceinline__ void loads_arrived() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory"); }
// the barrier alone: __syncthreads() would wait for all loads
__device__ __forceinline__ void meet()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// -------------------------------------------------------------------- work ---
// Sequences are packed: sequence s has the tokens first[s] .. first[s + 1] - 1.  The rows of a key head are its queries, group after
// group of the heads that share it: row = token * group + head of the group.  Blocks of BM rows are numbered so that the
// number of a sequence's first block follows from first[s] alone, floor(first[s] group / BM) + s, without a sum over the
// sequences before it; some numbers between two sequences belong to nobody.
__device__ __forceinline__ int block_start(int first, int s, int group, int BM) { return (int)((long long)first * group / BM) + s; }
inline long long block_numbers(long long tokens, int n_seqs, int group, int BM) { return tokens * group / BM + n_seqs; }

// the last of n places whose start is not beyond `value` (place 0's never is); a wavefront looks at 64 at a time
template <class Start> __device__ __forceinline__ int last_not_beyond(int n, int value, int lane, Start start)
{
    const int last = n - 1;
    int lo = 0;
    while (n > 1) {
        const int step = (n + 63) / 64;
        const unsigned long long below = __ballot(lane * step < n && start(min(lo + lane * step, last)) <= value);
        const int k = max(0, __popcll(below) - 1);
        lo += k * step;
        n = min(step, n - k * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}
__device__ __forceinline__ int sequence_of_block(const int *first, int n_seqs, int group, int BM, int block, int lane)
{
    return last_not_beyond(n_seqs, block, lane, [&](int s) { return block_start(first[s], s, group, BM); });
}

// Of up to MOST_ORDERED sequences: their blocks in descending order of work, so that the longest start first and short ones fill the gaps.  count(n_q, n_k, x): how many
// blocks of such a sequence have a work of x or more, all of them for x = 0; `most`: a bound on the work.  n_q, n_k: of sequence lane % pad, where pad is
// the power of two that holds n_seqs (zeros past them): so many lanes add up a count, and the groups of them look at several x at once.  False: there are not so many blocks.
// Every workgroup does this for itself, in one to five microseconds.  (Heads of 128, 32 query and 8 key heads, against the order of the sequences: two sequences of 4000 tokens in all
// 87 -> 83 us; five of 6000 the same forwards and the keys' part of the gradient 289 -> 259; eleven of 6300, not causal, 12 and 4 heads of 64, 46 -> 41; sixteen of 6000 60 -> 58.5;
// 17 of 6000 52 -> 61; 40 of 8000 55 -> 79; and where all workgroups run at once only the time for it is left, sixteen of 1000 8.3 -> 9.6.)
constexpr int MOST_ORDERED = 16;
__device__ __forceinline__ int padded(int n_seqs) { return 1 << (32 - __builtin_clz(n_seqs - 1)); }      // (n_seqs >= 2)
template <class Count> __device__ __forceinline__ bool nth_heaviest(int n_seqs, int n_q, int n_k, int nth, int most, int lane, int &s, int &block, Count count)
{
    const int pad = padded(n_seqs), groups = 64 / pad, group = lane / pad;
    auto over_sequences = [&](int v) {
        for (int d = 1; d < pad; d <<= 1) v += __shfl_xor(v, d);
        return v;
    };
    if (__builtin_amdgcn_readfirstlane(over_sequences(count(n_q, n_k, 0))) <= nth) return false;
    int lo = 0, n = most + 1;      // the largest x of which there are more than nth lies in lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + groups) / (groups + 1), at = (group + 1) * step;
        const int more = __popcll(__ballot(over_sequences(count(n_q, n_k, lo + min(at, n))) > nth && at < n)) / pad;
        lo += more * step;
        n = min(step, n - more * step);
    }
    const int here = count(n_q, n_k, lo), heavier = count(n_q, n_k, lo + 1);
    nth -= __builtin_amdgcn_readfirstlane(over_sequences(heavier));      // among those of work lo, in the order of the sequences
    int upto = here - heavier;
    for (int d = 1; d < pad; d <<= 1) {
        const int v = __shfl_up(upto, d);
        if (lane >= d) upto += v;
    }
    s = min(__builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < n_seqs && upto <= nth))), n_seqs - 1);
    block = __builtin_amdgcn_readlane(heavier, s) + nth - (s ? __builtin_amdgcn_readlane(upto, s - 1) : 0);
    return true;
}

// One sequence's part of the work.  What the arrays say is brought into the range of the buffers: an array that
// is not in order gives wrong results, but no access outside.
struct Sequence {
    int q0, n_q, k0, n_k;
};
__device__ __forceinline__ Sequence sequence_at(const int *first_q, const int *first_k, int s, int tokens_q, int tokens_k)
{
    // (the same in all lanes, which the compiler has to be told: an address that it takes to differ costs a loop over the lanes)
    auto entry = [&](const int *first, int i) { return __builtin_amdgcn_readfirstlane(first[i]); };
    Sequence r;
    r.q0 = min(max(entry(first_q, s), 0), tokens_q);
    r.n_q = min(max(entry(first_q, s + 1), r.q0), tokens_q) - r.q0;
    r.k0 = min(max(entry(first_k, s), 0), tokens_k);
    r.n_k = min(max(entry(first_k, s + 1), r.k0), tokens_k) - r.k0;
    return r;
}

// `running`: how many workgroups run at once
inline bool ordered_for(int n_seqs, long long workgroups, long long running) { return n_seqs > 1 && n_seqs <= MOST_ORDERED && workgroups > running; }

// Which sequence and which of its blocks a workgroup's number stands for; false: none.  Blocks of BM rows (keys: BM keys), if `ordered` heaviest first, by steps of 64 keys (rows): causal
// rows see more the later they are, causal keys are seen by more the earlier they are.
template <int BM>
__device__ __forceinline__ bool rows_of_workgroup(const int *first_q, const int *first_k, int n_seqs, bool ordered, int tokens_q, int tokens_k, int group, bool causal, int number, int numbers, int lane, int &s, int &block)
{
    if (ordered) {
        const int at = lane & (padded(n_seqs) - 1), i = min(at, n_seqs - 1);
        const int q0 = min(max(first_q[i], 0), tokens_q), k0 = min(max(first_k[i], 0), tokens_k);
        const int n_q = at < n_seqs ? min(max(first_q[i + 1], q0), tokens_q) - q0 : 0, n_k = at < n_seqs ? min(max(first_k[i + 1], k0), tokens_k) - k0 : 0;
        auto blocks = [&](int rows) { return (rows * group + BM - 1) / BM; };
        if (!nth_heaviest(n_seqs, n_q, n_k, number, tokens_k / 64, lane, s, block, [&](int q, int k, int x) {
                const int beyond = k - x * 64;
                if (x == 0 || !causal) return beyond >= 0 ? blocks(q) : 0;
                return beyond < 0 ? 0 : min(blocks(q), (int)((long long)beyond * group / BM) + 1);
            }))
            return false;
        if (causal) block = blocks(__builtin_amdgcn_readlane(n_q, s)) - 1 - block;
        return true;
    }
    if (causal) number = numbers - 1 - number;
    s = sequence_of_block(first_q, n_seqs, group, BM, number, lane);
    block = number - block_start(first_q[s], s, group, BM);
    return true;
}
template <int BM>
__device__ __forceinline__ bool keys_of_workgroup(const int *first_q, const int *first_k, int n_seqs, bool ordered, int tokens_q, int tokens_k, bool causal, int number, int lane, int &s, int &block)
{
    if (ordered) {
        const int at = lane & (padded(n_seqs) - 1), i = min(at, n_seqs - 1);
        const int q0 = min(max(first_q[i], 0), tokens_q), k0 = min(max(first_k[i], 0), tokens_k);
        const int n_q = at < n_seqs ? min(max(first_q[i + 1], q0), tokens_q) - q0 : 0, n_k = at < n_seqs ? min(max(first_k[i + 1], k0), tokens_k) - k0 : 0;
        return nth_heaviest(n_seqs, n_q, n_k, number, tokens_q / 64, lane, s, block, [&](int q, int k, int x) {
            const int blocks = (k + BM - 1) / BM;
            if (x == 0 || !causal) return q >= x * 64 ? blocks : 0;
            return q < x * 64 || k < x * 64 ? 0 : min(blocks, (k - x * 64) / BM + 1);
        });
    }
    s = sequence_of_block(first_k, n_seqs, 1, BM, number, lane);
    block = number - block_start(first_k[s], s, 1, BM);
    return true;
}

// Operands of a call; strides in bytes.
struct Side {
    Address at;
    long long token, head;
};
struct Args {
    Side q, k, v;
    Address o, lse, first_q, first_k;        // paged: first_k holds the sequences' lengths
    Address table;
    long long page;
    int n_seqs, tokens_q, tokens_k, heads, kv_heads, group, dim, causal, ordered;
    int page_shift, pages, width;
    Address parts;                           // workspace
    int wanted;                              // workgroups per key head that the work is shared out to; 0: one per block of rows
    float per_tile;                          // how many of them for a tile
    float c;                                 // scale log2(e): the exponentials are powers of two
};

// Weights are taken relative to a maximum that follows the scores only when they pass it by this many powers of two: the sums
// are rescaled a few times per row instead of at every tile.  2^(8 + BIAS) is within fp16.
constexpr float SLACK = 8.f;

// Work over a cache: that of a key head is a row of pieces (tiles, workgroups), sequence after sequence and job (a block of JOB rows) after job.  Shape says what a sequence has
// of it: of(A, q0, q1, length), and count() pieces.
//
// Sums over the sequences, 64 at a time, the first 64 looked at once
template <class Shape> struct Sums {
    static constexpr int JOB = Shape::JOB;
    const Args &A;
    const int *first, *lengths;
    int lane, q0, q1, length, upto;      // what the arrays say of sequence `lane`; the tiles of sequences 0 .. lane
    __device__ __forceinline__ Sums(const Args &A_, const int *first_, const int *lengths_, int lane_) : A(A_), first(first_), lengths(lengths_), lane(lane_)
    {
        const int s = min(lane, A.n_seqs - 1);
        q0 = first[s], q1 = first[s + 1], length = lengths[s];
        upto = up_to_lane(lane < A.n_seqs ? Shape::of(A, q0, q1, length).count() : 0);
    }
    template <class Other> __device__ __forceinline__ Sums(const Args &A_, const Sums<Other> &o) : A(A_), first(o.first), lengths(o.lengths), lane(o.lane), q0(o.q0), q1(o.q1), length(o.length)
    {
        upto = up_to_lane(lane < A.n_seqs ? Shape::of(A, q0, q1, length).count() : 0);
    }
    __device__ __forceinline__ int count(int s) const { return s < A.n_seqs ? Shape::of(A, first[s], first[s + 1], lengths[s]).count() : 0; }
    __device__ __forceinline__ int up_to_lane(int v) const
    {
        for (int d = 1; d < 64; d <<= 1) {
            const int u = __shfl_up(v, d);
            if (lane >= d) v += u;
        }
        return v;
    }
    __device__ __forceinline__ void entries(int s, int &from, int &to, int &len) const      // of one sequence
    {
        if (s < 64) {      // at hand
            from = __builtin_amdgcn_readlane(q0, s), to = __builtin_amdgcn_readlane(q1, s), len = __builtin_amdgcn_readlane(length, s);
        } else {
            typedef const __attribute__((address_space(4))) int *Uniform;
            from = ((Uniform)first)[s], to = ((Uniform)first)[s + 1], len = ((Uniform)lengths)[s];
        }
    }
    __device__ __forceinline__ int of_block(int block) const
    {
        if (A.n_seqs > 64) return sequence_of_block(first, A.n_seqs, A.group, JOB, block, lane);
        return max(__popcll(__ballot(lane < A.n_seqs && block_start(q0, lane, A.group, JOB) <= block)) - 1, 0);
    }
    // the tiles before sequence `end`
    __device__ __forceinline__ int before(int end) const
    {
        if (end <= 64) return end > 0 ? __builtin_amdgcn_readlane(upto, end - 1) : 0;
        int sum = 0;
        for (int s = 64 + lane; s < end; s += 64) sum += count(s);
        return __builtin_amdgcn_readlane(upto, 63) + __builtin_amdgcn_readlane(up_to_lane(sum), 63);
    }
    // the sequence that has tile `at` (which exists); `at` becomes the tile among its own
    __device__ __forceinline__ int locate(int &at) const
    {
        int now = upto;
        for (int s = 0; s < A.n_seqs; s += 64) {
            if (s) now = up_to_lane(count(s + lane));
            const int here = __builtin_amdgcn_readlane(now, 63);
            if (at < here) {
                const int l = __popcll(__ballot(now <= at));
                if (l) at -= __builtin_amdgcn_readlane(now, l - 1);
                return s + l;
            }
            at -= here;
        }
        return A.n_seqs;
    }
};
// workgroups that share `tiles` tiles: two tiles each at least
__device__ __forceinline__ int splits_of(int tiles, int splits) { return max(min(splits, tiles / 2), 1); }

// Parts of the same rows over different keys, unnormalised, in memory: the rows' maxima and sums, then the rows.
template <int D, int N> struct PartOfRows {
    static constexpr size_t FLOATS = N * (2 + D);
    float *at;
    __device__ __forceinline__ PartOfRows(Address workspace, size_t which) : at(global_at<float>(workspace) + which * FLOATS) {}
    __device__ __forceinline__ float *top(int row) const { return at + row; }
    __device__ __forceinline__ float *total(int row) const { return at + N + row; }
    __device__ __forceinline__ float *row(int row) const { return at + 2 * N + row * D; }
    // from the lane that has column `row` of the sums, both halves of the wavefront
    __device__ __forceinline__ void store(const v16f (&sums)[D / 32], float row_top, float row_total, int r, int h) const
    {
        if (h == 0) {
            *top(r) = row_top;
            *total(r) = row_total;
        }
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 4) *(v4f *)(row(r) + b * 32 + 2 * i + 4 * h) = (v4f){sums[b][i], sums[b][i + 1], sums[b][i + 2], sums[b][i + 3]};
    }
};
// Joins n_parts of the `joined` rows (two, four or eight) from row0 on, of which n_rows are there: o = sum of the parts' rows, each times 2^(its maximum - the
// largest), over the sum of their totals likewise, in the order of the parts.  256 threads, four elements each; the groups of threads that make up a row share
// out the parts.  Bound: latency, so all loads of sixteen parts and group are on their way before the first is used.  part(i): a PartOfRows; out(row): where
// the result goes; empty(row): it sees nothing.
template <class T, int D, class Part_, class Out, class Empty>
__device__ __forceinline__ void join_rows(int joined, int n_parts, int row0, int n_rows, int dim, Part_ part, Out out, Empty empty)
{
    constexpr int COLUMNS = D / 4, GROUPS = 256 / COLUMNS, HELD = 16;
    __shared__ float sums[GROUPS][D], tops[GROUPS], totals[GROUPS];
    const int column = threadIdx.x % COLUMNS, group = threadIdx.x / COLUMNS, lg = 31 - __builtin_clz(joined), sharing = GROUPS >> lg;
    const int i = group & (joined - 1), p0 = group >> lg, r = row0 + i;
    const bool mine = i < n_rows;
    auto weight = [](float top, float most) { return most == RB_NEG_INF ? 1.f : __builtin_amdgcn_exp2f(top - most); };
    float most = RB_NEG_INF, total = 0.f;      // of this group's parts
    v4f sum = {};
    for (int w0 = p0; w0 < n_parts; w0 += HELD * sharing) {
        v4f x[HELD];
#pragma unroll
        for (int j = 0; j < HELD; ++j) x[j] = mine && w0 + j * sharing < n_parts ? *(const v4f *)(part(w0 + j * sharing).row(r) + column * 4) : (v4f)(0.f);
        // the parts' maxima and totals, one per lane
        const bool has = mine && column < HELD && w0 + column * sharing < n_parts;
        float t = has ? *part(w0 + column * sharing).top(r) : RB_NEG_INF, part_total = has ? *part(w0 + column * sharing).total(r) : 0.f;
        float now = t;
        for (int d = COLUMNS / 2; d > 0; d >>= 1) now = fmaxf(now, __shfl_xor(now, d));
        now = fmaxf(now, most);
        const float before = weight(most, now), w = weight(t, now);
        most = now;
        part_total *= w;
        for (int d = COLUMNS / 2; d > 0; d >>= 1) part_total += __shfl_xor(part_total, d);
        total = total * before + part_total;
        sum *= before;
#pragma unroll
        for (int j = 0; j < HELD; ++j) sum += x[j] * __shfl(w, j, COLUMNS);
    }
    *(v4f *)&sums[group][column * 4] = sum;
    if (column == 0) tops[group] = most, totals[group] = total;
    __syncthreads();
    if (p0 == 0 && mine && column * 4 < dim) {
        for (int g = group; g < GROUPS; g += joined) most = fmaxf(most, tops[g]);
        sum = (v4f)(0.f);
        total = 0.f;
        for (int g = group; g < GROUPS; g += joined) {
            const float f = weight(tops[g], most);
            sum += *(const v4f *)&sums[g][column * 4] * f;
            total += totals[g] * f;
        }
        const float norm = 1.f / total;
        *(v2u *)(out(r) + column * 8) = empty(r) ? (v2u)(0u) : (v2u){T::pack(sum[0] * norm, sum[1] * norm), T::pack(sum[2] * norm, sum[3] * norm)};
    }
}

}  // namespace attn
}  // namespace rb
