// Gradient of attention over packed prompts.  With p_ij = exp(c q_i . k_j - lse_i), given do:
//   dv_j = sum_i p_ij do_i        dp_ij = do_i . v_j        delta_i = do_i . o_i
//   ds_ij = c p_ij (dp_ij - delta_i)        dq_i = sum_j ds_ij k_j        dk_j = sum_i ds_ij q_i
// Two kernels, one with the queries in place and the keys going by (dq), then one the other way round (dk, dv).  The scores are computed twice; in return
// every sum has one owner, which adds in one order: no atomics, the same bits every time, and the query heads that share a key head are summed in registers, or
// where keys are few by a few workgroups each of which has some of them, and a last kernel adds those up.
//
// o comes rounded, so do_i . o_i is off by some 2^-12 |do_i| |o_i|: as much as the rounding of ds does to dq and dk again.  The first kernel mends that: over a row,
// sum_j p_ij (dp_ij - delta_i) is what delta_i lacks (the weights add up to one), so it sums that beside dq, and sum_j p_ij k_j, which
// the missing part would have been multiplied with, and stores the full delta for the second kernel.  One product more than the
// five of the definition and the two that are computed twice.  In dq the missing part is taken from ds as rounded for the product, so where one key has nearly all the
// weight both cancel to the last bits; the second kernel subtracts delta from the same dp, product by product, as the first, and where one key has all of it ds is exactly zero.
//
// ds is rounded to the inputs' type before it meets k and q.  In fp16 that takes a scale: ds is p times something of the size of do, and both are small.  As the forward pass follows a row's
// maximum, each row's dq, and each key's dk, has a power of two of its own that follows the largest |ds| met so far (Unit): what a row or a key does not see takes no part in it, and
// what comes before a larger one keeps its bits, since the sums are fp32.
#include <hip/hip_runtime.h>
#include <algorithm>

#include "rabit.h"
#include "rb_attn.h"
#include "rb_attn_host.h"
#include "rb_internal.h"

namespace rb {
namespace attn {
namespace {

constexpr int ROWS = 64;

struct GradArgs {
    Side q, k, v, o;                    // o: strides of the contiguous o, do and dq
    Address go, lse, first_q, first_k;
    Address delta;                      // workspace: [tokens_q][heads] fp32
    Address parts;                      // workspace: [splits][dk, dv][tokens_k][kv_heads][dim] fp32, where there are several splits
    Address dq, dk, dv;
    int splits;                         // workgroups that share the query heads of the same keys
    int n_seqs, tokens_q, tokens_k, heads, kv_heads, group, dim, causal, ordered, ordered_keys;
    float c, scale;
};

// ------------------------------------------------------------------ delta ---
// Sixteen lanes per row, four rows per wavefront and step; a workgroup takes 64 tokens of one head of do and o.  Bound: bytes (6092 tokens of 32 heads of 128,
// bf16: 16.8 us, 6.0 TB/s, o being just written).
template <class T> __global__ __launch_bounds__(256) void delta_kernel(const GradArgs A)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = (lane & 15) * 8;
    const int head = blockIdx.x % A.heads, block = blockIdx.x / A.heads;
    for (int i = 0; i < 4; ++i) {
        const int token = block * 64 + (wave * 4 + i) * 4 + lane / 16;
        if (token >= A.tokens_q) continue;      // whole groups of 16 lanes
        v4u x = (v4u)(0u), y = (v4u)(0u);
        if (e < A.dim) {
            const long long at = token * A.o.token + head * A.o.head;
            x = *(const v4u *)(global_at<const uint8_t>(A.go) + at + e * 2);
            y = *(const v4u *)(global_at<const uint8_t>(A.o.at) + at + e * 2);
        }
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += T::widen(x[j] & 0xffffu) * T::widen(y[j] & 0xffffu) + T::widen(x[j] >> 16) * T::widen(y[j] >> 16);
        for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
        if ((lane & 15) == 0) global_at<float>(A.delta)[(long long)token * A.heads + head] = sum;
    }
}

// The power of two that the ds of a lane's column (a row's, a key's) are held in; 1 where the type has fp32's range.  It starts at 2^60, where fp16 resolves ds of 2^-98, and
// falls to bring the largest to 2^10 whenever one passes 2^15: 24 binades below stay at full precision, and it seldom moves.  It does not fall below 2^-60, which holds every finite ds.
template <class T> struct Unit {
    float unit = T::GRAD_BIAS ? 0x1p60f : 1.f;
    static __device__ __forceinline__ float power(uint32_t field) { return __uint_as_float(field << 23); }
    __device__ __forceinline__ float inverse() const { return power(254u - (__float_as_uint(unit) >> 23)); }
    // d: 16 of the column, with `unit` in them already; both halves of the wavefront call it.  What is held in the unit is to be multiplied by `moved`, the d are already
    __device__ __forceinline__ bool follow(v16f &d, float &moved)
    {
        if constexpr (!T::GRAD_BIAS) return false;
        float most = fabsf(d[0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) most = fmaxf(most, fabsf(d[i]));
        most = over_halves_max(most);
        if (!__ballot(most > 0x1p15f)) return false;
        const int field = __float_as_uint(unit) >> 23, now = most > 0x1p15f ? max(field + 137 - (int)(__float_as_uint(most) >> 23), 67) : field;
        moved = power(127 + now - field);
        unit = power(now);
#pragma unroll
        for (int i = 0; i < 16; ++i) d[i] *= moved;
        return true;
    }
};

// An infinity or a NaN in the tile?  (see make_finite: here the tile itself is needed as it is, and what is read transposed is cleaned)
template <class T, int D, int R, int W> __device__ __forceinline__ void look_through(const uint8_t *tile, int *found, int tid)
{
    using L = Tile<D>;
#pragma unroll
    for (int i = 0; i < R / L::GROUP_ROWS / W; ++i) {
        const v4u w = *(const lds_v4u *)(lds_byte *)(tile + (i * W + (tid >> 6)) * L::GROUP + (tid & 63) * 16);
        if (not_finite<T>(w.x) || not_finite<T>(w.y) || not_finite<T>(w.z) || not_finite<T>(w.w)) *found = 1;
    }
}
// sums of the second of two wavefronts are added to the first's, by way of LDS (all wavefronts of the workgroup call this); true in the first
template <int E> __device__ __forceinline__ bool add_halves(v16f (&sums)[E], uint8_t *by, int half, int lane)
{
    if (half == 1)
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < 16; i += 4) *(v4f *)(by + (e * 4 + i / 4) * 1024 + lane * 16) = (v4f){sums[e][i], sums[e][i + 1], sums[e][i + 2], sums[e][i + 3]};
    __syncthreads();
    if (half == 0)
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const v4f other = *(const v4f *)(by + (e * 4 + i / 4) * 1024 + lane * 16);
                sums[e][i] += other[0], sums[e][i + 1] += other[1], sums[e][i + 2] += other[2], sums[e][i + 3] += other[3];
            }
    __syncthreads();
    return half == 0;
}

// --------------------------------------------------------------- dk and dv ---
// A workgroup keeps 128 keys and values of one key head in LDS and takes the queries and do of all its query heads, 64 rows at a
// time, through LDS.  Eight wavefronts: four times 32 keys, by the upper and the lower 32 rows of a tile, whose sums are added at the end.  All operands come from LDS,
// since the two sums of 32 keys fill half of the registers (with keys and values in registers they spilled, which costs more than twice the time: what is spilled waits behind
// the loads).  Bound: matrix and vector instructions, which two wavefronts per SIMD overlap in part, and the power the former may draw (five sequences of 6000 tokens in all,
// 32 heads of 128, causal, bf16: 274 us, 0.63 PFLOP/s for its four products).  Blocks in the order of the sequences instead of the heaviest first: 289 us against 265.
constexpr int BN = 128;
__device__ __forceinline__ float *part_at(const GradArgs &A, int split, int which, long long row)
{
    return global_at<float>(A.parts) + ((long long)(split * 2 + which) * A.tokens_k * A.kv_heads + row) * A.dim;
}

template <class T, int D>
__global__ __launch_bounds__(512, 2) void keys_kernel(const GradArgs A)
{
    using L = Tile<D>;
    constexpr int W = 8, LOADS = Part<D, ROWS, W>::LOADS, E = D / 32;
    __shared__ __attribute__((aligned(16))) uint8_t queries_a[L::bytes(ROWS)], outs_a[L::bytes(ROWS)], queries_b[L::bytes(ROWS)], outs_b[L::bytes(ROWS)], keys[L::bytes(BN)], values[L::bytes(BN)];
    // of the rows: the exponent that their weights are taken relative to, and delta
    __shared__ __attribute__((aligned(16))) float rows_a[2][ROWS], rows_b[2][ROWS];
    __shared__ int found;
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), part = wave & 3, half = wave >> 2;
    const int kvh = blockIdx.x % A.kv_heads, block = blockIdx.x / A.kv_heads, split = blockIdx.y;      // causal: the first keys have the most rows
    const int first_g = A.group * split / A.splits, heads_of = A.group * (split + 1) / A.splits - first_g;
    const int *first_q = global_at<const int>(A.first_q), *first_k = global_at<const int>(A.first_k);
    int s, of_sequence;
    if (!keys_of_workgroup<BN>(first_q, first_k, A.n_seqs, A.ordered_keys, A.tokens_q, A.tokens_k, A.causal, block, lane, s, of_sequence)) return;
    const Sequence S = sequence_at(first_q, first_k, s, A.tokens_q, A.tokens_k);
    const int key0 = of_sequence * BN;
    if (key0 < 0 || key0 >= S.n_k) return;
    const int ahead = S.n_k - S.n_q;
    const int my_key = key0 + part * 32 + (lane & 31), key = min(my_key, S.n_k - 1);
    const int block_last = min(key0 + BN, S.n_k) - 1, wave_first = key0 + part * 32, wave_last = min(wave_first + 31, S.n_k - 1);

    Unit<T> held;
    const Part<D, ROWS, W> q_part(A.q.token, A.dim, wave * (ROWS / W), lane), o_part(A.o.token, A.dim, wave * (ROWS / W), lane);
    const int tile0 = A.causal ? max(key0 - ahead, 0) / ROWS : 0, tiles = (S.n_q + ROWS - 1) / ROWS - tile0;
    const int steps = __builtin_amdgcn_readfirstlane(tiles > 0 ? tiles * heads_of : 0);
    float next_lse = 0.f, next_delta = 0.f;      // of one row of the next tile, in the first wavefront
    int load_g = first_g, load_t = tile0, t = tile0;      // the tile to be asked for, and the one at hand
    auto load = [&](uint8_t *queries, uint8_t *outs) RB_INLINE {
        const int head = kvh * A.group + load_g, row = S.q0 + load_t * ROWS, rows = S.n_q - load_t * ROWS;
        if (wave == 0) {
            const long long at = (long long)(row + min(lane, rows - 1)) * A.heads + head;
            next_lse = global_at<const float>(A.lse)[at];
            next_delta = global_at<const float>(A.delta)[at];
        }
        const uint8_t *q_from = global_at<const uint8_t>(A.q.at) + (long long)row * A.q.token + head * A.q.head;
        const uint8_t *o_from = global_at<const uint8_t>(A.go) + (long long)row * A.o.token + head * A.o.head;
        q_part.template load<0, LOADS>(rows_buffer(q_from, A.q.token, rows, ROWS, A.dim), queries, wave);
        o_part.template load<0, LOADS>(rows_buffer(o_from, A.o.token, rows, ROWS, A.dim), outs, wave);
        if (++load_t == tile0 + tiles) load_t = tile0, ++load_g;
    };

    if (tid == 0) found = 0;
    if (steps > 0) load(queries_a, outs_a);
    {
        const Part<D, BN, W> k_part(A.k.token, A.dim, wave * (BN / W), lane), v_part(A.v.token, A.dim, wave * (BN / W), lane);
        const uint8_t *from_k = global_at<const uint8_t>(A.k.at) + (long long)(S.k0 + key0) * A.k.token + kvh * A.k.head;
        const uint8_t *from_v = global_at<const uint8_t>(A.v.at) + (long long)(S.k0 + key0) * A.v.token + kvh * A.v.head;
        k_part.template load<0, BN / L::GROUP_ROWS / W>(rows_buffer(from_k, A.k.token, S.n_k - key0, BN, A.dim), keys, wave);
        v_part.template load<0, BN / L::GROUP_ROWS / W>(rows_buffer(from_v, A.v.token, S.n_k - key0, BN, A.dim), values, wave);
    }

    const Rows<D> rows(lane);
    const Columns<D> columns(lane);
    v16f sums_k[E] = {}, sums_v[E] = {};
    auto step = [&](int n, uint8_t *queries, uint8_t *outs, float (&rows_of)[2][ROWS], uint8_t *next_queries, uint8_t *next_outs) RB_INLINE {
        if (wave == 0) {
            rows_of[0][lane] = next_lse * LOG2E - T::GRAD_BIAS;
            rows_of[1][lane] = next_delta;
        }
        loads_arrived();
        __syncthreads();
        if (n + 1 < steps) load(next_queries, next_outs);
        bool dirty = false;
        if (A.causal && block_last > ahead + t * ROWS) {      // some key of the workgroup is not seen by all rows
            look_through<T, D, ROWS, W>(queries, &found, tid);
            look_through<T, D, ROWS, W>(outs, &found, tid);
            __syncthreads();
            dirty = __builtin_amdgcn_readfirstlane(found) != 0;
        }
        const int row0 = t * ROWS + half * 32;
        if (++t == tile0 + tiles) t = tile0;
        const bool any = !A.causal || wave_first <= ahead + row0 + 31;
        v16f x = {}, y = {};
        if (any) {
            // both operands come from LDS
            constexpr int AHEAD = 3;
            auto right = [&](int i) RB_INLINE { return rows.read(i % 2 ? values : keys, part, i / 2); };
            v4u r[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) r[i] = right(i);
            stream_operands<D / 8, AHEAD>([&](int i) RB_INLINE { return rows.read(i % 2 ? outs : queries, half, i / 2); },
                                          [&](int i, v4u a) RB_INLINE {
                                              if (i % 2)
                                                  y = T::mfma(a, r[i % AHEAD], y);
                                              else
                                                  x = T::mfma(a, r[i % AHEAD], x);
                                              if (i + AHEAD < D / 8) r[i % AHEAD] = right(i + AHEAD);
                                          });
        }
        if (dirty) {      // everybody has the scores: what is read transposed is cleaned
            __syncthreads();
            make_finite<T, D, ROWS, W>(queries, &found, tid);
            make_finite<T, D, ROWS, W>(outs, &found, tid);
            __syncthreads();
        }
        if (!any) return;
        const bool masked = row0 + 32 > S.n_q || (A.causal && wave_last > ahead + row0);
        const int least = (A.causal ? my_key - ahead : 0) - row0 - 4 * h, beyond = S.n_q - row0 - 4 * h;      // the first row that sees this key; the end of the rows
        const int mine = half * 32 + 4 * h;
        uint32_t w[8], z[8];
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const v4f zero_at = *(const v4f *)&rows_of[0][mine + 2 * i], delta = *(const v4f *)&rows_of[1][mine + 2 * i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = i + j;
                x[r] = __builtin_amdgcn_exp2f(fmaf(x[r], A.c, -zero_at[j]));
                y[r] = x[r] * (y[r] - delta[j]) * held.unit;      // ds, from the dp that queries_kernel has, bit for bit
                if (masked && (8 * (r / 4) + r % 4 < least || 8 * (r / 4) + r % 4 >= beyond)) x[r] = y[r] = 0.f;
            }
            w[i / 2] = T::pack(x[i], x[i + 1]), w[i / 2 + 1] = T::pack(x[i + 2], x[i + 3]);
        }
        float moved;
        if (held.follow(y, moved))
#pragma unroll
            for (int e = 0; e < E; ++e) sums_k[e] *= moved;
#pragma unroll
        for (int i = 0; i < 16; i += 2) z[i / 2] = T::pack(y[i], y[i + 1]);
        const v4u pw[2] = {{w[0], w[1], w[2], w[3]}, {w[4], w[5], w[6], w[7]}}, dz[2] = {{z[0], z[1], z[2], z[3]}, {z[4], z[5], z[6], z[7]}};
        stream_operands<4 * E, 4>([&](int i) RB_INLINE { return columns.read(i % 2 ? queries : outs, i / 2 % E, 2 * half + i / (2 * E)); },
                                  [&](int i, v4u a) RB_INLINE {
                                      const int e = i / 2 % E, k = i / (2 * E);
                                      if (i % 2)
                                          sums_k[e] = T::mfma(a, dz[k], sums_k[e]);
                                      else
                                          sums_v[e] = T::mfma(a, pw[k], sums_v[e]);
                                  });
    };
    for (int n = 0; n < steps; n += 2) {
        step(n, queries_a, outs_a, rows_a, queries_b, outs_b);
        if (n + 1 < steps) step(n + 1, queries_b, outs_b, rows_b, queries_a, outs_a);
    }
    loads_arrived();      // (the values, where there are no rows)
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(found) && half == 0)      // (only the rows of tiles that were cleaned, and their keys see it)
        for (int g = first_g; g < first_g + heads_of; ++g)
            for (int r = tile0 * ROWS; r < min(S.n_q, (max(block_last - ahead, 0) + ROWS - 1) / ROWS * ROWS); ++r)
                add_not_finite<T, D>(sums_v, global_at<const uint8_t>(A.go) + (long long)(S.q0 + r) * A.o.token + (kvh * A.group + g) * A.o.head, A.dim, h, my_key <= ahead + r);

    uint8_t *const mine = part == 0 ? queries_a : part == 1 ? outs_a : part == 2 ? queries_b : outs_b;
    static_assert(E * 4096 <= L::bytes(ROWS), "sums of 32 keys");
    if constexpr (T::GRAD_BIAS)
#pragma unroll
        for (int e = 0; e < E; ++e) sums_k[e] *= held.inverse();      // (each half has a unit of its own)
    add_halves<E>(sums_v, mine, half, lane);
    add_halves<E>(sums_k, mine, half, lane);
    if (half == 1) return;
    const bool real = my_key < S.n_k;
    const long long at = (long long)(S.k0 + key) * A.kv_heads + kvh;
    const float scale_v = 1.f / (1 << T::GRAD_BIAS), scale_k = A.scale / (1 << T::GRAD_BIAS);
    if (A.splits > 1) {
        float *const k_part_at = part_at(A, split, 0, at), *const v_part_at = part_at(A, split, 1, at);
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int to = e * 32 + 2 * i + 4 * h;
                if (!real || to >= A.dim) continue;
                *(v4f *)(k_part_at + to) = (v4f){sums_k[e][i], sums_k[e][i + 1], sums_k[e][i + 2], sums_k[e][i + 3]} * scale_k;
                *(v4f *)(v_part_at + to) = (v4f){sums_v[e][i], sums_v[e][i + 1], sums_v[e][i + 2], sums_v[e][i + 3]} * scale_v;
            }
        return;
    }
    store_columns<T, D>(sums_v, scale_v, global_at<uint8_t>(A.dv) + at * (A.dim * 2), A.dim, h, real, false);
    store_columns<T, D>(sums_k, scale_k, global_at<uint8_t>(A.dk) + at * (A.dim * 2), A.dim, h, real, false);
}

// The splits' sums, one after the other, in fp32: four elements per thread.  Bound: latency, so four parts are on their way at once (four splits of 230 tokens: 4 us).
template <class T, int D> __global__ __launch_bounds__(256) void join_kernel(const GradArgs A)
{
    constexpr int COLUMNS = D / 4, KEYS = 256 / COLUMNS;
    const int lane = threadIdx.x & 63, kvh = blockIdx.x % A.kv_heads, e = threadIdx.x % COLUMNS * 4;
    const int *first_q = global_at<const int>(A.first_q), *first_k = global_at<const int>(A.first_k);
    int s, of_sequence;
    if (!keys_of_workgroup<BN>(first_q, first_k, A.n_seqs, A.ordered_keys, A.tokens_q, A.tokens_k, A.causal, blockIdx.x / A.kv_heads, lane, s, of_sequence)) return;
    const Sequence S = sequence_at(first_q, first_k, s, A.tokens_q, A.tokens_k);
    const int key0 = of_sequence * BN, key = key0 + blockIdx.y * KEYS + threadIdx.x / COLUMNS;
    if (key0 < 0 || key >= S.n_k || e >= A.dim) return;
    const long long at = (long long)(S.k0 + key) * A.kv_heads + kvh;
    v4f sums[2] = {};
    for (int split = 0; split < A.splits; split += 4) {
        v4f x[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int which = 0; which < 2; ++which) x[i][which] = split + i < A.splits ? *(const v4f *)(part_at(A, split + i, which, at) + e) : (v4f)(0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int which = 0; which < 2; ++which) sums[which] += x[i][which];
    }
#pragma unroll
    for (int which = 0; which < 2; ++which)
        *(v2u *)(global_at<uint8_t>(which ? A.dv : A.dk) + (at * A.dim + e) * 2) = (v2u){T::pack(sums[which][0], sums[which][1]), T::pack(sums[which][2], sums[which][3])};
}

// A workgroup has a compute unit to itself.  Where the keys are too few to give each one, the heads that share a key head are shared out as well (230 tokens of 8 query and
// 2 key heads of 96 33 -> 16.5 us and 4 for the join; 2000 tokens of 16 and 1 of 128 all kernels 937 -> 154 us).
int splits_for(long long blocks, int kv_heads, int group, int compute_units) { return (int)std::clamp(compute_units / std::max(blocks * kv_heads, 1ll), 1ll, (long long)group); }

// ---------------------------------------------------------------------- dq ---
// The same the other way round: 128 rows' q and do of one key head stay in LDS, keys and values go by, 64 at a time.  Eight wavefronts: four times 32 rows,
// by the first and the second 32 keys of a tile, whose sums are added at the end.  (The same sequences: 239 us, 0.72 PFLOP/s for four products.  Four wavefronts that keep q and do
// in registers, 32 keys at a time: 205 to 213 us there against 240, but 28 against 23.5 where a workgroup has a compute unit to itself, 512 tokens of 32 heads.)
template <class T, int D>
__global__ __launch_bounds__(512, 2) void queries_kernel(const GradArgs A)
{
    using L = Tile<D>;
    constexpr int W = 8, KEYS = 64, LOADS = Part<D, KEYS, W>::LOADS, E = D / 32;
    __shared__ __attribute__((aligned(16))) uint8_t keys_a[L::bytes(KEYS)], values_a[L::bytes(KEYS)], keys_b[L::bytes(KEYS)], values_b[L::bytes(KEYS)];
    __shared__ __attribute__((aligned(16))) uint8_t queries[L::bytes(BN)], outs[L::bytes(BN)];
    __shared__ float lacking_of[2][BN], rounded_of[2][BN];
    __shared__ int found;
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), part = wave & 3, half = wave >> 2;
    const int kvh = blockIdx.x % A.kv_heads;
    const int *first_q = global_at<const int>(A.first_q), *first_k = global_at<const int>(A.first_k);
    int s, of_sequence;
    if (!rows_of_workgroup<BN>(first_q, first_k, A.n_seqs, A.ordered, A.tokens_q, A.tokens_k, A.group, A.causal, blockIdx.x / A.kv_heads, gridDim.x / A.kv_heads, lane, s, of_sequence)) return;
    const Sequence S = sequence_at(first_q, first_k, s, A.tokens_q, A.tokens_k);
    const int row0 = of_sequence * BN, n_rows = S.n_q * A.group;
    if (row0 < 0 || row0 >= n_rows) return;

    const int my_row = row0 + part * 32 + (lane & 31);
    const int row = min(my_row, n_rows - 1), token = row / A.group, head = kvh * A.group + row % A.group;
    const int ahead = S.n_k - S.n_q;
    auto last_key = [&](int r) { return A.causal ? min(ahead + min(r, n_rows - 1) / A.group, S.n_k - 1) : S.n_k - 1; };
    const int limit = A.causal ? ahead + token : S.n_k - 1;
    const int block_least = last_key(row0), block_most = last_key(row0 + BN - 1);
    const int wave_least = __builtin_amdgcn_readfirstlane(last_key(row0 + part * 32)), wave_most = __builtin_amdgcn_readfirstlane(last_key(row0 + part * 32 + 31));
    const int n_tiles = __builtin_amdgcn_readfirstlane(max(block_most + 1, 0) + KEYS - 1) / KEYS;

    const Part<D, KEYS, W> k_part(A.k.token, A.dim, wave * (KEYS / W), lane), v_part(A.v.token, A.dim, wave * (KEYS / W), lane);
    const uint8_t *k_base = global_at<const uint8_t>(A.k.at) + S.k0 * A.k.token + kvh * A.k.head;
    const uint8_t *v_base = global_at<const uint8_t>(A.v.at) + S.k0 * A.v.token + kvh * A.v.head;
    auto load = [&](int t, uint8_t *keys, uint8_t *values) RB_INLINE {
        k_part.template load<0, LOADS>(rows_buffer(k_base + (long long)t * KEYS * A.k.token, A.k.token, S.n_k - t * KEYS, KEYS, A.dim), keys, wave);
        v_part.template load<0, LOADS>(rows_buffer(v_base + (long long)t * KEYS * A.v.token, A.v.token, S.n_k - t * KEYS, KEYS, A.dim), values, wave);
    };
    if (tid == 0) found = 0;
    if (n_tiles > 0) load(0, keys_a, values_a);

    const Rows<D> rows(lane);
    const Columns<D> columns(lane);
    const long long row_at = (long long)(S.q0 + token) * A.o.token + head * A.o.head;
    {
        const uint8_t *from_q = global_at<const uint8_t>(A.q.at) + (S.q0 + token) * A.q.token + head * A.q.head, *from_o = global_at<const uint8_t>(A.go) + row_at;
        if (half == 0)
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                rows.write(queries, part, k, k * 16 + h * 8 < A.dim ? *(const v4u *)(from_q + k * 32 + h * 16) : (v4u)(0u));
                rows.write(outs, part, k, k * 16 + h * 8 < A.dim ? *(const v4u *)(from_o + k * 32 + h * 16) : (v4u)(0u));
            }
    }
    const long long stat = (long long)(S.q0 + token) * A.heads + head;
    const float delta = global_at<const float>(A.delta)[stat], zero_at = global_at<const float>(A.lse)[stat] * LOG2E - T::GRAD_BIAS;
    Unit<T> held;
    float less = -delta * held.unit;

    v16f sums[E] = {}, means[E] = {};      // sum_j ds_ij k_j, sum_j p_ij k_j
    float lacking = 0.f, rounded = 0.f;    // sum_j ds_ij, and of them as the products have them, in the unit
    float first_dp = 0.f;                  // dp of the first key (h = 0)
    auto step = [&](int t, uint8_t *keys, uint8_t *values, uint8_t *next_keys, uint8_t *next_values) RB_INLINE {
        loads_arrived();
        meet();
        if (t + 1 < n_tiles) load(t + 1, next_keys, next_values);
        bool dirty = false;
        if (block_least < min(t * KEYS + KEYS, S.n_k) - 1) {      // some row of the workgroup does not see all of the tile's keys
            look_through<T, D, KEYS, W>(keys, &found, tid);
            meet();
            dirty = __builtin_amdgcn_readfirstlane(found) != 0;
        }
        const int key0 = t * KEYS + half * 32;
        const bool any = key0 <= wave_most;
        v16f x = {}, y = {};
        if (any) {
            constexpr int AHEAD = 3;
            auto right = [&](int i) RB_INLINE { return rows.read(i % 2 ? outs : queries, part, i / 2); };
            v4u r[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) r[i] = right(i);
            stream_operands<D / 8, AHEAD>([&](int i) RB_INLINE { return rows.read(i % 2 ? values : keys, half, i / 2); },
                                          [&](int i, v4u a) RB_INLINE {
                                              if (i % 2)
                                                  y = T::mfma(a, r[i % AHEAD], y);
                                              else
                                                  x = T::mfma(a, r[i % AHEAD], x);
                                              if (i + AHEAD < D / 8) r[i % AHEAD] = right(i + AHEAD);
                                          });
        }
        if (dirty) {      // everybody has the scores: what is read transposed is cleaned
            meet();
            make_finite<T, D, KEYS, W>(keys, &found, tid);
            meet();
        }
        if (!any) return;
        if (t == 0) first_dp = y[0];
        const bool masked = key0 + 31 > wave_least;
        const int seen = limit - key0 - 4 * h;
        uint32_t w[8], z[8];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            float p[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = i + j;
                p[j] = __builtin_amdgcn_exp2f(fmaf(x[r], A.c, -zero_at));
                y[r] = p[j] * fmaf(y[r], held.unit, less);      // ds
                if (masked && 8 * (r / 4) + r % 4 > seen) p[j] = y[r] = 0.f;
            }
            w[i / 2] = T::pack(p[0], p[1]);
        }
        float moved;
        if (held.follow(y, moved)) {
            less *= moved, lacking *= moved, rounded *= moved;
#pragma unroll
            for (int e = 0; e < E; ++e) sums[e] *= moved;
        }
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            lacking += y[i] + y[i + 1];
            z[i / 2] = T::pack(y[i], y[i + 1]);
            rounded = T::sum(z[i / 2], rounded);
        }
        const v4u pw[2] = {{w[0], w[1], w[2], w[3]}, {w[4], w[5], w[6], w[7]}}, dz[2] = {{z[0], z[1], z[2], z[3]}, {z[4], z[5], z[6], z[7]}};
        stream_operands<2 * E, 4>([&](int i) RB_INLINE { return columns.read(keys, i % E, 2 * half + i / E); },
                                  [&](int i, v4u a) RB_INLINE {
                                      sums[i % E] = T::mfma(a, dz[i / E], sums[i % E]);
                                      means[i % E] = T::mfma(a, pw[i / E], means[i % E]);
                                  });
    };
    for (int t = 0; t < n_tiles; t += 2) {
        step(t, keys_a, values_a, keys_b, values_b);
        if (t + 1 < n_tiles) step(t + 1, keys_b, values_b, keys_a, values_a);
    }
    const float outside = held.inverse();      // (each half has a unit of its own)
    lacking = over_halves_sum(lacking) / (1 << T::GRAD_BIAS) * outside;
    rounded = over_halves_sum(rounded) / (1 << T::GRAD_BIAS) * outside;
    const int in_block = part * 32 + (lane & 31);
    if (h == 0) lacking_of[half][in_block] = lacking, rounded_of[half][in_block] = rounded;
    __syncthreads();
    lacking = lacking_of[0][in_block] + lacking_of[1][in_block];
    rounded = rounded_of[0][in_block] + rounded_of[1][in_block];
#pragma unroll
    for (int e = 0; e < E; ++e) sums[e] = sums[e] * outside - means[e] * rounded;
    uint8_t *const mine = part == 0 ? keys_a : part == 1 ? keys_b : part == 2 ? values_a : values_b;
    static_assert(E * 4096 <= L::bytes(KEYS), "sums of 32 rows");
    if (!add_halves<E>(sums, mine, half, lane)) return;
    // A row that sees one key: its weight is one, dp = delta and ds = 0 by definition, whatever the rounding of scores, sums and lse left (times zero: NaN stays)
    const bool one = limit == 0;
    if (h == 0 && my_row < n_rows) global_at<float>(A.delta)[stat] = one ? first_dp : delta + lacking;
    store_columns<T, D>(sums, one ? 0.f : A.scale / (1 << T::GRAD_BIAS), global_at<uint8_t>(A.dq) + row_at, A.dim, h, my_row < n_rows, limit < 0);
}

template <class T, int D> int launch(GradArgs A, int compute_units, hipStream_t stream)
{
    const long long deltas = (long long)((A.tokens_q + 63) / 64) * A.heads;
    const long long keys = block_numbers(A.tokens_k, A.n_seqs, 1, BN) * A.kv_heads, queries = block_numbers(A.tokens_q, A.n_seqs, A.group, BN) * A.kv_heads;
    if (deltas > 0x7fffffffll || keys > 0x7fffffffll || queries > 0x7fffffffll || (long long)A.tokens_q * A.group > 0x7fff0000ll) return RB_ERR_SHAPE;
    A.splits = splits_for(block_numbers(A.tokens_k, A.n_seqs, 1, BN), A.kv_heads, A.group, compute_units);
    A.ordered = ordered_for(A.n_seqs, queries, compute_units), A.ordered_keys = ordered_for(A.n_seqs, keys * A.splits, compute_units);
    hipLaunchKernelGGL((delta_kernel<T>), dim3((unsigned)deltas), dim3(256), 0, stream, A);
    hipLaunchKernelGGL((queries_kernel<T, D>), dim3((unsigned)queries), dim3(512), 0, stream, A);
    hipLaunchKernelGGL((keys_kernel<T, D>), dim3((unsigned)keys, A.splits), dim3(512), 0, stream, A);
    if (A.splits > 1) hipLaunchKernelGGL((join_kernel<T, D>), dim3((unsigned)keys, BN * D / 1024), dim3(256), 0, stream, A);
    return hipGetLastError() == hipSuccess ? RB_OK : RB_ERR_HIP;
}

size_t rounded(size_t n) { return (n + 255) / 256 * 256; }
size_t delta_bytes(const rb_heads *H, int tokens_q) { return rounded((size_t)tokens_q * H->heads * 4); }
// What up to so many keys can need: for each number of splits, the most keys that have it.  (More sequences are not fewer blocks.)
size_t parts_bytes(const rb_heads *H, int tokens_k)
{
    const int units = rb::mx::device_groups(), group = H->heads / H->kv_heads;
    long long most = 0;
    for (long long splits = 2; splits <= std::min(group, units / H->kv_heads); ++splits) most = std::max(most, splits * std::min((long long)tokens_k, units / (splits * H->kv_heads) * BN));
    return (size_t)most * 2 * H->kv_heads * H->dim * 4;
}

}  // namespace
}  // namespace attn
}  // namespace rb

using namespace rb::attn;

extern "C" size_t rb_attn_grad_workspace_bytes(const rb_heads *H, int tokens_q, int tokens_k)
{
    if (check_heads(H) != RB_OK || tokens_q < 1 || tokens_k < 1) return 0;
    return delta_bytes(H, tokens_q) + parts_bytes(H, tokens_k);
}

extern "C" int rb_attn_prompt_grad(const rb_heads *H, const void *go, const void *q, const void *k, const void *v, const void *o, const float *lse, const int32_t *first_q,
                                   const int32_t *first_k, int n_seqs, int tokens_q, int tokens_k, int causal, float scale, void *dq, void *dk, void *dv, void *workspace,
                                   size_t workspace_bytes, void *stream)
{
    const int rc = check_heads(H);
    if (rc != RB_OK) return rc;
    if (!go || !q || !k || !v || !o || !lse || !first_q || !dq || !dk || !dv) return RB_ERR_NULL;
    if (n_seqs < 1 || n_seqs > MAX_SEQS || tokens_q < 1 || tokens_k < 1 || tokens_q > MAX_TOKENS || tokens_k > MAX_TOKENS || (!first_k && tokens_k != tokens_q)) return RB_ERR_SHAPE;
    if (check_scale(scale) != RB_OK) return RB_ERR_VALUE;
    for (const void *p : {go, q, k, v, o, (const void *)dq, (const void *)dk, (const void *)dv})
        if ((uintptr_t)p & 15) return RB_ERR_ALIGN;
    if (((uintptr_t)first_q | (uintptr_t)first_k | (uintptr_t)lse) & 3) return RB_ERR_ALIGN;
    if (workspace_bytes < rb_attn_grad_workspace_bytes(H, tokens_q, tokens_k) || !workspace) return RB_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 15) return RB_ERR_ALIGN;
    GradArgs A = {};
    A.q = side(q, H->q_token, H->q_head), A.k = side(k, H->k_token, H->k_head), A.v = side(v, H->v_token, H->v_head);
    A.o = side(o, (long long)H->heads * H->dim, H->dim);
    A.go = rb::address_of(go), A.lse = rb::address_of(lse), A.first_q = rb::address_of(first_q), A.first_k = rb::address_of(first_k ? first_k : first_q);
    A.delta = rb::address_of(workspace);
    A.parts = A.delta + delta_bytes(H, tokens_q);
    A.dq = rb::address_of(dq), A.dk = rb::address_of(dk), A.dv = rb::address_of(dv);
    A.n_seqs = n_seqs, A.tokens_q = tokens_q, A.tokens_k = tokens_k;
    A.heads = H->heads, A.kv_heads = H->kv_heads, A.group = H->heads / H->kv_heads, A.dim = H->dim, A.causal = causal != 0;
    A.c = scale * LOG2E, A.scale = scale;
    const int units = rb::mx::device_groups();
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (H->dtype == RB_F16) return A.dim <= 64 ? launch<F16, 64>(A, units, st) : launch<F16, 128>(A, units, st);
    return A.dim <= 64 ? launch<BF16, 64>(A, units, st) : launch<BF16, 128>(A, units, st);
}
