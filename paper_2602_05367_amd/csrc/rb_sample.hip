// The next token from logits, with temperature, top-k, top-p and min-p, drawn with a given random number.
//
// With w_j = exp((x_j - max) / T): what is left after the filters is a prefix of the tokens in descending order, all above some border t and the first `ties` of those equal to it.  A
// histogram of the logits below the maximum, counts and weights, says in which of its bins a border lies, what is above it, and the bin's few logits are then ranked
// among themselves: nothing is sorted.  The token is found in the order of the indexes: sums per piece of the row, then within the one that u falls into.
//
// Weights are whole numbers of units of 2^-38, in 64 bits: their sums depend on no order, so histograms may be summed by atomics.
#include <hip/hip_runtime.h>

#include "rabit.h"
#include "rb_device.h"

namespace rb {
namespace sample {
namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64, BINS = 2 * THREADS, PIECES = 64, LISTED = THREADS;
constexpr float RANGE = 39.f;      // -log2 of the weights that round to nothing
typedef unsigned long long Weight;

struct Args {
    Address logits, u, temperature, top_k, top_p, min_p, tokens;
    long long stride;      // in bytes
    int rows, vocab;
};

struct F16 {
    static constexpr int N = 8, SIZE = 2;      // elements of 16 bytes
    static __device__ __forceinline__ float at(const uint32_t *w, int i) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i / 2] >> i % 2 * 16)); }
};
struct BF16 {
    static constexpr int N = 8, SIZE = 2;
    static __device__ __forceinline__ float at(const uint32_t *w, int i) { return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); }
};
struct F32 {
    static constexpr int N = 4, SIZE = 4;
    static __device__ __forceinline__ float at(const uint32_t *w, int i) { return __uint_as_float(w[i]); }
};

__device__ __forceinline__ float not_below(double x)
{
    const float f = (float)x;
    return f < x ? nextafterf(f, __builtin_inff()) : f;
}
// Floats in their order as whole numbers (0 and -0 have to be the same already)
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = __float_as_uint(x);
    return b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float(o ^ (o & 0x80000000u ? 0x80000000u : 0xffffffffu)); }

// What a row's weights come from.  (x - max) / T is taken from halves, which do not overflow, and times log2(e) / T in two parts: rounded once.
struct Scale {
    float half_max, most, hi, lo;
    // -log2 of x's weight; a larger x never has a larger one
    __device__ __forceinline__ float below(float x) const
    {
        const float d = x == most ? 0.f : __builtin_fmaf(x, -0.5f, half_max);
        return __builtin_fmaf(d, hi, d * lo);
    }
    static __device__ __forceinline__ Weight weight(float below)
    {
        // 2^14 + w in 64 bits: its last bits are those of w in units of 2^-38
        constexpr double ONE = 16384.0;
        return below < RANGE ? __builtin_bit_cast(Weight, (double)__builtin_amdgcn_exp2f(-below) + ONE) - __builtin_bit_cast(Weight, ONE) : 0;
    }
    __device__ __forceinline__ Weight of(float x) const { return weight(below(x)); }
};

__device__ __forceinline__ Weight shuffle_up(Weight v, int d)
{
    return (Weight)__shfl_up((uint32_t)(v >> 32), d) << 32 | __shfl_up((uint32_t)v, d);
}
template <class V> __device__ __forceinline__ V up_to_lane(V v, int lane)
{
    for (int d = 1; d < 64; d <<= 1) {
        V u;
        if constexpr (sizeof(V) == 8)
            u = shuffle_up(v, d);
        else
            u = __shfl_up(v, d);
        if (lane >= d) v += u;
    }
    return v;
}
__device__ __forceinline__ Weight of_lane(Weight v, int lane)
{
    return (Weight)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// One border: `target` counts (top-k) or weight (top-p) are reached among the logits equal to x; more of them and of weight lie above
struct Border {
    float x;
    int above, equal;
    Weight weight_above;
};

// A workgroup does a row.  Its wavefronts have consecutive parts of it, and 16 bytes per lane at a time.
template <class E> __global__ __launch_bounds__(THREADS) void sample_kernel(const Args A)
{
    __shared__ uint32_t counts[BINS];
    __shared__ Weight weights[BINS];
    __shared__ uint32_t piece_ties[WAVES * PIECES];
    __shared__ Weight piece_weights[WAVES * PIECES];
    __shared__ uint32_t listed[LISTED];
    __shared__ Weight listed_weights[LISTED];
    __shared__ uint32_t wave_counts[WAVES], n_listed;
    __shared__ Weight wave_weights[WAVES];
    __shared__ float wave_max[WAVES];
    __shared__ Border found;
    __shared__ int found_bin;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = blockIdx.x;
    const uint8_t *logits = global_at<const uint8_t>(A.logits) + row * A.stride;
    constexpr int TILE = 64 * E::N;      // elements of a wavefront's step
    const int tiles = (A.vocab + TILE - 1) / TILE, each = (tiles + WAVES - 1) / WAVES, from_tile = min(wave * each, tiles), to_tile = min(from_tile + each, tiles);

    // a lane's elements of a tile; NaN past the row's end
    auto load = [&](int tile, float (&x)[E::N]) {
        const int at = tile * TILE + lane * E::N;
        uint32_t w[4] = {};
        if (at + E::N <= A.vocab) {
            __builtin_memcpy(w, logits + (long long)at * E::SIZE, 16);
#pragma unroll
            for (int i = 0; i < E::N; ++i) x[i] = E::at(w, i) + 0.f;      // (0 for -0)
        } else {
#pragma unroll
            for (int i = 0; i < E::N; ++i) {
                x[i] = __builtin_nanf("");
                if (at + i < A.vocab) {
                    uint32_t one[4] = {};
                    __builtin_memcpy(one, logits + (long long)(at + i) * E::SIZE, E::SIZE);
                    x[i] = E::at(one, 0) + 0.f;
                }
            }
        }
    };
    auto for_all = [&](auto use) {
        for (int tile = from_tile; tile < to_tile; ++tile) {
            float x[E::N];
            load(tile, x);
#pragma unroll
            for (int i = 0; i < E::N; ++i) use(x[i]);
        }
    };

    float most = -__builtin_inff();
    for_all([&](float x) { most = fmaxf(most, x); });      // (NaN is passed over)
    for (int d = 1; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
    if (lane == 0) wave_max[wave] = most;
    __syncthreads();
    most = wave_max[lane % WAVES];
    for (int d = 1; d < WAVES; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));
    if (most == -__builtin_inff()) {      // nothing that may be drawn
        if (tid == 0) global_at<int>(A.tokens)[row] = -1;
        return;
    }

    const float temperature = A.temperature ? global_at<const float>(A.temperature)[row] : 1.f, min_p = A.min_p ? global_at<const float>(A.min_p)[row] : 0.f;
    float top_p = A.top_p ? global_at<const float>(A.top_p)[row] : 1.f, u = global_at<const float>(A.u)[row];
    int top_k = A.top_k ? global_at<const int>(A.top_k)[row] : 0;
    const bool greedy = !(temperature > 0.f);
    if (top_k < 1 || top_k > A.vocab) top_k = A.vocab;
    if (!(top_p < 1.f)) top_p = 1.f;
    u = u >= 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
    const double c = 2 * 1.4426950408889634 / (greedy ? 1.0 : (double)temperature);
    Scale scale;
    scale.most = most, scale.half_max = 0.5f * most;
    scale.hi = (float)fmin(c, 0x1p+127), scale.lo = (float)(fmin(c, 0x1p+127) - (double)scale.hi);

    // What is left: above `border`, and the first `ties` of those equal to it
    float border = -__builtin_inff();
    int ties = 0;
    if (greedy) {
        border = most, ties = 1;
    } else {
        if (min_p > 0.f) {      // w >= min_p: x >= max + T log(min_p), the smallest float that is
            border = min_p < 1.f ? fmaxf(not_below((double)most + (double)temperature * log((double)min_p)), -0x1.fffffep+127f) : most;
            ties = 0x7fffffff;
        }
        if (top_k < A.vocab || top_p < 1.f) {
            for (int i = tid; i < BINS; i += THREADS) counts[i] = 0, weights[i] = 0;
            __syncthreads();
            auto bin_of = [&](float below) { return min((int)(below * (BINS / RANGE)), BINS - 1); };
            for_all([&](float x) {
                const float below = scale.below(x);
                if (x > -__builtin_inff() && below < RANGE) {
                    atomicAdd(&counts[bin_of(below)], 1u);
                    atomicAdd(&weights[bin_of(below)], Scale::weight(below));
                }
            });
            __syncthreads();
            // what lies before each bin: two bins a thread
            const uint32_t c0 = counts[2 * tid], c1 = counts[2 * tid + 1];
            const Weight w0 = weights[2 * tid], w1 = weights[2 * tid + 1];
            uint32_t upto_c = up_to_lane(c0 + c1, lane);
            Weight upto_w = up_to_lane(w0 + w1, lane);
            if (lane == 63) wave_counts[wave] = upto_c, wave_weights[wave] = upto_w;
            __syncthreads();
            const uint32_t sum_c = up_to_lane(lane < WAVES ? wave_counts[lane] : 0u, lane);
            const Weight sum_w = up_to_lane(lane < WAVES ? wave_weights[lane] : (Weight)0, lane);
            if (wave) upto_c += __builtin_amdgcn_readlane(sum_c, wave - 1), upto_w += of_lane(sum_w, wave - 1);
            const uint32_t all_c = __builtin_amdgcn_readlane(sum_c, WAVES - 1);
            const Weight all_w = of_lane(sum_w, WAVES - 1);

            // The border at which `target` (counts or weight) is reached; there is one
            auto find = [&](bool by_count, Weight target) -> Border {
                auto reached = [&](uint32_t count, Weight weight) { return (by_count ? (Weight)count : weight) >= target; };
                __syncthreads();
                if (tid == 0) n_listed = 0;
                if (reached(upto_c, upto_w) && !reached(upto_c - c1 - c0, upto_w - w1 - w0)) {
                    const bool second = !reached(upto_c - c1, upto_w - w1);
                    found_bin = 2 * tid + second;
                    found.above = upto_c - c1 - (second ? 0 : c0), found.weight_above = upto_w - w1 - (second ? 0 : w0);
                    found.equal = second ? c1 : c0;
                }
                __syncthreads();
                const int bin = found_bin, n = found.equal;
                Border b = found;
                __syncthreads();
                if (n <= LISTED) {      // the bin's logits, each ranked among them
                    for_all([&](float x) {
                        const float below = scale.below(x);
                        if (x > -__builtin_inff() && below < RANGE && bin_of(below) == bin) {
                            const uint32_t at = atomicAdd(&n_listed, 1u);
                            listed[at] = ordered(x);
                            listed_weights[at] = Scale::weight(below);
                        }
                    });
                    __syncthreads();
                    if (tid < n) {
                        const uint32_t mine = listed[tid];
                        int above = b.above, equal = 0;
                        Weight weight_above = b.weight_above;
                        for (int i = 0; i < n; ++i) {
                            const uint32_t o = listed[i];
                            above += o > mine, equal += o == mine;
                            weight_above += o > mine ? listed_weights[i] : 0;
                        }
                        if (!reached(above, weight_above) && reached(above + equal, weight_above + equal * listed_weights[tid])) {
                            found.x = from_ordered(mine);
                            found.above = above, found.equal = equal, found.weight_above = weight_above;
                        }
                    }
                } else {      // by their bits, eleven at a time: those that have the `prefix` found so far
                    uint32_t prefix = 0;
                    for (int shift = 21, bits = 11; shift >= 0; bits = min(shift, 11), shift -= max(bits, 1)) {
                        for (int i = tid; i < BINS; i += THREADS) counts[i] = 0, weights[i] = 0;
                        __syncthreads();
                        for_all([&](float x) {
                            const float below = scale.below(x);
                            const uint32_t o = ordered(x);
                            if (x > -__builtin_inff() && below < RANGE && bin_of(below) == bin && (shift + bits == 32 || o >> (shift + bits) == prefix)) {
                                atomicAdd(&counts[o >> shift & ((1u << bits) - 1)], 1u);
                                atomicAdd(&weights[o >> shift & ((1u << bits) - 1)], Scale::weight(below));
                            }
                        });
                        __syncthreads();
                        if (tid == 0) {
                            int i = (1 << bits) - 1;      // from the largest down
                            for (; i > 0 && !reached(b.above + counts[i], b.weight_above + weights[i]); --i) b.above += counts[i], b.weight_above += weights[i];
                            found = b, found.equal = counts[i], found_bin = i;
                        }
                        __syncthreads();
                        b = found;
                        prefix = prefix << bits | (uint32_t)found_bin;
                        __syncthreads();
                        if (shift == 0) break;
                    }
                    if (tid == 0) found.x = from_ordered(prefix);
                }
                __syncthreads();
                b = found;
                return b;
            };
            auto tighten = [&](float x, int n) {
                if (x > border)
                    border = x, ties = n;
                else if (x == border)
                    ties = min(ties, n);
            };
            Weight kept = all_w;
            if ((uint32_t)top_k < all_c) {
                const Border b = find(true, (Weight)top_k);
                tighten(b.x, top_k - b.above);
                kept = b.weight_above + (Weight)(top_k - b.above) * scale.of(b.x);
            }
            if (top_p < 1.f) {
                const double wanted = ceil((double)top_p * (double)kept);
                const Weight target = wanted >= 1.0 ? min((Weight)wanted, kept) : 1;
                const Border b = find(false, target);
                const Weight one = max(scale.of(b.x), (Weight)1);
                tighten(b.x, (int)min((target - b.weight_above + one - 1) / one, (Weight)0x7fffffff));
            }
        }
    }

    // sums over pieces of the row, in its order
    const int per_piece = (each + PIECES - 1) / PIECES;      // tiles
    for (int i = tid; i < WAVES * PIECES; i += THREADS) piece_ties[i] = 0, piece_weights[i] = 0;
    __syncthreads();
    for (int tile = from_tile; tile < to_tile; ++tile) {
        float x[E::N];
        load(tile, x);
        Weight sum = 0;
        uint32_t equal = 0;
#pragma unroll
        for (int i = 0; i < E::N; ++i) {
            if (x[i] > border) sum += scale.of(x[i]);
            equal += x[i] == border;
        }
        const int piece = wave * PIECES + (tile - from_tile) / per_piece;
        if (sum) atomicAdd(&piece_weights[piece], sum);
        if (equal) atomicAdd(&piece_ties[piece], equal);
    }
    __syncthreads();
    const Weight tie = border > -__builtin_inff() ? scale.of(border) : 0;
    // a wavefront's pieces, one per lane; then the wavefronts
    uint32_t upto_ties = up_to_lane(piece_ties[tid], lane);
    if (lane == 63) wave_counts[wave] = upto_ties;
    __syncthreads();
    const uint32_t ties_of_waves = up_to_lane(lane < WAVES ? wave_counts[lane] : 0u, lane);
    if (wave) upto_ties += __builtin_amdgcn_readlane(ties_of_waves, wave - 1);
    auto kept_ties = [&](uint32_t before, uint32_t n) { return (Weight)(min(before + n, (uint32_t)ties) - min(before, (uint32_t)ties)); };
    const uint32_t ties_before = upto_ties - piece_ties[tid];
    const Weight mine = piece_weights[tid] + kept_ties(ties_before, piece_ties[tid]) * tie;
    Weight upto = up_to_lane(mine, lane);
    if (lane == 63) wave_weights[wave] = upto;
    __syncthreads();
    const Weight sum_of_waves = up_to_lane(lane < WAVES ? wave_weights[lane] : (Weight)0, lane);
    if (wave) upto += of_lane(sum_of_waves, wave - 1);
    const Weight total = of_lane(sum_of_waves, WAVES - 1);
    const Weight target = min((Weight)((double)u * (double)total), total - 1);
    const unsigned long long here = __ballot(upto > target && upto - mine <= target);
    if (!here) return;

    // this wavefront has the piece: its tiles, then the lanes' elements
    const int piece = __builtin_ctzll(here);
    Weight before = of_lane(upto - mine, piece);
    uint32_t equal_before = __builtin_amdgcn_readlane(ties_before, piece);
    for (int tile = from_tile + piece * per_piece; tile < min(from_tile + (piece + 1) * per_piece, to_tile); ++tile) {
        float x[E::N];
        load(tile, x);
        uint32_t equal = 0;
#pragma unroll
        for (int i = 0; i < E::N; ++i) equal += x[i] == border;
        const uint32_t upto_equal = up_to_lane(equal, lane);
        uint32_t rank = equal_before + upto_equal - equal;
        Weight w[E::N], sum = 0;
#pragma unroll
        for (int i = 0; i < E::N; ++i) {
            w[i] = x[i] > border ? scale.of(x[i]) : x[i] == border && rank < (uint32_t)ties ? tie : 0;
            rank += x[i] == border;
            sum += w[i];
        }
        const Weight upto_lane = before + up_to_lane(sum, lane);
        const unsigned long long lanes = __ballot(upto_lane > target);
        if (lanes) {
            if (lane == __builtin_ctzll(lanes)) {
                Weight at = upto_lane - sum;
                int i = 0;
#pragma unroll
                for (int j = 0; j < E::N; ++j) {
                    at += w[j];
                    i += at <= target;
                }
                global_at<int>(A.tokens)[row] = tile * TILE + lane * E::N + i;
            }
            return;
        }
        before = of_lane(upto_lane, 63);
        equal_before += __builtin_amdgcn_readlane(upto_equal, 63);
    }
}

constexpr int MAX_ROWS = 1 << 20, MAX_VOCAB = 1 << 22;
constexpr long long MAX_STRIDE = 1ll << 40;

}  // namespace
}  // namespace sample
}  // namespace rb

using namespace rb::sample;

extern "C" int rb_sample(const void *logits, int dtype, long long stride, int rows, int vocab, const float *u, const float *temperature, const int32_t *top_k,
                         const float *top_p, const float *min_p, int32_t *tokens, void *stream)
{
    if (!logits || !u || !tokens) return RB_ERR_NULL;
    if (dtype != RB_F16 && dtype != RB_BF16 && dtype != RB_F32) return RB_ERR_UNSUPPORTED;
    if (rows < 1 || rows > MAX_ROWS || vocab < 1 || vocab > MAX_VOCAB || stride < vocab || stride >= MAX_STRIDE) return RB_ERR_SHAPE;
    const int size = dtype == RB_F32 ? 4 : 2;
    if ((uintptr_t)logits % size != 0 || (((uintptr_t)u | (uintptr_t)temperature | (uintptr_t)top_k | (uintptr_t)top_p | (uintptr_t)min_p | (uintptr_t)tokens) & 3)) return RB_ERR_ALIGN;
    const Args A = {rb::address_of(logits), rb::address_of(u), rb::address_of(temperature), rb::address_of(top_k), rb::address_of(top_p), rb::address_of(min_p),
                    rb::address_of(tokens), stride * size, rows, vocab};
    const dim3 grid((unsigned)rows), threads(THREADS);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == RB_F16)
        hipLaunchKernelGGL((sample_kernel<F16>), grid, threads, 0, st, A);
    else if (dtype == RB_BF16)
        hipLaunchKernelGGL((sample_kernel<BF16>), grid, threads, 0, st, A);
    else
        hipLaunchKernelGGL((sample_kernel<F32>), grid, threads, 0, st, A);
    return hipGetLastError() == hipSuccess ? RB_OK : RB_ERR_HIP;
}
