// The next token from logits, with temperature, top-k, top-p and min-p, drawn with a given random number.
//
// With w_j = exp((x_j - max) / T): what the filters leave is a prefix of the tokens in descending order, equal ones by their index.  Nothing is sorted.  A
// histogram over -log2 w, counts and weights, says in which of its bins the last token of that prefix lies; what lies in earlier bins is left for sure, and the few tokens of that
// bin are candidates, which are ranked among themselves.  The token is then found in the order of the indexes: sums over pieces of the row, and within the piece that u falls into.
//
// Weights are whole numbers of units, 2^-45 of the largest one, or coarser where all of a long row together would not fit 64 bits: sums depend on no order, so histograms may be summed by
// atomics, and the roundings of a row of up to 2^20 tokens are together below a step of u.  (Units of 2^-30, one word each: without filters 25 us in place of 27, with them the same; but a row's many tokens
// of 2^-31 each were then nothing, or twice what they are.)
//
// Bound: not by the row's bytes (256 rows of 128000 bf16 are 65 MB, 10 us), but by instructions and, with few rows, by the steps that follow each other.  A logit costs
// a subtraction, two products, an exponential and its rounding to units in the histogram and again in the sums: some 72 and 57 to 86 cycles per wavefront and element, 16 and 19 us of the 52
// that those rows take with top-p; reading them and their maximum are 9, the borders, the candidates and the choice 6.  (Weights do not fit the registers beside the logits, to be computed once.)
// Measured there: no filter 27 us, top-k of 50 22.6, top-p 52, all filters mixed 59, greedy 16.  One row of 32000 fp16: 11.7 us with top-k and top-p, 9.6 without, one launch: eight steps with
// barriers between them are all but 1.3 us.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <type_traits>

#include "rabit.h"
#include "rb_device.h"
#include "rb_internal.h"

namespace rb {
namespace sample {
namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64, PER_THREAD = 3, BINS = PER_THREAD * THREADS, BIN_BITS = 11, PIECES = 64, LISTED = 2 * THREADS;
static_assert(BINS >= 1 << BIN_BITS);
// (Three bins of -log2 w a thread are 0.015 wide.  With two, more lanes meet in one: 256 rows of 128000 bf16, top-p, 59 us in place of 52, 48 of 131071 fp32 43 in place of 39; four took the same time:
// what is saved among the lanes and candidates is spent on clearing and adding up)
constexpr float RANGE = 46.5f;      // -log2 of weights that round to nothing
typedef unsigned long long Weight;
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// word j of a tile's, j differing among lanes
__device__ __forceinline__ uint32_t word(v4u w, int j)
{
    const uint32_t lo = j & 1 ? w[1] : w[0], hi = j & 1 ? w[3] : w[2];
    return j & 2 ? hi : lo;
}
struct F16 {
    static constexpr int N = 8, SIZE = 2;      // elements of 16 bytes
    static __device__ __forceinline__ float at(v4u w, int i) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i / 2] >> i % 2 * 16)); }
    static __device__ __forceinline__ float any(v4u w, int i) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(word(w, i / 2) >> i % 2 * 16)); }
    static constexpr uint32_t NONE = 0x7e007e00u;      // NaN
    // 0 for plus infinity, NaN for all else
    static __device__ __forceinline__ uint32_t infinite(uint32_t w) { return ((w & 0xffffu) == 0x7c00u ? 0u : 0x7e00u) | (w >> 16 == 0x7c00u ? 0u : 0x7e000000u); }
};
struct BF16 {
    static constexpr int N = 8, SIZE = 2;
    static __device__ __forceinline__ float at(v4u w, int i) { return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); }
    static __device__ __forceinline__ float any(v4u w, int i) { return __uint_as_float(word(w, i / 2) >> i % 2 * 16 << 16); }
    static constexpr uint32_t NONE = 0x7fc07fc0u;
    static __device__ __forceinline__ uint32_t infinite(uint32_t w) { return ((w & 0xffffu) == 0x7f80u ? 0u : 0x7fc0u) | (w >> 16 == 0x7f80u ? 0u : 0x7fc00000u); }
};
struct F32 {
    static constexpr int N = 4, SIZE = 4;
    static __device__ __forceinline__ float at(v4u w, int i) { return __uint_as_float(w[i]); }
    static __device__ __forceinline__ float any(v4u w, int i) { return __uint_as_float(word(w, i)); }
    static constexpr uint32_t NONE = 0x7fc00000u;
    static __device__ __forceinline__ uint32_t infinite(uint32_t w) { return w == 0x7f800000u ? 0u : NONE; }
};

__device__ __forceinline__ float not_below(double x)
{
    const float f = (float)x;
    return f < x ? nextafterf(f, __builtin_inff()) : f;
}
// A token's place in the descending order as one number: larger comes first (0 and -0 are the same)
typedef unsigned long long Place;
constexpr int INDEX_BITS = 22, PLACE_BITS = 32 + INDEX_BITS, MAX_VOCAB = 1 << INDEX_BITS;
__device__ __forceinline__ Place place(float x, int index)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return (Place)(b ^ ((uint32_t)((int)b >> 31) | 0x80000000u)) << INDEX_BITS | (MAX_VOCAB - 1 - index);
}
__device__ __forceinline__ int index_of(Place p) { return MAX_VOCAB - 1 - (int)(p & (MAX_VOCAB - 1)); }

// What a row's weights come from.  (x - max) / T is taken from halves, which do not overflow, and times log2(e) / T in two parts: rounded once.
struct Scale {
    float half_max, hi, lo;
    int bits;      // the largest weight is 2^bits units: 2^45, or so many that all of a row, were they that large, fit 64 bits
    __device__ __forceinline__ void units_for(int vocab) { bits = min(32 + __builtin_clz(vocab), 45); }
    // -log2 of x's weight; a larger x never has a larger one.  (NaN stays NaN: none)
    __device__ __forceinline__ float below(float x) const
    {
        const float d = __builtin_fmaf(x, -0.5f, half_max);
        return __builtin_fmaf(d, hi, d * lo);
    }
    // The weight; zero for infinity and NaN
    static __device__ __forceinline__ float share(float below) { return fminf(fmaxf(__builtin_amdgcn_exp2f(-below), 0.f), 1.f); }
    // in units, to the nearest, ties to even: what is left in the lower bits of a number of 64 bits that has the unit as its last.  Nothing beyond RANGE
    __device__ __forceinline__ Weight weight(float below) const
    {
        const uint32_t high = (uint32_t)(1023 + 52 - bits) << 20;
        const Weight sum = __builtin_bit_cast(Weight, (double)share(below) + __builtin_bit_cast(double, (Weight)high << 32));
        return (Weight)((uint32_t)(sum >> 32) - high) << 32 | (uint32_t)sum;
    }
};
// The sum of N weights in units, each rounded as above: to the nearest 2^-23, as the lower bits of 1 + w, and what that leaves as those of a number whose last bit is the unit.
// (Four instructions of 32 bits a weight and no conversion.)
template <int N> struct SumOf {
    uint32_t upper = 0, lower = 0;
    static __device__ __forceinline__ float offset(const Scale &scale) { return __uint_as_float((uint32_t)(127 + 23 - scale.bits) << 23 | 0x400000u); }      // (a multiple of 2^-23)
    __device__ __forceinline__ void add(const Scale &scale, float below)
    {
        const float w = Scale::share(below), up = w + 1.f;
        upper += __float_as_uint(up);
        lower += __float_as_uint(w - (up - (1.f + offset(scale))));
    }
    __device__ __forceinline__ Weight units(const Scale &scale) const
    {
        return ((Weight)(upper - N * 0x3f800000u) << (scale.bits - 23)) + (Weight)(long long)(int)(lower - N * __float_as_uint(offset(scale)));
    }
};

// Sums over the lanes up to each, by data-parallel moves
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS> __device__ __forceinline__ Weight moved(Weight v) { return (Weight)moved<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 | moved<CTRL, ROWS>((uint32_t)v); }
template <class V> __device__ __forceinline__ V up_to_lane(V v)
{
    v += moved<0x111, 0xf>(v);      // one, two, four and eight lanes on within sixteen, then the last of the sixteen before, then of the 32
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);
    v += moved<0x143, 0xc>(v);
    return v;
}
// The largest of a wavefront's lanes, or of its sixteens, whose last lanes then have it
template <int CTRL, int ROWS> __device__ __forceinline__ float larger(float v)
{
    return fmaxf(v, __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)__float_as_uint(v), (int)__float_as_uint(v), CTRL, ROWS, 0xf, false)));
}
__device__ __forceinline__ float largest_of_sixteen(float v) { return larger<0x118, 0xf>(larger<0x114, 0xf>(larger<0x112, 0xf>(larger<0x111, 0xf>(v)))); }
__device__ __forceinline__ float largest_of_lanes(float v) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(larger<0x143, 0xc>(larger<0x142, 0xa>(largest_of_sixteen(v)))), 63)); }
__device__ __forceinline__ uint32_t of_lane(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ Weight of_lane(Weight v, int lane) { return (Weight)of_lane((uint32_t)(v >> 32), lane) << 32 | of_lane((uint32_t)v, lane); }

struct Candidate {
    Place place;
    Weight weight;      // with what it is a candidate for
};
struct Found {      // as it is met
    float x;
    int index;
};
constexpr Weight FOR_COUNT = 1ull << 62, FOR_WEIGHT = 1ull << 63, ONLY_WEIGHT = FOR_COUNT - 1;
// What several threads find out for all: each use has a place of its own, so one barrier is enough
enum Use { BOUND, BORDER, SECOND, FIRST, USES };
struct Reached {
    int bin;
    uint32_t count;      // before the bin, and
    Weight before, here; // weight before it and in it
};
struct Shared {
    Weight weights[BINS];
    uint32_t counts[BINS];
    Weight pieces[PIECES];
    Found found[LISTED];
    Candidate listed[LISTED];
    Weight wave_weights[USES][WAVES];
    uint32_t wave_counts[USES][WAVES];
    float wave_max[WAVES];
    double derived[2];      // see Given
    Reached reached[USES];
    uint32_t n_listed, n_candidates;
    Place found_place[2];
    Weight found_weight[2];
    bool differ;
    // what the threads' largest are counted in, where the list is to be
    __device__ __forceinline__ uint32_t *tops() { return (uint32_t *)listed; }
    // (before a list is used)
    __device__ __forceinline__ void begin_list(uint32_t n)
    {
        n_listed = n, n_candidates = 0;
        for (int i = 0; i < 2; ++i) found_place[i] = 0, found_weight[i] = 0;
        differ = false;
    }
};

// Of a workgroup's threads: sums up to each, and over all (there is a barrier inside)
template <class V> __device__ __forceinline__ V over_waves(V upto, const V *waves, int lane, int wave, V &all)
{
    const V sums = up_to_lane(lane < WAVES ? waves[lane] : (V)0);
    all = of_lane(sums, WAVES - 1);
    return wave ? upto + of_lane(sums, wave - 1) : upto;
}
__device__ __forceinline__ void up_to_thread(Shared &S, Use use, uint32_t &count, Weight &weight, uint32_t &all_counts, Weight &all_weights, int lane, int wave)
{
    count = up_to_lane(count), weight = up_to_lane(weight);
    if (lane == 63) S.wave_counts[use][wave] = count, S.wave_weights[use][wave] = weight;
    __syncthreads();
    count = over_waves(count, S.wave_counts[use], lane, wave, all_counts);
    weight = over_waves(weight, S.wave_weights[use], lane, wave, all_weights);
}

// A row is cut into `groups` parts, one for a workgroup where there are several, and each of those into PIECES / groups pieces, of whole tiles
struct Cut {
    int groups, tiles, of_group, per_piece;
    __host__ __device__ Cut(int groups_, int vocab, int tile)
        : groups(groups_), tiles((vocab + tile - 1) / tile), of_group((tiles + groups - 1) / groups), per_piece((of_group + PIECES / groups - 1) / (PIECES / groups))
    {
    }
    __device__ __forceinline__ int piece_of(int tile) const { return groups == 1 ? tile / per_piece : tile / of_group * (PIECES / groups) + tile % of_group / per_piece; }
    __device__ __forceinline__ void tiles_of(int piece, int &from, int &to) const
    {
        const int group = piece / (PIECES / groups);
        from = group * of_group + piece % (PIECES / groups) * per_piece;
        to = min(min(from + per_piece, (group + 1) * of_group), tiles);
    }
};

struct Args {
    Address logits, u, temperature, top_k, top_p, min_p, tokens;
    Address workspace;
    long long stride;      // in bytes
    int rows, vocab, groups;
};
constexpr float ALL_BINS = __builtin_inff();
// What a histogram says: tokens of bins before `sure` are left; for those of low .. high (the border of top-p) and of count_bin (that of top-k) it has to be seen
struct Bins {
    int sure = BINS, low = BINS, high = -1, count_bin = BINS;
    uint32_t count_before = 0;                           // tokens before count_bin, and
    Weight weight_before_count = 0, weight_before_low = 0, all = 0;      // weights; of all
    // the bins that matter end here
    __device__ __forceinline__ float end() const { return sure == BINS ? ALL_BINS : (float)(max(max(sure - 1, high), count_bin < BINS ? count_bin : -1) + 1); }
    __device__ __forceinline__ bool is_candidate(int bin) const { return bin == count_bin || (bin >= low && bin <= high); }
    __device__ __forceinline__ Weight candidate(int bin) const { return (bin == count_bin ? FOR_COUNT : 0) | (bin >= low && bin <= high ? FOR_WEIGHT : 0); }
};
static_assert(sizeof(Bins) <= 64, "a place of a row's");
// What the workgroups of a row hand on: for each row what they add up, for each part what it found
struct Parts {
    Weight *weights, *pieces;
    uint32_t *counts, *n_listed;
    Bins *bins;
    Found *found;
    float *maxima;
    double *derived;      // see Given
    static constexpr int LISTED_EACH = 512;
    static constexpr size_t ROW = BINS * 12 + PIECES * sizeof(Weight) + 64 + 16, PART = LISTED_EACH * sizeof(Found) + 8;      // bytes
    static constexpr size_t bytes(size_t rows, size_t parts) { return rows * ROW + parts * PART; }
    __device__ __forceinline__ Parts(Address workspace, size_t rows, size_t parts)
    {
        weights = global_at<Weight>(workspace);
        pieces = weights + rows * BINS;
        derived = (double *)(pieces + rows * PIECES);
        found = (Found *)(derived + 2 * rows);
        bins = (Bins *)(found + parts * LISTED_EACH);
        counts = (uint32_t *)((uint8_t *)bins + rows * 64);
        maxima = (float *)(counts + rows * BINS);
        n_listed = (uint32_t *)(maxima + parts);
    }
};

// One row's parameters, and what follows from them once its maximum is known
struct Given {
    float temperature, min_p, top_p, u;
    int top_k;
    __device__ __forceinline__ Given(const Args &A, int row)
        : temperature(A.temperature ? global_at<const float>(A.temperature)[row] : 1.f), min_p(A.min_p ? global_at<const float>(A.min_p)[row] : 0.f),
          top_p(A.top_p ? global_at<const float>(A.top_p)[row] : 1.f), u(global_at<const float>(A.u)[row]), top_k(A.top_k ? global_at<const int>(A.top_k)[row] : 0)
    {
    }
    __device__ __forceinline__ bool greedy() const { return !(temperature > 0.f); }
    // What takes a quotient and a logarithm in 64 bits, by one wavefront each while the row is on its way: 2 log2(e) / T, and T log(min_p), which is how far below the largest min_p's border lies
    __device__ __forceinline__ void derive(double *to, int wave) const
    {
        if (wave == WAVES - 1) to[0] = fmin(2 * 1.4426950408889634 / (greedy() ? 1.0 : (double)temperature), 0x1p+127);
        if (wave == WAVES - 2 && min_p > 0.f && min_p < 1.f) to[1] = (double)temperature * log((double)min_p);
    }
};
struct Row : Given {
    Scale scale;
    float least;      // no token below it is left (min-p; greedy: the largest alone)
    bool by_count, by_weight, infinite;      // filtered by top-k, by top-p; only logits of plus infinity are left, which count as 0 then
    __device__ __forceinline__ Row(const Given &G, const double *derived, int vocab, float most) : Given(G)
    {
        infinite = most == __builtin_inff();
        if (infinite) most = 0.f;
        const bool greedy = this->greedy();
        u = u >= 0.f && !greedy ? fminf(u, 0x1.fffffep-1f) : 0.f;
        by_count = !greedy && top_k >= 1 && top_k < vocab, by_weight = !greedy && top_p < 1.f;
        least = -0x1.fffffep+127f;
        if (greedy || min_p >= 1.f)
            least = most;
        else if (min_p > 0.f)      // w >= min_p: x >= max + T log(min_p), the smallest float that is
            least = fmaxf(least, not_below((double)most + derived[1]));
        const double c = derived[0];
        scale.units_for(vocab);
        scale.half_max = 0.5f * most;
        scale.hi = (float)c;
        if ((double)scale.hi > c) scale.hi = __uint_as_float(__float_as_uint(scale.hi) - 1u);      // (lo not below zero: where both parts overflow, so does their sum)
        scale.lo = (float)(c - (double)scale.hi);
    }
    // a token's bin is this one's whole part (within RANGE one of them, whatever it is rounded to)
    static __device__ __forceinline__ float bin_of(float below) { return below * ((BINS - 0.01f) / RANGE); }
};

// The tiles of a wavefront, 64 lanes times 16 bytes each: a workgroup's wavefronts have consecutive ones
template <class E> struct Tiles {
    static constexpr int TILE = 64 * E::N;
    const uint8_t *row;
    int vocab, from, to, lane;
    __device__ __forceinline__ Tiles(const Args &A, int number, int from_, int to_, int lane_)
        : row(global_at<const uint8_t>(A.logits) + number * A.stride), vocab(A.vocab), from(from_), to(to_), lane(lane_)
    {
    }
    static __device__ __forceinline__ Tiles of_wave(const Args &A, int number, const Cut &C, int group, int wave, int lane)
    {
        const int end = min((group + 1) * C.of_group, C.tiles), each = (C.of_group + WAVES - 1) / WAVES, from = min(group * C.of_group + wave * each, end);
        return Tiles(A, number, from, min(from + each, end), lane);
    }
    // A tile that the row fills, whatever lies there of another
    __device__ __forceinline__ v4u load(int tile) const
    {
        v4u w = (v4u)(E::NONE);
        if (vocab >= E::N) __builtin_memcpy(&w, row + (long long)min(tile * TILE + lane * E::N, vocab - E::N) * E::SIZE, 16);
        return w;
    }
    // The last tile of a row that does not fill it, NaN past its end
    __device__ __forceinline__ bool is_cut(int tile) const { return (tile + 1) * TILE > vocab; }
    __device__ __forceinline__ v4u load_cut(int tile) const
    {
        const int at = tile * TILE + lane * E::N;
        uint32_t e[E::N];
#pragma unroll
        for (int i = 0; i < E::N; ++i) {
            e[i] = E::NONE & (E::SIZE == 4 ? ~0u : 0xffffu);
            if (at + i < vocab) {
                if constexpr (E::SIZE == 4)
                    e[i] = *(const uint32_t *)(row + (long long)(at + i) * 4);
                else
                    e[i] = *(const uint16_t *)(row + (long long)(at + i) * 2);
            }
        }
        v4u w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = E::SIZE == 4 ? e[j] : e[2 * j % E::N] | e[(2 * j + 1) % E::N] << 16;
        return w;
    }
    static __device__ __forceinline__ v4u as_row_says(const Row &R, v4u w)
    {
        if (R.infinite) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = E::infinite(w[j]);
        }
        return w;
    }
};
template <class E> __device__ __forceinline__ float largest_of(v4u w)      // (NaN is passed over)
{
    float t = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < E::N; ++i) t = fmaxf(t, E::at(w, i));
    return t;
}

// Tiles kept in registers, or, HELD = 0, read anew each time, four at a time.  Held, the row is read once; read anew it comes from the L2 but waits for it each time (256 rows of 128000 bf16: top-k 22.6 and
// 28 us, top-p 52 and 58, no filter 27 and 29, greedy 16 and 24; of 65536 fp32, top-p, 38 and 48).  Sixteen tiles are what a wavefront of 128 registers has room for; longer rows are read anew (256 of 128000 fp32: no
// filter 49 us, top-p 79; of 152000 bf16 32 and 67).
template <class E, int HELD> struct Elements : Tiles<E> {
    // word j of each tile: one place of a vector, so that a loop over the tiles is one copy of its body (sixteen do not fit the instruction cache)
    typedef uint32_t Words __attribute__((ext_vector_type(HELD ? HELD : 1)));
    Words held[4];
    float top[HELD ? HELD / 2 : 1];      // of a lane's elements, the largest of each two tiles
    using Tiles<E>::from;
    using Tiles<E>::to;
    template <class Meanwhile> __device__ __forceinline__ Elements(const Tiles<E> &tiles, Meanwhile meanwhile) : Tiles<E>(tiles)
    {
        if constexpr (HELD != 0) {
            v4u w[HELD];
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (from + i < to) w[i] = this->load(from + i);
            meanwhile();
            if (from < to && this->is_cut(to - 1)) {
                const v4u last = this->load_cut(to - 1);
#pragma unroll
                for (int i = 0; i < HELD; ++i)
                    if (from + i == to - 1) w[i] = last;
            }
#pragma unroll
            for (int i = 0; i < HELD; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) held[j][i] = w[i][j];
#pragma unroll
            for (int i = 0; i < HELD; i += 2) {
                top[i / 2] = from + i < to ? largest_of<E>(w[i]) : -__builtin_inff();
                if (from + i + 1 < to) top[i / 2] = fmaxf(top[i / 2], largest_of<E>(w[i + 1]));
            }
        } else {
            meanwhile();
        }
    }
    template <class Use> __device__ __forceinline__ void each_tile(Use use) const
    {
        if constexpr (HELD != 0) {
#pragma unroll 1
            for (int i = 0; i < to - from; ++i) use(from + i, (v4u){held[0][i], held[1][i], held[2][i], held[3][i]});
        } else {
            const int end = from < to && this->is_cut(to - 1) ? to - 1 : to;
            for (int tile = from; tile < end; tile += 4) {
                v4u w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (tile + i < end) w[i] = this->load(tile + i);
#pragma unroll 1
                for (int i = 0; i < 4; ++i) {
                    if (tile + i < end) use(tile + i, w[0]);
                    w[0] = w[1], w[1] = w[2], w[2] = w[3];
                }
            }
            if (end < to) use(end, this->load_cut(end));
        }
    }
    // use(tile, its elements) for those that may have one in a bin before `end`
    template <class Use> __device__ __forceinline__ void each(const Row &R, float end, Use use) const
    {
        if constexpr (HELD != 0) {
            uint32_t skipped = 0;      // one bit for each two tiles
            if (end != ALL_BINS && !R.infinite) {
#pragma unroll
                for (int i = 0; i < HELD / 2; ++i) skipped |= __ballot(Row::bin_of(R.scale.below(top[i])) < end) ? 0u : 1u << i;
            }
            each_tile([&](int tile, v4u w) {
                if (!(skipped >> (tile - from) / 2 & 1)) use(tile, Tiles<E>::as_row_says(R, w));
            });
        } else {
            each_tile([&](int tile, v4u w) {
                w = Tiles<E>::as_row_says(R, w);
                if (end == ALL_BINS || __ballot(Row::bin_of(R.scale.below(largest_of<E>(w))) < end)) use(tile, w);
            });
        }
    }
    __device__ __forceinline__ float largest() const
    {
        float t = -__builtin_inff();
        if constexpr (HELD != 0) {
#pragma unroll
            for (int i = 0; i < HELD / 2; ++i) t = fmaxf(t, top[i]);
        } else {
            each_tile([&](int, v4u w) { t = fmaxf(t, largest_of<E>(w)); });
        }
        return t;
    }
};

__device__ __forceinline__ Weight shuffled(Weight w, int d) { return (Weight)__shfl_xor((uint32_t)(w >> 32), d) << 32 | (uint32_t)__shfl_xor((uint32_t)w, d); }
__device__ __forceinline__ float largest_of_workgroup(Shared &S, float t, int lane, int wave)
{
    static_assert(WAVES == 16);
    t = largest_of_lanes(t);
    if (lane == 0) S.wave_max[wave] = t;
    __syncthreads();
    return __uint_as_float(of_lane(__float_as_uint(largest_of_sixteen(S.wave_max[lane % WAVES])), 63));
}

__device__ __forceinline__ void clear_bins(Shared &S, int tid)
{
    for (int i = tid; i < BINS; i += THREADS) S.counts[i] = 0, S.weights[i] = 0;
    __syncthreads();
}
// What is counted and listed from zero on (a barrier has to follow)
__device__ __forceinline__ void clear_all(Shared &S, int tid)
{
    for (int i = tid; i < BINS; i += THREADS) S.counts[i] = 0, S.weights[i] = 0, S.tops()[i] = 0;
    if (tid < PIECES) S.pieces[tid] = 0;
    if (tid == 0) S.begin_list(0);
}
// The bins before `end`
template <class E, class Elements_> __device__ __forceinline__ void histogram(Shared &S, const Row &R, const Elements_ &elements, float end)
{
    elements.each(R, end, [&](int, v4u w) {
#pragma unroll
        for (int half = 0; half < E::N; half += 4) {
            float below[4];
            Weight weight[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) below[i] = R.scale.below(E::at(w, half + i));
#pragma unroll
            for (int i = 0; i < 4; ++i) weight[i] = R.scale.weight(below[i]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float at = Row::bin_of(below[i]);
                if (below[i] < RANGE && at < end) {
                    const int bin = (int)at;
                    if (R.by_count) atomicAdd(&S.counts[bin], 1u);
                    if (R.by_weight) atomicAdd(&S.weights[bin], weight[i]);
                }
            }
        }
    });
    __syncthreads();
}

// What a thread knows of the bins: its own, and the sums up to its last
struct Sums {
    uint32_t counts[PER_THREAD], upto_count = 0, all_count;
    Weight weights[PER_THREAD], upto_weight = 0, all_weight;
    __device__ __forceinline__ void add_up(Shared &S, Use use, int lane, int wave)
    {
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i) upto_count += counts[i], upto_weight += weights[i];
        up_to_thread(S, use, upto_count, upto_weight, all_count, all_weight, lane, wave);
    }
    // The bin in which the counts, or the weights, reach `target`, which all of them do: one thread says so
    __device__ __forceinline__ void say(Reached &to, bool by_count, Weight target, int tid) const
    {
        Reached r = {PER_THREAD * tid, upto_count, upto_weight, 0};
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i) r.count -= counts[i], r.before -= weights[i];
        if ((by_count ? r.count : r.before) >= target || (by_count ? upto_count : upto_weight) < target) return;
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i) {
            r.here = weights[i];
            if ((by_count ? r.count + counts[i] : r.before + weights[i]) >= target) break;
            r.count += counts[i], r.before += weights[i], ++r.bin;
        }
        to = r;
    }
};
__device__ __forceinline__ Sums sums_of(const Shared &S, int tid)
{
    Sums s;
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) s.counts[i] = S.counts[PER_THREAD * tid + i], s.weights[i] = S.weights[PER_THREAD * tid + i];
    return s;
}
// the weight at which the shortest prefix that has top_p of `all` ends: one token at least
__device__ __forceinline__ Weight target_of(float top_p, Weight all)
{
    const double wanted = ceil((double)top_p * (double)all);
    return wanted >= 1.0 ? min((Weight)wanted, all) : 1;
}

__device__ __forceinline__ Bins borders(Shared &S, const Row &R, Sums sums, int tid, int lane, int wave)
{
    Bins B;
    sums.add_up(S, BORDER, lane, wave);
    Weight least = B.all = sums.all_weight, most = B.all;      // what top-k leaves, whatever is left of its bin
    if (R.by_count && (uint32_t)R.top_k <= sums.all_count) {
        sums.say(S.reached[BORDER], true, (Weight)R.top_k, tid);
        __syncthreads();
        const Reached r = S.reached[BORDER];
        B.sure = B.count_bin = r.bin, B.count_before = r.count;
        least = B.weight_before_count = r.before, most = r.before + r.here;
    }
    if (R.by_weight) {
        const Weight low = target_of(R.top_p, least), high = target_of(R.top_p, most);
        sums.say(S.reached[SECOND], false, low, tid);
        if (high != low) sums.say(S.reached[BOUND], false, high, tid);
        __syncthreads();
        const Reached r = S.reached[SECOND];
        B.sure = B.low = min(r.bin, B.count_bin), B.weight_before_low = r.before;
        B.high = min(high != low ? S.reached[BOUND].bin : r.bin, B.count_bin);
    }
    return B;
}
// The first bins that top-k can reach into: every token of the first top_k is in them, since so many threads have one there.
// largest: of this thread's tokens.
__device__ __forceinline__ float bins_of_top_k(Shared &S, const Row &R, float largest, int tid, int lane, int wave)
{
    if (!R.by_count || R.top_k > THREADS / 2) return ALL_BINS;
    const float below = R.scale.below(!R.infinite ? largest : largest == __builtin_inff() ? 0.f : __builtin_nanf(""));
    uint32_t *const tops = S.tops(), k = (uint32_t)R.top_k;
    if (below < RANGE) atomicAdd(&tops[(int)Row::bin_of(below)], 1u);
    __syncthreads();
    static_assert(BINS * sizeof(uint32_t) <= sizeof(S.listed));
    uint32_t own[PER_THREAD], here = 0;
#pragma unroll
    for (int i = 0; i < PER_THREAD; ++i) here += own[i] = tops[PER_THREAD * tid + i];
    const uint32_t upto_lane = up_to_lane(here);
    if (lane == 63) S.wave_counts[BOUND][wave] = upto_lane;
    __syncthreads();
    uint32_t all;
    const uint32_t upto = over_waves(upto_lane, S.wave_counts[BOUND], lane, wave, all);
    uint32_t before = upto - here;
    if (all < k) return ALL_BINS;
    if (before < k && upto >= k) {
        int reached = PER_THREAD * tid;
#pragma unroll
        for (int i = 0; i < PER_THREAD - 1; ++i) reached += (before += own[i]) < k;
        S.reached[FIRST].bin = reached;
    }
    __syncthreads();
    const int bin = S.reached[FIRST].bin;
    return bin < BINS - 1 ? (float)(bin + 1) : ALL_BINS;
}

// All tokens of bins before `end` into the list, as far as there is room; their histogram.  False: they are more
template <class E, class Elements_> __device__ __forceinline__ bool gather(Shared &S, const Row &R, const Elements_ &elements, float end, int lane)
{
    elements.each(R, end, [&](int tile, v4u w) {
        uint32_t found = 0;      // one bit for each
#pragma unroll
        for (int i = 0; i < E::N; ++i) found |= Row::bin_of(R.scale.below(E::at(w, i))) < end ? 1u << i : 0u;
        while (__ballot(found)) {
            if (found) {
                const int i = __builtin_ctz(found);
                found &= found - 1;
                const float x = E::any(w, i), below = R.scale.below(x);
                const int bin = (int)Row::bin_of(below);
                const uint32_t n = atomicAdd(&S.n_listed, 1u);
                if (n < LISTED) S.found[n] = {x, (tile * 64 + lane) * E::N + i};
                atomicAdd(&S.counts[bin], 1u);
                atomicAdd(&S.weights[bin], R.scale.weight(below));
            }
        }
    });
    __syncthreads();
    return S.n_listed <= LISTED;
}

// A wavefront's sums by pieces, its tiles in their order: the lanes' are added up once a piece
struct PieceSums {
    Shared &S;
    const Cut &C;
    int lane, piece, next;      // the piece at hand, the tile where it ends
    Weight sum = 0;
    __device__ __forceinline__ PieceSums(Shared &S_, const Cut &C_, int from, int lane_) : S(S_), C(C_), lane(lane_), piece(C_.piece_of(from))
    {
        int first;
        C.tiles_of(piece, first, next);
    }
    __device__ __forceinline__ void add(int tile, Weight w)
    {
        if (tile >= next) {
            end();
            piece = C.piece_of(tile);
            int first;
            C.tiles_of(piece, first, next);
        }
        sum += w;
    }
    __device__ __forceinline__ void end()
    {
        if (__ballot(sum != 0)) {
            sum = up_to_lane(sum);
            if (lane == 63) atomicAdd(&S.pieces[piece], sum);
        }
        sum = 0;
    }
};

// Weights of the tokens that are left for sure, by pieces of the row; candidates into the list, as far as there is room.  Without min-p (!MIN_P) no logit is compared with its border (256 rows of 128000 bf16, no filter, 27 us for 28)
template <class E, bool MIN_P, class Elements_> __device__ __forceinline__ void collect(Shared &S, const Row &R, const Bins &B, const Cut &C, const Elements_ &elements, int lane)
{
    const float sure = B.sure == BINS ? ALL_BINS : (float)B.sure, below_least = R.scale.below(R.least);
    // (without candidates, min-p's border ends it as well)
    const float end = B.sure < BINS ? B.end() : below_least < RANGE ? floorf(Row::bin_of(below_least)) + 1.f : ALL_BINS;
    // (bins between the two borders, if there are any, have none)
    const bool all_candidates = B.count_bin == BINS || B.low == BINS || B.count_bin <= B.high + 1;
    PieceSums sums(S, C, elements.from, lane);
    if (B.sure == BINS) {      // no filter but min-p's
        elements.each(R, end, [&](int tile, v4u w) {
            SumOf<E::N> sum;
#pragma unroll
            for (int i = 0; i < E::N; ++i) {
                const float x = E::at(w, i), below = R.scale.below(x);
                sum.add(R.scale, !MIN_P || x >= R.least ? below : __builtin_inff());
            }
            sums.add(tile, sum.units(R.scale));
        });
    } else {
        elements.each(R, end, [&](int tile, v4u w) {
            SumOf<E::N> sum;
            bool any = false;
#pragma unroll
            for (int half = 0; half < E::N; half += 4) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = E::at(w, half + i), below = R.scale.below(x), at = Row::bin_of(below);
                    any |= at < end && !(at < sure);
                    sum.add(R.scale, at < sure && (!MIN_P || x >= R.least) ? below : __builtin_inff());
                }
            }
            uint32_t candidates = 0;      // one bit for each
            if (__ballot(any)) {
#pragma unroll
                for (int i = 0; i < E::N; ++i) {
                    const float at = Row::bin_of(R.scale.below(E::at(w, i)));
                    candidates |= at >= sure && at < end ? 1u << i : 0u;
                }
            }
            while (__ballot(candidates)) {      // (also those that min-p does not leave: they count for top-k and top-p)
                if (candidates) {
                    const int i = __builtin_ctz(candidates);
                    candidates &= candidates - 1;
                    const float x = E::any(w, i);
                    if (all_candidates || B.is_candidate((int)Row::bin_of(R.scale.below(x)))) {
                        const uint32_t n = atomicAdd(&S.n_listed, 1u);
                        if (n < LISTED) S.found[n] = {x, (tile * 64 + lane) * E::N + i};
                    }
                }
            }
            sums.add(tile, sum.units(R.scale));
        });
    }
    sums.end();
    __syncthreads();
}

template <class E, class Elements_> __device__ __forceinline__ void collect(Shared &S, const Row &R, const Bins &B, const Cut &C, const Elements_ &elements, int lane)
{
    if (R.least > -0x1.fffffep+127f)
        collect<E, true>(S, R, B, C, elements, lane);
    else
        collect<E, false>(S, R, B, C, elements, lane);
}

// Among the candidates: the first one, in their order, with which top-k, and of those before it, with which top-p is reached.  How many are before a candidate, and their weights, need
// neither border; consecutive lanes share a candidate's comparisons.
__device__ __forceinline__ Place resolve(Shared &S, const Row &R, const Bins &B, int n, int tid, int lane)
{
    const bool by_count = B.count_bin < BINS, by_weight = R.by_weight, both = by_count && by_weight;
    bool same = false;      // equal logits, which only the index orders, and of one bin, so candidates for the same: worth looking where they are many
    if (n > 64) {
        const Candidate first = S.listed[0];
        for (int i = tid; i < n; i += THREADS)
            if (S.listed[i].place >> INDEX_BITS != first.place >> INDEX_BITS) S.differ = true;
        __syncthreads();
        same = !S.differ;
    }
    const int shift = n > 1 ? max(10 - (32 - __builtin_clz(n - 1)), 0) : 4, sharing = 1 << min(shift, 4);
    static_assert(LISTED == 2 * THREADS && THREADS == 1 << 10);
    Candidate mine[2] = {};
    uint32_t rank[2] = {};
    Weight before_count[2] = {}, before_weight[2] = {};      // weights of those before it: candidates for top-k, for top-p
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int i = tid / sharing + r * (THREADS / sharing);
        if (i >= n) break;
        mine[r] = S.listed[i];
        if (same) {
#pragma unroll 4
            for (int j = lane & (sharing - 1); j < n; j += sharing) rank[r] += (uint32_t)S.listed[j].place > (uint32_t)mine[r].place;
        } else if (both) {
#pragma unroll 4
            for (int j = lane & (sharing - 1); j < n; j += sharing) {
                const Candidate c = S.listed[j];
                const bool ahead = c.place > mine[r].place, counts = ahead && (c.weight & FOR_COUNT), weighs = ahead && (c.weight & FOR_WEIGHT);
                rank[r] += counts;
                before_count[r] += counts ? c.weight & ONLY_WEIGHT : 0;
                before_weight[r] += weighs ? c.weight & ONLY_WEIGHT : 0;
            }
        } else {
#pragma unroll 4
            for (int j = lane & (sharing - 1); j < n; j += sharing) {
                const Candidate c = S.listed[j];
                const bool ahead = c.place > mine[r].place;
                rank[r] += ahead;
                before_weight[r] += ahead ? c.weight & ONLY_WEIGHT : 0;
            }
        }
        for (int d = 1; d < sharing; d <<= 1) {
            rank[r] += __shfl_xor(rank[r], d);
            if (!same) before_weight[r] += shuffled(before_weight[r], d);
            if (both && !same) before_count[r] += shuffled(before_count[r], d);
        }
        if (same) before_weight[r] = rank[r] * (mine[r].weight & ONLY_WEIGHT);
        if (!both || same) before_count[r] = before_weight[r];
    }
    Place border = 0;
    Weight left = B.all;
    if (by_count) {
        const uint32_t last = (uint32_t)R.top_k - B.count_before - 1;
#pragma unroll
        for (int r = 0; r < 2; ++r)
            if ((mine[r].weight & FOR_COUNT) && rank[r] == last) S.found_place[0] = mine[r].place, S.found_weight[0] = before_count[r] + (mine[r].weight & ONLY_WEIGHT);
        __syncthreads();
        border = S.found_place[0], left = B.weight_before_count + S.found_weight[0];
    }
    if (by_weight) {
        const Weight target = target_of(R.top_p, left) - B.weight_before_low;
#pragma unroll
        for (int r = 0; r < 2; ++r)
            if ((mine[r].weight & FOR_WEIGHT) && before_weight[r] < target && before_weight[r] + (mine[r].weight & ONLY_WEIGHT) >= target) S.found_place[1] = mine[r].place;
        __syncthreads();
        border = max(border, S.found_place[1]);
    }
    return border;
}

// The same among all tokens, by their places' bits, a histogram of some at a time: where the candidates are more than the list holds (thousands of equal logits).
// Behind `least` none counts.
template <class E, class Elements_>
__device__ __forceinline__ Place resolve_all(Shared &S, const Row &R, const Elements_ &elements, bool by_count, Weight target, Place least, Weight &weight, int tid, int lane, int wave)
{
    Place prefix = 0;
    weight = 0;
    Weight count = 0;
    for (int left = PLACE_BITS; left > 0;) {
        const int bits = min(left, BIN_BITS);
        left -= bits;
        clear_bins(S, tid);
        elements.each(R, ALL_BINS, [&](int tile, v4u w) {
#pragma unroll 1
            for (int i = 0; i < E::N; ++i) {
                const float x = E::at(w, i), below = R.scale.below(x);
                const Place p = place(x, (tile * 64 + lane) * E::N + i);
                if (below < RANGE && p >= least && p >> (left + bits) == prefix) {
                    const int bin = (int)((1u << bits) - 1 - (uint32_t)(p >> left & ((1u << bits) - 1)));      // from the largest down
                    atomicAdd(&S.counts[bin], 1u);
                    atomicAdd(&S.weights[bin], R.scale.weight(below));
                }
            }
        });
        __syncthreads();
        Sums sums = sums_of(S, tid);
        sums.add_up(S, BORDER, lane, wave);
        if ((by_count ? sums.all_count : sums.all_weight) < target - (by_count ? count : weight)) return 0;      // (never: top-k's and top-p's are reached)
        sums.say(S.reached[BORDER], by_count, target - (by_count ? count : weight), tid);
        __syncthreads();
        const Reached r = S.reached[BORDER];
        count += r.count, weight += r.before;
        prefix = prefix << bits | (Place)((1u << bits) - 1 - r.bin);
        if (left == 0) weight += r.here;
    }
    return prefix;
}

// The border: the last token that top-k and top-p leave (0: they leave all).  Candidates that are left join the pieces.
template <class E> __device__ __forceinline__ Place settle(Shared &S, const Args &A, int row, const Row &R, const Bins &B, const Cut &C, int tid, int lane, int wave)
{
    if (B.count_bin == BINS && B.low == BINS) return 0;
    Place border = 0;
    if (S.n_listed <= LISTED) {
        // candidates into a list of their own; of the rest, which only a list of all that top-k can leave has, what lies before both borders is left
        for (int i = tid; i < (int)S.n_listed; i += THREADS) {
            const Found f = S.found[i];
            const float below = R.scale.below(f.x);
            const int bin = (int)Row::bin_of(below);
            const Weight what_for = B.candidate(bin);
            if (what_for)
                S.listed[atomicAdd(&S.n_candidates, 1u)] = {place(f.x, f.index), R.scale.weight(below) | what_for};
            else if (bin < B.sure && f.x >= R.least)
                atomicAdd(&S.pieces[C.piece_of(f.index / Tiles<E>::TILE)], R.scale.weight(below));
        }
        __syncthreads();
        const int n = (int)S.n_candidates;
        border = resolve(S, R, B, n, tid, lane);
        for (int i = tid; i < n; i += THREADS) {      // (a candidate of top-k alone lies behind top-p's border, or there is none)
            const Candidate c = S.listed[i];
            if (c.place >= border && c.place >= place(R.least, MAX_VOCAB - 1)) atomicAdd(&S.pieces[C.piece_of(index_of(c.place) / Tiles<E>::TILE)], c.weight & ONLY_WEIGHT);
        }
    } else {
        const Elements<E, 0> elements(Tiles<E>::of_wave(A, row, Cut(1, A.vocab, Tiles<E>::TILE), 0, wave, lane), [] {});      // (the whole row)
        Weight weight, left = B.all;
        if (B.count_bin < BINS) border = resolve_all<E>(S, R, elements, true, (Weight)R.top_k, 0, left, tid, lane, wave);
        if (R.by_weight) border = max(border, resolve_all<E>(S, R, elements, false, target_of(R.top_p, left), border, weight, tid, lane, wave));
        if (tid < PIECES) S.pieces[tid] = 0;
        __syncthreads();
        PieceSums sums(S, C, elements.from, lane);
        elements.each(R, ALL_BINS, [&](int tile, v4u w) {
            Weight sum = 0;
#pragma unroll 1
            for (int i = 0; i < E::N; ++i) {
                const float x = E::at(w, i), below = R.scale.below(x);
                if (x >= R.least && place(x, (tile * 64 + lane) * E::N + i) >= border) sum += R.scale.weight(below);
            }
            sums.add(tile, sum);
        });
        sums.end();
    }
    __syncthreads();
    return border;
}

// The token: the piece that u falls into, a tile of it per wavefront, the elements of the lanes
template <class E> __device__ __forceinline__ void pick(Shared &S, const Args &A, int row, const Row &R, Place border, const Cut &C, int lane, int wave)
{
    static_assert(PIECES == 64, "one per lane");
    const Weight mine = S.pieces[lane], upto = up_to_lane(mine), total = of_lane(upto, 63);
    const Weight target = min((Weight)((double)R.u * (double)total), total - 1);
    const int piece = __builtin_ctzll(__ballot(upto > target));
    Weight before = of_lane(upto - mine, piece);
    int from, to;
    C.tiles_of(piece, from, to);
    const Tiles<E> tiles(A, row, from, to, lane);
    for (; from < to; from += WAVES) {
        const int tile = from + wave, at = (tile * 64 + lane) * E::N;
        v4u w = (v4u)(E::NONE);
        if (tile < to) w = Tiles<E>::as_row_says(R, tiles.is_cut(tile) ? tiles.load_cut(tile) : tiles.load(tile));
        Weight own[E::N];
        Weight sum = 0;
#pragma unroll
        for (int i = 0; i < E::N; ++i) {
            const float x = E::at(w, i);
            own[i] = x >= R.least && place(x, at + i) >= border ? R.scale.weight(R.scale.below(x)) : 0;
            sum += own[i];
        }
        Weight upto_lane = up_to_lane(sum), all;
        __syncthreads();
        if (lane == 63) S.wave_weights[FIRST][wave] = upto_lane;
        __syncthreads();
        upto_lane = before + over_waves(upto_lane, S.wave_weights[FIRST], lane, wave, all);
        if (upto_lane > target && upto_lane - sum <= target) {
            Weight upto_i = upto_lane - sum;
            int i = 0;
#pragma unroll
            for (int j = 0; j < E::N; ++j) {
                upto_i += own[j];
                i += upto_i <= target;
            }
            global_at<int>(A.tokens)[row] = at + i;
        }
        before += all;
        if (before > target) return;
    }
}

// One workgroup does a row
template <class E, int HELD> __global__ __launch_bounds__(THREADS) void row_kernel(const Args A)
{
    __shared__ Shared S;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = blockIdx.x;
    const Cut C(1, A.vocab, Tiles<E>::TILE);
    const Given G(A, row);
    const Elements<E, HELD> elements(Tiles<E>::of_wave(A, row, C, 0, wave, lane), [&] {
        G.derive(S.derived, wave);
        clear_all(S, tid);
    });
    const float largest = elements.largest(), most = largest_of_workgroup(S, largest, lane, wave);
    if (most == -__builtin_inff()) {      // nothing that may be drawn
        if (tid == 0) global_at<int>(A.tokens)[row] = -1;
        return;
    }
    const Row R(G, S.derived, A.vocab, most);
    Bins B;
    bool listed = false;
    if (R.by_count || R.by_weight) {
        // top-k: the tokens that can be among the first are few, and all that follows is done with those
        const float end = bins_of_top_k(S, R, largest, tid, lane, wave);
        if (end != ALL_BINS) {
            listed = gather<E>(S, R, elements, end, lane);
            if (!listed) {      // more than are listed
                __syncthreads();
                clear_all(S, tid);
                __syncthreads();
            }
        }
        if (!listed) histogram<E>(S, R, elements, end);
        B = borders(S, R, sums_of(S, tid), tid, lane, wave);
    }
    if (!listed) collect<E>(S, R, B, C, elements, lane);
    const Place border = settle<E>(S, A, row, R, B, C, tid, lane, wave);
    pick<E>(S, A, row, R, border, C, lane, wave);
}

// Several workgroups do a row (48 rows of 131071 fp32 with top-p: 39 to 41 us, one workgroup each 56; one row 25 and 53), in four launches: its maximum; the histogram, which they add up in memory; what is left for sure and the candidates; the border and the
// token.  What they hand on lies in the workspace.
enum Step { MAXIMUM, HISTOGRAM, COLLECT };
__device__ __forceinline__ float largest_of_row(const Parts &P, size_t first, int groups, int lane)
{
    float t = lane < groups ? P.maxima[first + lane] : -__builtin_inff();
    return largest_of_lanes(t);
}
template <class E, Step STEP, int HELD> __global__ __launch_bounds__(THREADS) void part_kernel(const Args A)
{
    __shared__ Shared S;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = blockIdx.x / A.groups, group = blockIdx.x % A.groups;
    const Cut C(A.groups, A.vocab, Tiles<E>::TILE);
    const Given G(A, row);
    const Parts P(A.workspace, (size_t)A.rows, (size_t)A.rows * A.groups);
    const size_t first = (size_t)row * A.groups, mine = first + group, bins = (size_t)row * BINS;
    const Elements<E, HELD> elements(Tiles<E>::of_wave(A, row, C, group, wave, lane), [&] {
        if constexpr (STEP == MAXIMUM) {
            if (group == 0) G.derive(P.derived + 2 * row, wave);
        } else {
            clear_all(S, tid);
        }
    });
    if constexpr (STEP == MAXIMUM) {
        for (int i = group * THREADS + tid; i < BINS; i += A.groups * THREADS) P.counts[bins + i] = 0, P.weights[bins + i] = 0;
        const float most = largest_of_workgroup(S, elements.largest(), lane, wave);
        if (tid == 0) P.maxima[mine] = most;
    } else {
        const float most = largest_of_row(P, first, A.groups, lane);
        if (most == -__builtin_inff()) return;
        __syncthreads();
        const Row R(G, P.derived + 2 * row, A.vocab, most);
        const bool filtered = R.by_count || R.by_weight;
        if constexpr (STEP == HISTOGRAM) {
            if (!filtered) return;
            histogram<E>(S, R, elements, ALL_BINS);
            for (int i = tid; i < BINS; i += THREADS) {
                if (S.counts[i]) atomicAdd(&P.counts[bins + i], S.counts[i]);
                if (S.weights[i]) atomicAdd(&P.weights[bins + i], S.weights[i]);
            }
        } else {
            Bins B;
            if (filtered) {
                Sums sums;
#pragma unroll
                for (int i = 0; i < PER_THREAD; ++i) sums.counts[i] = P.counts[bins + PER_THREAD * tid + i], sums.weights[i] = P.weights[bins + PER_THREAD * tid + i];
                B = borders(S, R, sums, tid, lane, wave);
                if (group == 0 && tid == 0) P.bins[row] = B;
            }
            collect<E>(S, R, B, C, elements, lane);
            const int pieces = PIECES / A.groups, n = (int)S.n_listed;
            if (tid < pieces) P.pieces[(size_t)row * PIECES + group * pieces + tid] = S.pieces[group * pieces + tid];
            for (int i = tid; i < min(n, Parts::LISTED_EACH); i += THREADS) P.found[mine * Parts::LISTED_EACH + i] = S.found[i];
            if (tid == 0) P.n_listed[mine] = n;
        }
    }
}
template <class E> __global__ __launch_bounds__(THREADS) void token_kernel(const Args A)
{
    __shared__ Shared S;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = blockIdx.x;
    const Given G(A, row);
    const Parts P(A.workspace, (size_t)A.rows, (size_t)A.rows * A.groups);
    const size_t first = (size_t)row * A.groups;
    if (tid < PIECES) S.pieces[tid] = P.pieces[(size_t)row * PIECES + tid];
    Bins B = P.bins[row];
    const float most = largest_of_row(P, first, A.groups, lane);
    if (most == -__builtin_inff()) {      // nothing that may be drawn
        if (tid == 0) global_at<int>(A.tokens)[row] = -1;
        return;
    }
    const Row R(G, P.derived + 2 * row, A.vocab, most);
    const Cut C(A.groups, A.vocab, Tiles<E>::TILE);
    if (R.by_count || R.by_weight) {
        // the parts' candidates one after the other; one that has more than its room: as if they were too many
        const uint32_t has = lane < A.groups ? P.n_listed[first + lane] : 0, upto = up_to_lane(has > Parts::LISTED_EACH ? (uint32_t)LISTED + 1 : has), n = of_lane(upto, 63);
        if (tid == 0) S.begin_list(n);
        if (n <= LISTED) {
            for (int g = wave; g < A.groups; g += WAVES) {
                const int count = of_lane(has, g), to = of_lane(upto, g) - count;
                for (int i = lane; i < count; i += 64) S.found[to + i] = P.found[(first + g) * Parts::LISTED_EACH + i];
            }
        }
    } else {
        B = Bins();
    }
    __syncthreads();
    const Place border = settle<E>(S, A, row, R, B, C, tid, lane, wave);
    pick<E>(S, A, row, R, border, C, lane, wave);
}

constexpr int MAX_ROWS = 1 << 20;
constexpr long long MAX_STRIDE = 1ll << 40;

// Workgroups of a row: powers of two, as many as there are compute units for, of SHARE logits at least (one row of 128000 bf16, top-p: 24.9 us with 4096, 24.0 with 2048, 26.7 with 8192; four of 151936
// fp32 25.9, 26.9 and 26.4); one, where that is a launch in place of four and has 8 tiles a wavefront at most (64 rows of 32000 fp32, top-k and top-p: 12.9 us, four launches 28.6; 7 rows
// of 50001 bf16, no filter: 13.9 and 15.0.  From there on several are faster: 128000 bf16 with top-p 24.9 us, one workgroup 43.9, no filter 14.8 and 18.9)
constexpr int SHARE = 4096, MOST_GROUPS = 64, SINGLE = 8 * WAVES;
int compute_units() { return std::max(mx::device_groups(), 2); }
int groups_of(int rows, int tiles, int tile, int compute_units)
{
    int groups = 1;
    if (tiles <= SINGLE) return 1;
    while (groups < MOST_GROUPS && 2ll * groups * rows <= compute_units && (long long)tiles * tile >= 2ll * groups * SHARE) groups *= 2;
    return groups;
}

template <class E, int HELD> void launch_parts(const Args &A, hipStream_t stream)
{
    const dim3 parts((unsigned)(A.rows * A.groups)), threads(THREADS);
    hipLaunchKernelGGL((part_kernel<E, MAXIMUM, HELD>), parts, threads, 0, stream, A);
    if (A.top_k || A.top_p) hipLaunchKernelGGL((part_kernel<E, HISTOGRAM, HELD>), parts, threads, 0, stream, A);
    hipLaunchKernelGGL((part_kernel<E, COLLECT, HELD>), parts, threads, 0, stream, A);
}
template <class E> int launch(Args A, hipStream_t stream)
{
    const int tiles = (A.vocab + Tiles<E>::TILE - 1) / Tiles<E>::TILE;
    const dim3 rows((unsigned)A.rows), threads(THREADS);
    // With top-k alone a row's few tokens are found by one workgroup before several have met, if no row has more than 512 of them: one row of 128000 bf16, the first 50: 14.5 us, with sixteen
    // workgroups 22.1; 300: 19.5 and 22.5; 1000, for which every bin counts, 36.3 and 23.0.  48 rows of 131071 fp32: 22.6 and 32.6; 27.7 and 33.9; 46.7 and 34.5.  One row of 200000 fp32: 25.0 and 21.7
    A.groups = A.top_k && !A.top_p && tiles <= 32 * WAVES ? 1 : groups_of(A.rows, tiles, Tiles<E>::TILE, compute_units());
    if (A.groups > 1) {
        const int of_group = (tiles + A.groups - 1) / A.groups;
        if (of_group <= 4 * WAVES)
            launch_parts<E, 4>(A, stream);
        else if (of_group <= 16 * WAVES)
            launch_parts<E, 16>(A, stream);
        else
            launch_parts<E, 0>(A, stream);
        hipLaunchKernelGGL((token_kernel<E>), rows, threads, 0, stream, A);
    } else if (tiles <= 4 * WAVES) {
        hipLaunchKernelGGL((row_kernel<E, 4>), rows, threads, 0, stream, A);
    } else if (tiles <= 16 * WAVES) {
        hipLaunchKernelGGL((row_kernel<E, 16>), rows, threads, 0, stream, A);
    } else {
        hipLaunchKernelGGL((row_kernel<E, 0>), rows, threads, 0, stream, A);
    }
    return hipGetLastError() == hipSuccess ? RB_OK : RB_ERR_HIP;
}

}  // namespace
}  // namespace sample
}  // namespace rb

using namespace rb::sample;

extern "C" size_t rb_sample_workspace_bytes(int dtype, int rows, int vocab)
{
    if ((dtype != RB_F16 && dtype != RB_BF16 && dtype != RB_F32) || rows < 1 || rows > MAX_ROWS || vocab < 1 || vocab > MAX_VOCAB) return 0;
    const int tile = 64 * (dtype == RB_F32 ? F32::N : F16::N), tiles = (vocab + tile - 1) / tile, units = compute_units();
    // whatever fewer rows take: no more parts than compute units, of rows that have two at least
    return groups_of(1, tiles, tile, units) > 1 ? Parts::bytes(units / 2, units) : 0;
}

extern "C" int rb_sample(const void *logits, int dtype, long long stride, int rows, int vocab, const float *u, const float *temperature, const int32_t *top_k,
                         const float *top_p, const float *min_p, int32_t *tokens, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!logits || !u || !tokens) return RB_ERR_NULL;
    if (dtype != RB_F16 && dtype != RB_BF16 && dtype != RB_F32) return RB_ERR_UNSUPPORTED;
    if (rows < 1 || rows > MAX_ROWS || vocab < 1 || vocab > MAX_VOCAB || stride < vocab || stride >= MAX_STRIDE) return RB_ERR_SHAPE;
    const int size = dtype == RB_F32 ? 4 : 2;
    if ((uintptr_t)logits % size != 0 || (((uintptr_t)u | (uintptr_t)temperature | (uintptr_t)top_k | (uintptr_t)top_p | (uintptr_t)min_p | (uintptr_t)tokens) & 3)) return RB_ERR_ALIGN;
    if (workspace_bytes < rb_sample_workspace_bytes(dtype, rows, vocab) || (workspace_bytes && !workspace)) return RB_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 15) return RB_ERR_ALIGN;
    Args A = {};
    A.logits = rb::address_of(logits), A.u = rb::address_of(u), A.temperature = rb::address_of(temperature), A.top_k = rb::address_of(top_k);
    A.top_p = rb::address_of(top_p), A.min_p = rb::address_of(min_p), A.tokens = rb::address_of(tokens), A.workspace = rb::address_of(workspace);
    A.stride = stride * size, A.rows = rows, A.vocab = vocab;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == RB_F16 ? launch<F16>(A, st) : dtype == RB_BF16 ? launch<BF16>(A, st) : launch<F32>(A, st);
}
