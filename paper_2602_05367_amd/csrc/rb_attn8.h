// Heads in 8 bits: e4m3 elements in units of a power of two per token and head, 2^(byte - 127).
#pragma once
#include <type_traits>

#include "rb_attn.h"

namespace rb {
namespace attn {

__device__ __forceinline__ float unit8(uint32_t exponent) { return __uint_as_float(exponent << 23); }      // (the conversions read a float's exponent alone)

// eight elements times a unit, each exact in fp32 and rounded once: exact in T too, but for fp16's last bits, below 2^-24, and what is beyond its largest number
template <class T> __device__ __forceinline__ v4u widen8(v2u w, float unit);
template <> __device__ __forceinline__ v4u widen8<F16>(v2u w, float unit)
{
    auto two = [&](uint32_t u, auto high) RB_INLINE { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u, unit, decltype(high)::value)); };
    return (v4u){two(w.x, std::false_type()), two(w.x, std::true_type()), two(w.y, std::false_type()), two(w.y, std::true_type())};
}
template <> __device__ __forceinline__ v4u widen8<BF16>(v2u w, float unit)
{
    auto two = [&](uint32_t u, auto high) RB_INLINE { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, unit, decltype(high)::value)); };
    return (v4u){two(w.x, std::false_type()), two(w.x, std::true_type()), two(w.y, std::false_type()), two(w.y, std::true_type())};
}

// The largest magnitude that is held: what rounds to a number of T again in e4m3's four bits
template <class T> constexpr float MOST8 = 0;
template <> inline constexpr float MOST8<F16> = 61440.f;
template <> inline constexpr float MOST8<BF16> = 0x1.ep+127f;
// |x| as far as it counts for the unit
template <class T> __device__ __forceinline__ float bounded8(float x)
{
    x = fabsf(x);
    return x < __builtin_inff() ? fminf(x, MOST8<T>) : 0.f;
}
// The byte of the unit that holds a head whose largest is `most`: most / unit in (224, 448]
__device__ __forceinline__ int exponent8(float most)
{
    const uint32_t bits = __float_as_uint(most);
    return max((int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u), 1);
}
template <class T> __device__ __forceinline__ uint32_t narrow8(const float (&x)[4], int exponent)
{
    const float per = __uint_as_float((uint32_t)(254 - exponent) << 23);
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = fabsf(x[i]) < __builtin_inff() ? fminf(fmaxf(x[i], -MOST8<T>), MOST8<T>) * per : __builtin_nanf("");
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
}

// 16 bytes per lane from a buffer to LDS, one lane's after the other's (a function of its own: inside of another, the host's compiler does not take the size).  Not kept by the caches: each
// byte is used once (48 sequences of 250000 positions together, the call: 111 us, kept 119)
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t from, uint8_t *to, uint32_t offset)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, (int)offset, 0, 0, 2);
}

// ROWS rows of a head on their way from a cache into a tile of T's, in registers: eight a load, which lie in one page.  Rows past the end of a buffer, and
// elements past a head's last, are zeros.
template <int D, int ROWS> struct Rows8 {
    using L = Tile<D>;
    static constexpr int LOADS = ROWS / 8, PIECE = D / 8;
    typedef std::conditional_t<D == 128, v4u, v2u> Piece;
    Piece w[LOADS];
    uint32_t exponent[LOADS];
    // where this lane's piece of eight rows lies
    static __device__ __forceinline__ uint32_t at(long long stride, int dim, int lane) { return lane % 8 * PIECE < dim ? (uint32_t)(lane / 8 * stride) + lane % 8 * PIECE : NOWHERE; }
    // load i: `rows` rows (of eight; <= 0: nothing) from `base` on, their exponents from `exponents` on
    __device__ __forceinline__ void load(int i, const uint8_t *base, const uint8_t *exponents, long long stride, int rows, int dim, uint32_t at, int lane)
    {
        rows = min(rows, 8);
        const __amdgpu_buffer_rsrc_t from = buffer(base, rows <= 0 ? 0u : (uint32_t)((rows - 1) * (int)stride + dim));
        if constexpr (D == 128)
            w[i] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(from, (int)at, 0, 0));
        else
            w[i] = __builtin_bit_cast(v2u, __builtin_amdgcn_raw_buffer_load_b64(from, (int)at, 0, 0));
        exponent[i] = __builtin_amdgcn_raw_buffer_load_b8(buffer(exponents, (uint32_t)max(rows, 0)), lane / 8, 0, 0);
    }
    // into rows first .. first + ROWS - 1 of a tile
    template <class T> __device__ __forceinline__ void write(uint8_t *tile, int first, int lane) const
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = lane / 8;      // the permutation is the same eight rows on
            uint8_t *to = tile + (first / 8 + i) * (8 / L::GROUP_ROWS * L::GROUP) + L::row_at(r) + ((lane % 8 * (PIECE / 8)) ^ L::spread(r)) * 16;
            const float unit = unit8(exponent[i]);
            *(lds_v4u *)(lds_byte *)to = widen8<T>((v2u){w[i].x, w[i].y}, unit);
            if constexpr (D == 128) *(lds_v4u *)(lds_byte *)(to + 16) = widen8<T>((v2u){w[i].z, w[i].w}, unit);
        }
    }
};

// four elements without the NaN among them
__device__ __forceinline__ uint32_t without_nan8(uint32_t w)
{
    const uint32_t sevens = (w & 0x7f7f7f7fu) + 0x01010101u;      // 0x80 in the bytes that are NaN
    return w & ~((sevens >> 7 & 0x01010101u) * 0xffu);
}

template <class T, int D>
__device__ __forceinline__ void add_not_finite8(v16f (&sums)[D / 32], const uint8_t *from, uint32_t exponent, int dim, int h, bool seen)
{
    const __amdgpu_buffer_rsrc_t row = buffer(from, dim);
    add_not_finite<T, D>(sums, seen, [&](int e) RB_INLINE {
        const v4u four = widen8<T>((v2u){__builtin_bit_cast(uint32_t, __builtin_amdgcn_raw_buffer_load_b32(row, h * 4, e, 0)), 0u}, unit8(exponent));
        return (v2u){four.x, four.y};
    });
}

}  // namespace attn
}  // namespace rb
