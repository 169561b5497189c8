// Microscaled formats: blocks of 32 numbers along a row share a power of two (block and scale as in
// the OCP Microscaling Formats Specification v1.0); the elements are int8 (whole numbers, |q| <= 127),
// e4m3 or e2m1.  With a the block's largest magnitude and k = floor(log2 a), one more where the
// significand a / 2^k is at least `over` (a would round past the largest element),
//     shared byte  S = clamp(k - emax + 127, 0, 254)     255 where the block is not finite
//     element      round to nearest even (x 2^(127-S)), codes 0 where S = 255
//     value        element 2^(S-127)                     NaN where S = 255
// so the rounding to the element is the only inexact step.  In memory
//     codes  [rows][32 blocks] bytes, e2m1 [rows][16 blocks] (the even element in the low half);
//     scales [rows][blocks rounded up to 4] bytes;       everything past a row's end is zero.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mg {

enum class Num { F32 = 0, F16 = 1, BF16 = 2 };              // the MG_F32 ... codes of the C ABI
enum class Mx { INT8 = 0, E4M3 = 1, E2M1 = 2 };             // the MG_MX_INT8 ... codes

constexpr int kMxBlock = 32;
constexpr int64_t kMemoryCacheBytes = 256ll << 20;      // the chip's memory-side cache

__host__ __device__ inline int64_t mx_blocks(int64_t cols) { return (cols + kMxBlock - 1) / kMxBlock; }
__host__ __device__ inline int64_t mx_scale_pitch(int64_t cols) { return (mx_blocks(cols) + 3) & ~(int64_t)3; }
__host__ __device__ inline int64_t mx_code_pitch(Mx f, int64_t cols)
{
    return mx_blocks(cols) * (f == Mx::E2M1 ? kMxBlock / 2 : kMxBlock);
}

template <Mx F> struct MxTraits;
template <> struct MxTraits<Mx::INT8> { static constexpr int emax = 6; static constexpr uint32_t over = 0x7f0000u; };   // 255/128
template <> struct MxTraits<Mx::E4M3> { static constexpr int emax = 8; static constexpr uint32_t over = 0x680000u; };   // 29/16
template <> struct MxTraits<Mx::E2M1> { static constexpr int emax = 2; static constexpr uint32_t over = 0x600000u; };   // 7/4

// S of a block whose largest magnitude has these float bits (sign cleared).  Adding 2^23 - over to
// the bits carries into the exponent exactly where the significand is >= over; a number below the
// normal range is first doubled, which gives it an exponent field where it can matter (S >= 1).
template <Mx F> __device__ inline uint32_t mx_shared(uint32_t amax)
{
    constexpr uint32_t bump = 0x800000u - MxTraits<F>::over;
    const bool sub = amax < 0x800000u;
    const int k = (int)(((sub ? 2 * amax : amax) + bump) >> 23) - (sub ? 1 : 0);
    const int s = min(max(k - MxTraits<F>::emax, 0), 254);
    return amax >= 0x7f800000u ? 255u : (uint32_t)s;
}

__device__ inline float mx_bits(uint32_t b) { return __builtin_bit_cast(float, b); }
__device__ inline uint32_t mx_word(float f) { return __builtin_bit_cast(uint32_t, f); }

// 2^(127-S); S = 254 gives the subnormal 2^-127, S = 255 zero (so the codes become zero)
__device__ inline float mx_inverse(uint32_t s)
{
    return mx_bits(s < 254u ? (254u - s) << 23 : (s == 254u ? 0x400000u : 0u));
}

// 2^(S-127), S = 0 being subnormal; NaN for S = 255
__device__ inline float mx_power(uint32_t s)
{
    return mx_bits(s == 0u ? 0x400000u : s == 255u ? 0x7fc00000u : s << 23);
}

// Four elements (already divided by the scale) as one word: int8 and e4m3 a byte each.
template <Mx F> __device__ inline uint32_t mx_encode4(const float *y)
{
    if constexpr (F == Mx::INT8) {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int q = (int)rintf(y[i]);
            w |= (uint32_t)(min(max(q, -127), 127) & 255) << (8 * i);
        }
        return w;
    } else {
        static_assert(F == Mx::E4M3, "eight-bit elements");
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    }
}

// Two e2m1 elements into byte `Sel` of `old` (round to nearest even, saturating).
template <int Sel> __device__ inline uint32_t mx_encode_pair(uint32_t old, float a, float b)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, 1.0f, Sel);
}

// The storage types of plain numbers.
template <Num T> struct NumTraits;
template <> struct NumTraits<Num::F32> { using type = float; static constexpr int bytes = 4; };
template <> struct NumTraits<Num::F16> { using type = _Float16; static constexpr int bytes = 2; };
template <> struct NumTraits<Num::BF16> { using type = __bf16; static constexpr int bytes = 2; };

using v4u = __attribute__((ext_vector_type(4))) uint32_t;

// Numbers in 16 bytes, and how many lanes that hold so many share a block.
template <Num T> constexpr int kPerLane = 16 / NumTraits<T>::bytes;
template <Num T> constexpr int kBlockLanes = kMxBlock / kPerLane<T>;

// 16 bytes from an address that need only be aligned to its element (the hardware takes any).
__device__ inline v4u load16(const void *p)
{
    v4u v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

template <Num T> __device__ inline void widen(v4u w, float *f)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (T == Num::F32) {
            f[i] = mx_bits(w[i]);
        } else if constexpr (T == Num::BF16) {
            f[2 * i] = mx_bits(w[i] << 16);
            f[2 * i + 1] = mx_bits(w[i] & 0xffff0000u);
        } else {
            f[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)w[i]);
            f[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i] >> 16));
        }
    }
}

// The numbers of a row from column c on that 16 bytes hold; zeros past the row's end.
template <Num T> __device__ inline v4u load_row(const void *row, int64_t c, int64_t cols)
{
    using E = typename NumTraits<T>::type;
    const E *p = (const E *)row + c;
    if (c + kPerLane<T> <= cols) return load16(p);
    if (c >= cols) return v4u{0, 0, 0, 0};
    E e[kPerLane<T>];
#pragma unroll
    for (int i = 0; i < kPerLane<T>; ++i) e[i] = c + i < cols ? p[i] : (E)0.0f;
    v4u v;
    __builtin_memcpy(&v, e, 16);
    return v;
}

// Largest of the lanes that share a block (8 or 4 neighbours): xor 1, xor 2 within a quad, then the
// mirror image within 8 lanes.
template <int Lanes> __device__ inline uint32_t block_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));     // quad_perm 1,0,3,2
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));     // quad_perm 2,3,0,1
    if constexpr (Lanes == 8)
        v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));   // row_half_mirror
    return v;
}

// This lane's numbers divided by its block's scale (zeros where the block is not finite); the shared byte.
template <Mx F, Num T> __device__ inline uint32_t scale_block(float *f)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kPerLane<T>; ++i) m = max(m, mx_word(f[i]) & 0x7fffffffu);
    const uint32_t s = mx_shared<F>(block_max<kBlockLanes<T>>(m));
    const float inv = mx_inverse(s);
#pragma unroll
    for (int i = 0; i < kPerLane<T>; ++i) f[i] = s == 255u ? 0.0f : f[i] * inv;
    return s;
}

// This lane's elements in 4 bits: 16 bits of 4, a word of 8.
template <Num T> __device__ inline uint32_t encode_e2m1(const float *f)
{
    uint32_t w = mx_encode_pair<0>(0u, f[0], f[1]);
    w = mx_encode_pair<1>(w, f[2], f[3]);
    if constexpr (kPerLane<T> == 8) {
        w = mx_encode_pair<2>(w, f[4], f[5]);
        w = mx_encode_pair<3>(w, f[6], f[7]);
    }
    return w;
}

}  // namespace mg
