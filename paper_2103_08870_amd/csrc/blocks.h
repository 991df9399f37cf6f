// Matrices held in 8 bits: e4m3 codes with one exponent per block of 128 columns (gfx950).
#pragma once
#include "device_helpers.h"

namespace lgc {

constexpr int kChunkCols = 8;     // columns that one lane handles at a time: 16 lanes make a block

typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef short s2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
// accesses at any address that the element's size divides (the hardware takes them)
typedef u4 u4e __attribute__((aligned(2)));
typedef u2 u2e __attribute__((aligned(2)));

struct Bf16 { uint16_t bits; };
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(Bf16 x) { return __uint_as_float((uint32_t)x.bits << 16); }
// to the nearest, ties to even; NaNs stay NaNs
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    bf2 r = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ void store_one(float *p, float x) { *p = x; }
__device__ __forceinline__ void store_one(Bf16 *p, float x) { p->bits = (uint16_t)bf16_pair(x, x); }

// How many of the eight columns from `col` on a row of `cols` has.
__device__ __forceinline__ int count_at(uint32_t col, uint32_t cols) { return col >= cols ? 0 : cols - col >= 8 ? 8 : (int)(cols - col); }

// The eight elements of a row from column `col` on, as they lie in memory: a load that is under way until they are unpacked.  Where the row has fewer, the last eight
// that it has are asked for instead, so that no lane needs loads of its own (which the others' would be waited for before); a row of fewer than eight has them all.
template <typename T>
struct Chunk {
    u4 part[sizeof(T) / 2];
};
__device__ __forceinline__ Chunk<float> fetch_chunk(const float *row, uint32_t col, uint32_t cols) {
    Chunk<float> c;
    if (cols >= 8) {
        const float *at = row + min(col, cols - 8);
        c.part[0] = *(const u4u *)at;
        c.part[1] = *(const u4u *)(at + 4);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) c.part[i / 4][i % 4] = col + i < cols ? __float_as_uint(row[col + i]) : 0u;
    }
    return c;
}
__device__ __forceinline__ Chunk<Bf16> fetch_chunk(const Bf16 *row, uint32_t col, uint32_t cols) {
    Chunk<Bf16> c;
    if (cols >= 8) c.part[0] = *(const u4e *)(row + min(col, cols - 8));
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = col + 2 * i, hi = lo + 1;
            c.part[0][i] = (lo < cols ? row[lo].bits : 0u) | (hi < cols ? (uint32_t)row[hi].bits << 16 : 0u);
        }
    }
    return c;
}
// Elements that do not exist become zeros.
template <typename T>
__device__ __forceinline__ void unpack(const Chunk<T> &c, uint32_t col, uint32_t cols, float (&x)[8]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(c.part[i / 4][i % 4]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(c.part[0][i] << 16); x[2 * i + 1] = __uint_as_float(c.part[0][i] & 0xffff0000u); }
    }
    if (cols >= 8 && col + 8 > cols)
        for (int k = count_at(col, cols); k < 8; ++k) {
#pragma unroll
            for (int i = 0; i < 7; ++i) x[i] = x[i + 1];
            x[7] = 0.f;
        }
}
template <typename T>
__device__ __forceinline__ void load_chunk(const T *row, uint32_t col, uint32_t cols, float (&x)[8]) { unpack(fetch_chunk(row, col, cols), col, cols, x); }
__device__ __forceinline__ void store_chunk(float *p, int count, const float (&x)[8]) {
    if (count >= 8) {
        *(f4u *)p = f4{x[0], x[1], x[2], x[3]};
        *(f4u *)(p + 4) = f4{x[4], x[5], x[6], x[7]};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < count) p[i] = x[i];
    }
}
__device__ __forceinline__ void store_chunk(Bf16 *p, int count, const float (&x)[8]) {
    if (count >= 8) {
        *(u4e *)p = u4{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7])};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < count) store_one(p + i, x[i]);
    }
}

// The largest of 16 neighbouring lanes' values, in all of them (rotations inside a row of lanes, register to register).
__device__ __forceinline__ uint32_t max_of_16(uint32_t x) {
    auto larger = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
    x = larger(x, __builtin_amdgcn_update_dpp(0u, x, 0x128, 0xf, 0xf, false));   // row_ror:8
    x = larger(x, __builtin_amdgcn_update_dpp(0u, x, 0x124, 0xf, 0xf, false));
    x = larger(x, __builtin_amdgcn_update_dpp(0u, x, 0x122, 0xf, 0xf, false));
    x = larger(x, __builtin_amdgcn_update_dpp(0u, x, 0x121, 0xf, 0xf, false));
    return x;
}

constexpr uint32_t kInfKey = 0x7f800000u;
constexpr uint32_t kLeastExp = 10;
constexpr uint32_t kMostExp = 247;   // of the block whose largest magnitude passes 1.75 * 2^127

// The exponent byte of a block whose largest finite magnitude has this key: the least E, from kLeastExp on, with magnitude <= 448 * 2^(E - 127)
// (448 = 1.75 * 2^8 is the largest code).  A scale that is a power of two makes the division exact, so that each element is rounded once, and it
// costs e4m3, itself a floating-point type, no precision.  From kLeastExp on the least code, 2^-9, stands for a normal number of fp32 and bf16.
__device__ __forceinline__ uint32_t block_exp(uint32_t key) {
    const int e = (int)(key >> 23) - 8 + ((key & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < (int)kLeastExp ? kLeastExp : (uint32_t)e;
}
__device__ __forceinline__ float exp_scale(uint32_t e) { return __uint_as_float(e << 23); }   // 2^(e - 127)

// Key of the largest finite magnitude of the eight elements that each of 16 neighbouring lanes holds, in all of them.  The maximum passes over NaNs by itself;
// only where it meets an infinity are elements looked at one by one.
__device__ __forceinline__ uint32_t most_of_16(const float (&x)[8]) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(x[i]));
    uint32_t most = max_of_16(__float_as_uint(m));
    if (most == kInfKey) {
        uint32_t key = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t k = key_of(x[i]);
            key = k < kInfKey && k > key ? k : key;
        }
        most = max_of_16(key);
    }
    return most;
}
// Codes of eight elements divided by the block's scale 2^(e - 127), rounded to the nearest (ties to even); the conversion turns infinities into NaN codes.
// At the largest e a number may round to code 256 (0x78), whose value is beyond fp32 and bf16: it becomes 240, which is still within 2^-4 of it.
__device__ __forceinline__ u2 codes_of(const float (&x)[8], uint32_t e) {
    const float scale = exp_scale(e);
    u2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const s2 lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s2{0, 0}, x[4 * i], x[4 * i + 1], scale, false);
        r[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, x[4 * i + 2], x[4 * i + 3], scale, true));
    }
    if (e == kMostExp)
#pragma unroll
        for (int i = 0; i < 2; ++i) r[i] -= ((0x80808080u - ((r[i] & 0x7f7f7f7fu) ^ 0x78787878u)) & 0x80808080u) >> 7;   // (of four bytes, 1 from those that are 0x78)
    return r;
}
__device__ __forceinline__ void values_of(const u2 codes, float scale, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes[i], scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes[i], scale, true);
        x[4 * i] = a[0]; x[4 * i + 1] = a[1]; x[4 * i + 2] = b[0]; x[4 * i + 3] = b[1];
    }
}

// 16 lanes store the block that they hold, eight elements each: codes at `codes` (the lane's own eight), exponent at `exp` (the block's).
// Elements that do not exist are zeros.  All 16 lanes must be active.
__device__ __forceinline__ void store_block(const float (&x)[8], uint8_t *codes, uint8_t *exp) {
    const uint32_t e = block_exp(most_of_16(x));
    *(u2 *)codes = codes_of(x, e);
    if ((threadIdx.x & 15) == 0) *exp = (uint8_t)e;
}

// Normal distribution's function below -|x|, over exp(-x^2 / 2): t * (c0 + c1 t + .. + c6 t^6) with t = 1 / (1 + p |x|), fitted (least largest relative
// error, by reweighted least squares) for 0 <= |x| <= 13.5, where it is off by 5.3e-7 at most; the tail keeps its relative precision, since nothing is
// subtracted from 1.  Measured, GELU is off by 1e-6 of the result at most from -2 on (fp32 with an exact erf: 1.5e-7 around 0, 5e-2 of the result at -5), by 2e-6 at -5
// and 8e-6 at -13, where the exponential's argument is rounded at its size; its slope by 4e-7, absolute.  One exponential and one reciprocal, for results that mostly go on
// to bf16 or 8 bits.
__device__ __forceinline__ float normal_below(float size, float gauss) {
    const float t = __builtin_amdgcn_rcpf(1.f + 0.26390194744793544f * size);
    float s = -0.0694093182682991f;
    s = fmaf(s, t, 0.20417608320713043f);
    s = fmaf(s, t, -0.07719594985246658f);
    s = fmaf(s, t, 0.14925582706928253f);
    s = fmaf(s, t, 0.08022129535675049f);
    s = fmaf(s, t, 0.10782003402709961f);
    s = fmaf(s, t, 0.10513176769018173f);
    return s * t * gauss;
}

constexpr float kLog2e = 1.4426950408889634f;

template <int kAct>
__device__ __forceinline__ float act(float x) {
    if constexpr (kAct == LGC_RELU) return x < 0.f ? 0.f : x;   // (a NaN stays)
    if constexpr (kAct == LGC_SILU) return x * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * x));
    const float below = normal_below(fabsf(x), __builtin_amdgcn_exp2f(-0.5f * kLog2e * x * x));
    return x * (x < 0.f ? below : 1.f - below);
}
template <int kAct>
__device__ __forceinline__ float act_slope(float x) {
    if constexpr (kAct == LGC_RELU) return x > 0.f ? 1.f : x <= 0.f ? 0.f : x;
    if constexpr (kAct == LGC_SILU) {
        const float p = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * x));
        return fmaf(x * p, 1.f - p, p);
    }
    const float gauss = __builtin_amdgcn_exp2f(-0.5f * kLog2e * x * x), below = normal_below(fabsf(x), gauss);
    return fmaf(x * gauss, 0.3989422804014327f, x < 0.f ? below : 1.f - below);
}

// Which (row, block) a number stands for: division by a block count known when the kernel is launched.
struct Divide {
    uint32_t by, magic, shift;
};
inline Divide divide_by(uint32_t d) {   // d >= 1; exact for dividends below 2^31
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return Divide{d, (uint32_t)(((1ull << 32) * ((1ull << s) - d)) / d + 1), s};
}
__device__ __forceinline__ uint32_t quotient(uint32_t x, const Divide &d) {
    const uint32_t t = __umulhi(x, d.magic);
    return (t + x) >> d.shift;   // t <= x < 2^31: the sum does not wrap
}

}  // namespace lgc
