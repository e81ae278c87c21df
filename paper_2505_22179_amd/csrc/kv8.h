// The 8-bit attention cache: what a code and its scale stand for, on the device.
//
// A head of one cached row (D values) has D codes of 8 bits and one fp16 scale.  The scales have so few significant bits -- four
// for int8 codes (seven bits), one for e4m3 codes (four bits) -- that code x scale always is an fp16 number: turning codes back rounds nothing,
// and the fp16 matrix products read exactly what w4a16_kv8_read returns.  A scale of arbitrary mantissa would give int8 codes an eighth of a
// bit more and cost a rounding, or two multiplications per score, everywhere the cache is read.
//   int8  s = amax / 127 rounded up to four significant bits (a multiple of 2^-24, at most 512), code = round(v / s) in +-127
//   e4m3  s = amax / 448 rounded up to a power of two (at least 2^-15), code = e4m3(v / s) in +-448, in +-240 where s = 256 (256 x 256
//         would be beyond fp16)
// A head with an infinity or a NaN has scale NaN and codes zero: every value of it reads back as NaN.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace w4 {

constexpr int kInt8 = W4A16_KV8_INT8, kE4m3 = W4A16_KV8_E4M3;
constexpr uint32_t kHalfInf = 0x7C00u, kHalfNan = 0x7E00u;
typedef _Float16 half2v __attribute__((ext_vector_type(2)));

// scale of a head whose largest magnitude is the finite fp16 number amax
template <int FMT>
__device__ __forceinline__ float kv8_scale(float amax)
{
    if constexpr (FMT == kInt8) {
        // The quotient is exact to 2^-24 and lies 2^-18 or more away from any number of four significant bits that it does not equal
        // (amax has eleven bits, 127 times such a number at most eleven), so that rounding up meets the right one.
        const float t = amax / 127.f;
        if (t < 0x1p-21f) return fmaxf(ceilf(t * 0x1p24f), 1.f) * 0x1p-24f;
        return fminf(__builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, t) + 0xFFFFFu) & ~0xFFFFFu), 512.f);
    } else {
        const float t = amax / 448.f;
        return fmaxf(__builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, t) + 0x7FFFFFu) & ~0x7FFFFFu), 0x1p-15f);
    }
}

// codes of four values, one per byte; v / s with a division, so that ties are met exactly
template <int FMT>
__device__ __forceinline__ uint32_t kv8_codes(const float (&v)[4], float s)
{
    if constexpr (FMT == kInt8) {
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int code = (int)fminf(fmaxf(rintf(v[e] / s), -127.f), 127.f);
            w |= ((uint32_t)code & 0xFFu) << (8 * e);
        }
        return w;
    } else {
        const float inv = 1.f / s;   // a power of two: the products are the quotients
        const float most = s == 256.f ? 240.f : 448.f;
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fminf(fmaxf(v[e] * inv, -most), most);
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
        return (uint32_t)w;
    }
}

// the numbers of four codes, unscaled: int8 through the fp16 numbers 1024 + (code + 128), whose low bits are the biased code
template <int FMT>
__device__ __forceinline__ void kv8_numbers(uint32_t w, half2v &lo, half2v &hi)
{
    if constexpr (FMT == kInt8) {
        const uint32_t biased = w ^ 0x80808080u;
        const half2v off = {(_Float16)-1152.f, (_Float16)-1152.f};
        lo = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, biased, 0x04010400u)) + off;
        hi = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, biased, 0x04030402u)) + off;
    } else {
        lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.f, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.f, true);
    }
}

// the values of four codes of one head; NaN for a NaN scale
template <int FMT>
__device__ __forceinline__ void kv8_values(uint32_t w, _Float16 scale, half2v &lo, half2v &hi)
{
    if constexpr (FMT == kInt8) {
        kv8_numbers<FMT>(w, lo, hi);
        const half2v s = {scale, scale};
        lo *= s;
        hi *= s;
    } else {
        lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, (float)scale, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, (float)scale, true);
    }
}

// Codes that are no numbers, or no fp16 numbers under their head's scale (bits).  The appends write none, but what a mask hides may hold them, and a probability
// of zero would make NaN of them.  kv8_suspect, for sixteen codes: whether there may be any -- an e4m3 byte of seven ones, or a scale under which the largest
// number, 448 or 128, comes to 65520 or is none; kv8_no_numbers: whether there are (few come here, so its loop is a loop).
template <int FMT>
__device__ __forceinline__ bool kv8_suspect(uint32_t __attribute__((ext_vector_type(4))) w, uint32_t scale)
{
    constexpr uint32_t kLargest = FMT == kInt8 ? 0x5FFCu : 0x5800u;   // 511, 128
    uint32_t ones = 0;
    if constexpr (FMT == kE4m3) {
#pragma unroll
        for (int e = 0; e < 4; ++e) ones |= (w[e] & 0x7F7F7F7Fu) + 0x01010101u;
    }
    return (ones & 0x80808080u) != 0 || (scale & 0x7FFFu) > kLargest;
}
template <int FMT>
__device__ __forceinline__ bool kv8_no_numbers(uint32_t __attribute__((ext_vector_type(4))) w, uint32_t scale)
{
    const half2v s = {__builtin_bit_cast(_Float16, (uint16_t)scale), __builtin_bit_cast(_Float16, (uint16_t)scale)};
    bool any = false;
#pragma unroll 1
    for (int e = 0; e < 4; ++e) {
        half2v n[2];
        kv8_numbers<FMT>(w[0], n[0], n[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t x = __builtin_bit_cast(uint32_t, (half2v)(n[i] * s)) & 0x7FFF7FFFu;
            any |= (x & 0xFFFFu) >= kHalfInf || x >= (kHalfInf << 16);
        }
        w = __builtin_shufflevector(w, w, 1, 2, 3, 0);
    }
    return any;
}

inline bool kv8_format_known(int format) { return format == kInt8 || format == kE4m3; }

}  // namespace w4
