// What the kernels of the microscaled 4-bit operators share: the packed layout, the conversions and the random numbers.
#pragma once
#include <type_traits>

#include "linear_math.h"

namespace rtn {

// ---- packed 4-bit values of a [R][C] matrix -------------------------------------------------------------------------
// 32 consecutive columns of a row share a scale 2^(s - 127), s one byte (E8M0; 255: the group held an infinity or NaN and stands
// for NaN); a value is an E2M1 code (0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign) times the scale.
//   codes   [ceil(R / 16)][ceil(C / 128)][64 lanes] of 16 bytes: lane l holds row l & 15, columns 32 (l >> 4) .. + 31, two to a
//           byte, which is the operand of v_mfma_scale_f32_16x16x128_f8f6f4 and one group of 32 a lane: 1 KiB in a row
//   scales  [ceil(R / 64)][ceil(C / 128)][64 lanes][4] behind them: byte i of lane l is that of lane l's group in the i-th of
//           four blocks of 16 rows, so that one register holds a lane's scales of 64 rows and the instruction picks the byte
// Rows and columns past the end are codes 0.
struct Mx4Shape {
    int64_t rb, kb, rg;  // blocks of 16 rows, of 128 columns; groups of four blocks of rows
    __host__ __device__ Mx4Shape(int64_t R, int64_t C) : rb((R + 15) / 16), kb((C + 127) / 128), rg((R + 63) / 64) {}
    __host__ __device__ int64_t codes() const { return rb * kb * 1024; }
    __host__ __device__ int64_t bytes() const { return codes() + rg * kb * 256; }
};

#if defined(__HIPCC__)
namespace {

struct F32 {};  // the type of unrounded inputs and outputs, beside BF16 and F16

// Elements k .. k + 7 of a row of `len` as floats, zeros past its end
template <class T>
__device__ __forceinline__ void load_values(const void* row, int64_t k, int64_t len, float (&v)[8])
{
    if constexpr (std::is_same_v<T, F32>) {
        const float* p = (const float*)row + k;
        if (k + 8 <= len) {
            __builtin_memcpy(v, p, 32);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k + i < len ? p[i] : 0.f;
        }
    } else {
        const u32x4 q = load_row8((const unsigned short*)row, k, len);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = half_of<T>(q[i >> 1], i & 1);
    }
}
template <class T>
constexpr int kBytesOf = std::is_same_v<T, F32> ? 4 : 2;

// The largest magnitude of some floats as bits (a NaN is larger than an infinity, and that than any number).  As signed numbers the positive ones
// are the larger, as unsigned ones the negative ones: a maximum of each kind over three values is one instruction.
struct Largest {
    int pos = 0;
    unsigned neg = 0;
    __device__ __forceinline__ void take(float a, float b)
    {
        const int i = __float_as_int(a), j = __float_as_int(b);
        const int m = i > j ? i : j;
        pos = m > pos ? m : pos;
        const unsigned u = (unsigned)i > (unsigned)j ? (unsigned)i : (unsigned)j;
        neg = u > neg ? u : neg;
    }
    __device__ __forceinline__ unsigned bits() const
    {
        const unsigned n = neg & 0x7fffffffu;
        return (unsigned)pos > n ? (unsigned)pos : n;
    }
};
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }

// Scale byte of a group from its largest magnitude a: floor(log2 a) - 2, at least -127, so a / 2^e is 4 .. 8.  Stochastic rounding takes
// one more where a / 2^e > 6, so that no value is beyond the largest code and the expected value stays v.
__device__ __forceinline__ int mx4_scale(unsigned a, bool stochastic)
{
    const int e = (int)(a >> 23) - 2 + (stochastic && (a & 0x7fffffu) > 0x400000u && a >= 0x01000000u), s = e < 0 ? 0 : e;
    return a >= 0x7f800000u ? 255 : s;  // (0 is 2^-127; a is below 2^-125 then, 4 of it)
}
__device__ __forceinline__ float mx4_factor(int s) { return s == 255 ? __uint_as_float(0x7fc00000u) : s ? __uint_as_float((unsigned)s << 23) : __uint_as_float(0x00400000u); }
// 2^-e; e is -127 .. 126
__device__ __forceinline__ float mx4_inverse(int s) { return __uint_as_float((unsigned)(254 - s) << 23); }

// Eight values to eight codes, the nearest, ties to the even code, 6 beyond 6.
__device__ __forceinline__ unsigned mx4_nearest(const float* v, int s)
{
    const float f = mx4_factor(s);
    unsigned q = 0;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0], v[1], f, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], f, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], f, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], f, 3);
    return s == 255 ? 0 : q;
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers, as easy as 1, 2, 3; 2011): ten rounds of two 32 x 32 -> 64
// products, the counter's words exchanged and xored with a key that grows by a constant each round.
__device__ __forceinline__ unsigned xor3(unsigned a, unsigned b, unsigned c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }
__device__ __forceinline__ uint4 philox(uint4 c, unsigned k0, unsigned k1)
{
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+s"(k0), "+s"(k1));  // scalar additions each round; kept across calls, the twenty words would spill
#endif
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
        c = make_uint4(xor3((unsigned)(b >> 32), c.y, k0), (unsigned)b, xor3((unsigned)(a >> 32), c.w, k1), (unsigned)a);
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
    return c;
}
// Whose numbers a group takes: its index row * groups + group of the packing, and which packing it is (1: the transposed one)
struct Mx4Random {
    uint64_t seed, group;
    unsigned transposed;
    // for elements 8 j .. + 7 of the group, 16 bits each
    __device__ __forceinline__ uint4 bits(int j) const
    {
        return philox(make_uint4((unsigned)group, (unsigned)(group >> 32), (unsigned)j, transposed), (unsigned)seed, (unsigned)(seed >> 32));
    }
};
// Eight values to eight codes: the code below |v| / 2^e, or the next one where 16 random bits k are below F, 65536 times the distance from it in
// units of the gap; with c = 65535 - k that is  c + ceil(F) >= 65536.  An fp32 number of 2^-126 times |v| / 2^e has the structure of the code,
// its numbers below 1 without a leading bit among them: the code is its bits from 22 on, and the 22 below are 64 F, rounded up if
// the product is.  So adding 64 c + 63 and taking the upper bits is all.  (The comparison with F spelt out: 252 vector instructions
// for 8 values of a wave with their random bits and all that goes with them, here 158; 16384 x 8192 both ways, bound by them, 229 -> 153 us.)
__device__ __forceinline__ unsigned mx4_stochastic(const float* v, int s, const uint4& r)
{
    float a[8] = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
#if defined(__HIP_DEVICE_COMPILE__)
    const float inv = mx4_inverse(s == 255 ? 127 : s);
    // both products towards plus infinity; the mode is back before any other instruction
    asm volatile("s_setreg_imm32_b32 hwreg(HW_REG_MODE, 0, 2), 1\n\t"
                 "v_mul_f32_e64 %0, |%0|, %8\n\tv_mul_f32_e64 %1, |%1|, %8\n\tv_mul_f32_e64 %2, |%2|, %8\n\tv_mul_f32_e64 %3, |%3|, %8\n\t"
                 "v_mul_f32_e64 %4, |%4|, %8\n\tv_mul_f32_e64 %5, |%5|, %8\n\tv_mul_f32_e64 %6, |%6|, %8\n\tv_mul_f32_e64 %7, |%7|, %8\n\t"
                 "v_mul_f32_e32 %0, %9, %0\n\tv_mul_f32_e32 %1, %9, %1\n\tv_mul_f32_e32 %2, %9, %2\n\tv_mul_f32_e32 %3, %9, %3\n\t"
                 "v_mul_f32_e32 %4, %9, %4\n\tv_mul_f32_e32 %5, %9, %5\n\tv_mul_f32_e32 %6, %9, %6\n\tv_mul_f32_e32 %7, %9, %7\n\t"
                 "s_setreg_imm32_b32 hwreg(HW_REG_MODE, 0, 2), 0"
                 : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]), "+v"(a[4]), "+v"(a[5]), "+v"(a[6]), "+v"(a[7])
                 : "v"(inv), "s"(0x00800000u));
#endif
    const unsigned words[4] = {r.x, r.y, r.z, r.w};
    unsigned q = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned k = i & 1 ? words[i >> 1] >> 10 : words[i >> 1] << 6;  // 64 k and bits around it
        const unsigned t = __float_as_uint(a[i]) + ((~k & 0x3fffffu) | 63u);
        const unsigned code = i < 6 ? t >> (22 - 4 * i) : t << (4 * i - 22);
        q |= (code & 7u << 4 * i) | (__float_as_uint(v[i]) >> (28 - 4 * i) & 8u << 4 * i);
    }
    return s == 255 ? 0 : q;
}
// The codes of a word as values / 2^e
__device__ __forceinline__ void mx4_values(unsigned q, float (&v)[8])
{
    auto pair = [&](auto sel) {
        constexpr int i = decltype(sel)::value;
        const f32x2 p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.f, i);
        v[2 * i] = p[0], v[2 * i + 1] = p[1];
    };
    pair(std::integral_constant<int, 0>{});
    pair(std::integral_constant<int, 1>{});
    pair(std::integral_constant<int, 2>{});
    pair(std::integral_constant<int, 3>{});
}

}  // namespace
#endif

}  // namespace rtn
