// What the kernels of the ternary linear layer and of the 8-bit activation checkpoints share: the 16-bit types,
// the activations and their slopes, the checkpoint's layout and the layout of prepared weights.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace rtn {

// ---- 8-bit checkpoint of a [M][C] tensor ------------------------------------------------------------------------
// Groups of 32 consecutive tokens of one channel share a power of two 2^e; a value is q 2^e, |q| <= 127.
//   codes   [ceil(M / 32)][ceil(C / 8)][32 tokens][8 channels] int8: 256 bytes per (32 tokens, 8 channels), so a thread
//           that has 8 tokens of 8 channels reads or writes 64 bytes in a row
//   scales  [ceil(M / 32)][8 ceil(C / 8)] uint8 behind them, e + 127 (E8M0); 255: the group held an infinity or NaN
// Tokens and channels past the end are zero.
struct CkptShape {
    int64_t tb, cb;  // blocks of 32 tokens, of 8 channels
    __host__ __device__ CkptShape(int64_t M, int64_t C) : tb((M + 31) / 32), cb((C + 7) / 8) {}
    __host__ __device__ int64_t codes() const { return tb * cb * 256; }
    __host__ __device__ int64_t bytes() const { return tb * cb * 264; }
};

// ---- prepared ternary weights of `rows` outputs over `cols` inputs ----------------------------------------------------
// Two bits a weight in the order the matrix instruction takes its operand (32 rows x 16 columns, lane l holding row l & 31,
// columns 8 (l >> 5) .. + 7): [ceil(rows / 32)][ceil(cols / 64)][64 lanes] of 8 bytes.  Word s of a lane holds its codes of the
// 16-column slices 2 s and 2 s + 1 of the 64 columns.  A code is (sign, non-zero) at bits 15:14 of a 16-bit half, which
// as bfloat16 and as float16 alike is -2, 0 or +2; the word keeps 8 codes per half, the one of register r at bits 15 - 2 r,
// 14 - 2 r, so an operand register of two weights is (word << 2 r) & 0xC000C000.  Padding is code 0.
// (Twice the weight, because its one bit is a shift and an AND away; from 2^127 on x and the sums then count as infinite.  +-1 or +-1/2
// instead, the seven bits by an integer product or a byte permutation: 16384 x 8192 x 8192 1474 us -> 1495 and 1513, 4096^3 with gelu
// 100 -> 105 and 105, for the last power of two of a range that activations do not come near.)
struct WeightShape {
    int64_t rb, cb;
    __host__ __device__ WeightShape(int64_t rows, int64_t cols) : rb((rows + 31) / 32), cb((cols + 63) / 64) {}
    __host__ __device__ int64_t bytes() const { return rb * cb * 512; }
};
constexpr unsigned kCodeMask = 0xC000C000u;

// ---- operand order of a [tokens][channels] 16-bit tensor whose product contracts over tokens (weight gradient) -------------
// [2 ceil(M / 64)][ceil(C / 32)][2 slices of 16 tokens][64 lanes][8 tokens]: lane l holds channel l & 31, tokens 8 (l >> 5) .. + 7.
// Tokens and channels past the end are zero.
__host__ __device__ inline int64_t operand_offset(int64_t tb, int64_t cb, int64_t blocks) { return (tb * blocks + cb) * 2048; }
__host__ __device__ inline int64_t operand_blocks(int64_t M) { return (M + 63) / 64 * 2; }
// bytes; a tile of 256 channels at the last blocks reads on behind them, values that reach no output
__host__ __device__ inline int64_t operand_bytes(int64_t M, int64_t C) { return operand_blocks(M) * ((C + 31) / 32) * 2048 + 8 * 2048; }

enum LinearAct { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };

#if defined(__HIPCC__)
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

struct BF16 {
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    // of a checkpoint's scale: 2^-126 is the least normal; 127 x 2^121 is finite, 64 x 2^122 is not
    static constexpr int kLeastExp = -126, kMostExp = 121;
    static __device__ __forceinline__ float to_float(unsigned short v) { return __uint_as_float((unsigned)v << 16); }
    static __device__ __forceinline__ unsigned short from_float(float f)
    {
        return __builtin_bit_cast(unsigned short, (__bf16)f);
    }
    static __device__ __forceinline__ unsigned pack(float lo, float hi)
    {
        return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
    }
    static __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
struct F16 {
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    // every float16 is a multiple of 2^-24, and so is what a checkpoint gives back; 64 x 2^10 is infinite
    static constexpr int kLeastExp = -24, kMostExp = 9;
    static __device__ __forceinline__ float to_float(unsigned short v) { return (float)__builtin_bit_cast(_Float16, v); }
    static __device__ __forceinline__ unsigned short from_float(float f)
    {
        return __builtin_bit_cast(unsigned short, (_Float16)f);
    }
    static __device__ __forceinline__ unsigned pack(float lo, float hi)
    {
        return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2){lo, hi}, f16x2));
    }
    static __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};
template <class T>
__device__ __forceinline__ unsigned pack2(float lo, float hi)
{
    return T::pack(lo, hi);
}
template <class T>
__device__ __forceinline__ float half_of(unsigned pair, int i)
{
    return T::to_float((unsigned short)(i ? pair >> 16 : pair & 0xffffu));
}

// 2^(c v) to about an ulp of the result's exponent's argument
__device__ __forceinline__ float exp_scaled(float v, float c) { return __builtin_amdgcn_exp2f(v * c); }
// The normal distribution's upper tail at |z|, Q, and e = exp(-z^2 / 2), as Q = e t (a1 + .. + a6 t^5), t = 1 / (1 + p |z|).  The
// polynomial is a fit of Q / e over |z| <= 14 (a linear program; the least largest error weighted 1 up to |z| = 1, falling to 1/30 from 4
// on): off by 5.6e-7 of itself near 0, where gelu is a difference of it, and by 1.7e-5 in the tail, where gelu is proportional to
// it and half a unit of float16 is 2.4e-4.  Fourteen operations and two transcendental ones where erff takes sixty: gelu behind a 4096 x 4096
// product 20 -> 9 us.
__device__ __forceinline__ float normal_tail(float z, float& e)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.29860541f, 1.f));
    e = exp_scaled(z * z, -0.72134752f);  // log2(e) / 2
    constexpr float a1 = 0.11965619f, a2 = 0.11148032f, a3 = 0.15152845f, a4 = -0.033207858f, a5 = 0.2316527f, a6 = -0.081110136f;
    return fmaf(fmaf(fmaf(fmaf(fmaf(a6, t, a5), t, a4), t, a3), t, a2), t, a1) * t * e;
}
// 16 bytes wherever they start (global accesses need no alignment on this target)
__device__ __forceinline__ u32x4 load16(const void* p)
{
    u32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
__device__ __forceinline__ void store16(void* p, u32x4 v) { __builtin_memcpy(p, &v, 16); }
// Elements k .. k + 7 of a row of `len`, zeros past its end: the row's last 16 bytes, shifted, where they do not all exist.  (One
// load; eight conditional ones wait for each other.)
__device__ __forceinline__ u32x4 load_row8(const unsigned short* row, int64_t k, int64_t len)
{
    if (k + 8 <= len) return load16(row + k);
    if (k >= len) return u32x4{0, 0, 0, 0};
    if (len < 8) {
        u32x4 v = {0, 0, 0, 0};
        for (int i = 0; i < 7; ++i)
            if (k + i < len) v[i >> 1] |= (unsigned)row[k + i] << (16 * (i & 1));
        return v;
    }
    const u32x4 t = load16(row + len - 8);
    const int s = (int)(k + 8 - len) * 16;  // 16 .. 112
    const uint64_t lo = t[0] | (uint64_t)t[1] << 32, hi = t[2] | (uint64_t)t[3] << 32;
    const uint64_t l = s < 64 ? lo >> s | hi << (64 - s) : hi >> (s - 64), u = s < 64 ? hi >> s : 0;
    return u32x4{(unsigned)l, (unsigned)(l >> 32), (unsigned)u, (unsigned)(u >> 32)};
}

// phi(z) in fp32.  gelu is z Phi(z) = max(z, 0) - |z| Q(|z|), Phi the normal distribution; silu z / (1 + exp(-z)).
template <int ACT>
__device__ __forceinline__ float act_value(float z)
{
    if constexpr (ACT == kActRelu) return z > 0.f ? z : (z == z ? 0.f : z);
    if constexpr (ACT == kActGelu) {
        float e;
        const float q = normal_tail(z, e);
        return fmaf(-fminf(fabsf(z), 64.f), q, fmaxf(z, 0.f));  // (Q is 0 from 14 on, and 0 times an infinity none)
    }
    if constexpr (ACT == kActSilu) return z * __builtin_amdgcn_rcpf(1.f + exp_scaled(z, -1.44269504f));
    return z;
}
// phi'(z): 1 / 0 of a relu (0 at 0, and a NaN gives NaN), Phi(z) + z times the normal density, s (1 + z (1 - s)).
template <int ACT>
__device__ __forceinline__ float act_slope(float z)
{
    if constexpr (ACT == kActRelu) return z > 0.f ? 1.f : (z == z ? 0.f : z);
    if constexpr (ACT == kActGelu) {
        float e;
        const float q = normal_tail(z, e);
        return fmaf(z * 0.39894228f, e, z < 0.f ? q : 1.f - q);
    }
    if constexpr (ACT == kActSilu) {
        const float s = __builtin_amdgcn_rcpf(1.f + exp_scaled(z, -1.44269504f));
        return s * (1.f + z * (1.f - s));
    }
    return 1.f;
}

// The scale of a group whose largest magnitude is `amax`: the exponent e, so that rint(amax 2^-e) is 64 .. 127 (amax 2^-e
// in [127.5, 128) would round to 128 and takes the next one), within T's range.  Returned as e + 127; 255: not finite.
template <class T>
__device__ __forceinline__ int ckpt_exponent(float amax)
{
    const unsigned u = __float_as_uint(amax);
    if (u >= 0x7f800000u) return 255;
    const int biased = (int)(u >> 23) - 6 + ((u & 0x7fffffu) >= 0x7f0000u);  // 127.5 / 64 = 1.1111111b
    constexpr int lo = T::kLeastExp + 127, hi = T::kMostExp + 127;
    return biased < lo ? lo : biased > hi ? hi : biased;
}
// Four values / 2^e as codes.  v / 2^e + 1.5 x 2^23 in one rounding has the nearest integer, ties to even, in its low
// byte.  CLAMP: beyond +-127 are only values at the end of T's range (and, of a float16 layer, z beyond it).
__device__ __forceinline__ unsigned ckpt_codes(float a, float b, float c, float d, float ia, float ib, float ic, float id, bool clamp)
{
    if (clamp) {
        a = __builtin_amdgcn_fmed3f(a * ia, -127.f, 127.f), b = __builtin_amdgcn_fmed3f(b * ib, -127.f, 127.f);
        c = __builtin_amdgcn_fmed3f(c * ic, -127.f, 127.f), d = __builtin_amdgcn_fmed3f(d * id, -127.f, 127.f);
        ia = ib = ic = id = 1.f;
    }
    const float magic = 12582912.f;
    const unsigned lo = __builtin_amdgcn_perm(__float_as_uint(fmaf(b, ib, magic)), __float_as_uint(fmaf(a, ia, magic)), 0x0c0c0400u);
    const unsigned hi = __builtin_amdgcn_perm(__float_as_uint(fmaf(d, id, magic)), __float_as_uint(fmaf(c, ic, magic)), 0x0c0c0400u);
    return lo | hi << 16;
}
__device__ __forceinline__ float ckpt_scale(int biased) { return __uint_as_float(biased == 255 ? 0x7fc00000u : (unsigned)biased << 23); }
// 2^-e; for e in -126 .. 122 both are normal
__device__ __forceinline__ float ckpt_inverse(int biased) { return __uint_as_float((unsigned)(biased == 255 ? 0 : 254 - biased) << 23); }

}  // namespace
#endif

}  // namespace rtn
