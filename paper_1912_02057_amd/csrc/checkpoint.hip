// Activations kept in 8 bits between the forward and the backward pass (CkptShape): into 8 bits, back, and into the operand
// order of the weight gradient's product, there together with the gradient that it meets.
//
// All of them are one pass over memory.  A wave has 32 tokens x 64 channels, a lane 4 tokens of 8 channels: 4 rows of 16 bytes
// of a 16-bit tensor (8 lanes beside each other read 128 bytes of a row), 32 bytes in a row of a checkpoint.  (8 tokens a lane need
// twice the registers: the gradient's pass over 16384 x 8192, without an activation, took 282 us with 190 of them and takes 212 with 163.)
#include "linear_math.h"
#include "rtn_kernels.h"

namespace rtn {

namespace {

constexpr int kTok = 4, kStrip = 64;  // tokens of a lane; channels of a wave

struct Micro {  // what a lane owns
    int64_t mb, c;  // block of 32 tokens; its first channel
    int t0;         // first of its tokens in the block
};
__device__ __forceinline__ Micro micro_of(int64_t mb, int64_t strip)
{
    const int lane = threadIdx.x & 63;
    return {mb, strip * kStrip + (lane & 7) * 8, (lane >> 3) * kTok};
}

// 8 channels of a row as they are; zeros past the end
__device__ __forceinline__ u32x4 load_row(const unsigned short* x, int64_t ld, int64_t m, int64_t M, int64_t c, int64_t C)
{
    return m < M ? load_row8(x + m * ld, c, C) : u32x4{0, 0, 0, 0};
}

template <class T>
__global__ __launch_bounds__(256) void k_ckpt_pack(CkptArgs a, int strips)
{
    const CkptShape cs(a.M, a.C);
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= cs.tb * strips) return;
    const int64_t mb = unit / strips;
    const Micro u = micro_of(mb, unit - mb * strips);
    u32x4 v[kTok];
#pragma unroll
    for (int t = 0; t < kTok; ++t)
        v[t] = load_row((const unsigned short*)a.x, a.ld, mb * 32 + u.t0 + t, a.M, u.c, a.C);
    unsigned ex[2] = {0, 0};
    float inv[8];
    bool end = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        unsigned am = 0;  // as bits: a NaN is larger than an infinity, and that than any number
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            const unsigned b = (v[t][i >> 1] >> (16 * (i & 1))) & 0x7fffu;
            am = b > am ? b : am;
        }
#pragma unroll
        for (int d = 8; d < 64; d *= 2) {
            const unsigned o = (unsigned)__shfl_xor((int)am, d);
            am = o > am ? o : am;
        }
        const int e = ckpt_exponent<T>(T::to_float((unsigned short)am));
        ex[i >> 2] |= (unsigned)e << (8 * (i & 3));
        inv[i] = ckpt_inverse(e);
        end |= e == T::kMostExp + 127;
    }
    const bool clamp = __any(end);
    if (u.c >= a.C) return;
    const int64_t blk = mb * cs.cb + (u.c >> 3);
    unsigned w[2 * kTok];
#pragma unroll
    for (int t = 0; t < kTok; ++t)
#pragma unroll
        for (int q = 0; q < 2; ++q)
            w[t * 2 + q] = ckpt_codes(half_of<T>(v[t][2 * q], 0), half_of<T>(v[t][2 * q], 1), half_of<T>(v[t][2 * q + 1], 0),
                                      half_of<T>(v[t][2 * q + 1], 1), inv[4 * q], inv[4 * q + 1], inv[4 * q + 2], inv[4 * q + 3], clamp);
    uint4* out = (uint4*)(a.ckpt + blk * 256 + u.t0 * 8);
#pragma unroll
    for (int i = 0; i < kTok / 2; ++i) out[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    if (u.t0 == 0) *(uint2*)(a.ckpt + cs.codes() + blk * 8) = make_uint2(ex[0], ex[1]);
}

// The tokens and channels of a lane of a checkpoint: codes and scales.
struct MicroCkpt {
    uint4 q[kTok / 2];
    uint2 e;
    __device__ __forceinline__ void load(const int8_t* ckpt, const CkptShape& cs, const Micro& u)
    {
        const int64_t blk = u.mb * cs.cb + (u.c >> 3);
        const uint4* p = (const uint4*)(ckpt + blk * 256 + u.t0 * 8);
#pragma unroll
        for (int i = 0; i < kTok / 2; ++i) q[i] = p[i];
        e = *(const uint2*)(ckpt + cs.codes() + blk * 8);
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < kTok / 2; ++i) q[i] = make_uint4(0, 0, 0, 0);
        e = make_uint2(0, 0);
    }
    __device__ __forceinline__ float scale(int i) const { return ckpt_scale((int)((i < 4 ? e.x : e.y) >> (8 * (i & 3)) & 255)); }
    // channel i of token t, to be multiplied by scale(i)
    __device__ __forceinline__ float code(int t, int i) const
    {
        const uint4& r = q[t >> 1];
        const unsigned w = t & 1 ? (i < 4 ? r.z : r.w) : (i < 4 ? r.x : r.y);
        return (float)((int)(w << (24 - 8 * (i & 3))) >> 24);
    }
};

template <class T>
__global__ __launch_bounds__(256) void k_ckpt_unpack(CkptArgs a, int strips)
{
    const CkptShape cs(a.M, a.C);
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= cs.tb * strips) return;
    const int64_t mb = unit / strips;
    const Micro u = micro_of(mb, unit - mb * strips);
    if (u.c >= a.C) return;
    MicroCkpt k;
    k.load(a.ckpt, cs, u);
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = k.scale(i);
#pragma unroll
    for (int t = 0; t < kTok; ++t) {
        const int64_t m = mb * 32 + u.t0 + t;
        if (m >= a.M) break;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = k.code(t, i) * s[i];
        unsigned short* y = (unsigned short*)a.y + m * a.ld + u.c;
        if (u.c + 8 <= a.C) {
            const u32x4 o = {pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])};
            __builtin_memcpy(y, &o, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (u.c + i < a.C) y[i] = T::from_float(v[i]);
        }
    }
}

// A wave's 32 tokens x 64 channels (v[channel][token pair] of each lane) -> the operand order of the weight gradient.  Through
// LDS, so that every store of the wave is 1 KiB in a row.  16-byte piece p of the wave's 4 KiB is kept at p ^ (p / 8 ^ p / 64) % 8,
// which spreads the writes over the banks.
__device__ __forceinline__ void store_operand(char* out, int64_t blocks, const Micro& u, const uint2 (&v)[8], char* lds)
{
    const int lane = threadIdx.x & 63;
    auto at = [&](int p) { return lds + 16 * (p ^ (((p >> 3) ^ (p >> 6)) & 7)); };
    const int c = (lane & 7) * 8, p0 = (c >> 5) * 128 + (u.t0 >> 3) * 32 + (c & 31), half = u.t0 & 4;
#pragma unroll
    for (int i = 0; i < 8; ++i) *(uint2*)(at(p0 + i) + half * 2) = v[i];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    const int64_t cb = (u.c - c) >> 5;
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (cb + (r >> 1) < blocks) *(u32x4*)(out + operand_offset(u.mb, cb, blocks) + r * 1024 + lane * 16) = *(const u32x4*)at(r * 64 + lane);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// The powers of two that dz (z) and dz alpha (za) are multiplied by on their way to float16.  dz and alpha may be of any size (a
// gradient without a loss scale is 1e-5, alpha 1 / sqrt(K)), and float16 has its 11 bits from 2^-14 on only: the largest dy is brought
// to 2^14 .. 2^15, which a slope (at most 1.13) leaves finite, and the largest alpha to 1/2 .. 1.  Then what is 2^-28 of the largest still has
// all its bits.  The products are exact in these factors, and the sums are divided by them (unit: 2^-z, 2^-za) in fp32.
struct GradUnits {
    float z = 1.f, za = 1.f, unit = 1.f, unit_a = 1.f;
    // What a lane takes of the parts: fetched here, looked at in `reduce`, behind the loads that do not depend on it
    uint4 q[kRangeParts / 256];
    unsigned al;
    __device__ __forceinline__ void fetch(const unsigned* range, int parts)
    {
        const int lane = threadIdx.x & 63;
        al = range[kRangeParts + lane];
#pragma unroll
        for (int i = 0; i < kRangeParts / 256; ++i)  // (past the last part: the first ones again)
            q[i] = *(const uint4*)(range + (256 * i < parts ? 256 * i : 0) + 4 * lane);
    }
    __device__ __forceinline__ void reduce()
    {
        unsigned m[2] = {0, al};
#pragma unroll
        for (int i = 0; i < kRangeParts / 256; ++i) {
            const unsigned a = q[i].x > q[i].y ? q[i].x : q[i].y, b = q[i].z > q[i].w ? q[i].z : q[i].w, c = a > b ? a : b;
            m[0] = c > m[0] ? c : m[0];
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const unsigned o = (unsigned)__shfl_xor((int)m[k], d);
                m[k] = o > m[k] ? o : m[k];
            }
        const unsigned top = __float_as_uint(F16::to_float((unsigned short)m[0]));
        const int s = top && top < 0x7f800000u ? 14 - ((int)(top >> 23) - 127) : 0;  // -1 .. 38
        int p = m[1] && m[1] < 0x7f800000u ? 126 - (int)(m[1] >> 23) : 0;            // (a subnormal alpha counts as 2^-127)
        p = p > 126 - s ? 126 - s : p < -126 - s ? -126 - s : p;                     // both 2^(s + p) and its inverse are normal
        z = power(s), za = power(s + p), unit = power(-s), unit_a = power(-s - p);
    }
    static __device__ __forceinline__ float power(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }
};

template <class T, int ACT, bool UNITS>
__device__ __forceinline__ void grad_unit(const GradArgs& a, int64_t tb0, int64_t strip, char* lds)
{
    const int64_t nb = (a.N + 31) / 32, tbs = operand_blocks(a.M);
    const CkptShape cs(a.M, a.N);
    float sum[8], al[8];
    GradUnits units;
    if constexpr (UNITS) units.fetch(a.range, a.parts);
    const int64_t c = micro_of(0, strip).c;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        sum[i] = 0.f;
        al[i] = c + i < a.N ? (a.alpha.ptr ? a.alpha.ptr[c + i] : 1.f) : 0.f;
    }
    for (int64_t mb = tb0; mb < tb0 + a.per && mb < tbs; ++mb) {
        const Micro u = micro_of(mb, strip);
        u32x4 v[kTok];
#pragma unroll
        for (int t = 0; t < kTok; ++t) v[t] = load_row((const unsigned short*)a.dy, a.lddy, mb * 32 + u.t0 + t, a.M, u.c, a.N);
        MicroCkpt k;
        if constexpr (ACT != kActNone) {
            if (u.c < a.N && mb < cs.tb)
                k.load(a.zq, cs, u);
            else
                k.zero();
        }
        if (UNITS && mb == tb0) {
            units.reduce();
            const bool vector = a.alpha.ptr;
            const float as = vector ? units.za : units.z;
#pragma unroll
            for (int i = 0; i < 8; ++i) al[i] *= as;
            if (blockIdx.x == 0 && threadIdx.x == 0) {
                float* unit = (float*)(a.range + kRangeParts + 64);
                unit[0] = units.unit, unit[1] = vector ? units.unit_a : units.unit;
            }
        }
        unsigned o[8][kTok / 2];
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[i] = half_of<T>(v[t][i >> 1], i & 1);
                if constexpr (ACT != kActNone) {
                    // a group that held an infinity or NaN makes the slopes of its real tokens NaN, not those past the end
                    const float g = d[i] * act_slope<ACT>(k.code(t, i) * k.scale(i));
                    d[i] = mb * 32 + u.t0 + t < a.M ? g : 0.f;
                }
                sum[i] += d[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const unsigned b = ACT == kActNone ? v[t][i >> 1] >> (16 * (i & 1)) & 0xffffu : (unsigned)T::from_float(d[i] * units.z);
                o[i][t >> 1] = t & 1 ? o[i][t >> 1] | b << 16 : b;
            }
            const int64_t m = mb * 32 + u.t0 + t;
            if (a.dza && m < a.M && u.c < a.lda)
                *(u32x4*)((unsigned short*)a.dza + m * a.lda + u.c) =
                    u32x4{pack2<T>(d[0] * al[0], d[1] * al[1]), pack2<T>(d[2] * al[2], d[3] * al[3]), pack2<T>(d[4] * al[4], d[5] * al[5]),
                          pack2<T>(d[6] * al[6], d[7] * al[7])};
        }
        if (a.dzt) {
            uint2 w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = make_uint2(o[i][0], o[i][1]);
            store_operand(a.dzt, nb, u, w, lds);
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        sum[i] += __shfl_xor(sum[i], 8);
        sum[i] += __shfl_xor(sum[i], 16);
        sum[i] += __shfl_xor(sum[i], 32);
    }
    const int64_t row = tb0 / a.per;
    if ((threadIdx.x & 63) < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < a.N) a.part[row * a.N + c + i] = sum[i];
}

// The layer's input from its checkpoint in operand order, 32 tokens x 64 channels of it
template <class T>
__device__ __forceinline__ void x_unit(const GradArgs& a, int64_t unit, char* lds)
{
    const int64_t mb = unit / a.x_strips;
    const Micro u = micro_of(mb, unit - mb * a.x_strips);
    const int64_t kb = (a.K + 31) / 32;
    const CkptShape cs(a.M, a.K);
    MicroCkpt k;
    if (u.c < a.K && mb < cs.tb)
        k.load(a.xq, cs, u);
    else
        k.zero();
    uint2 o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float s = k.scale(i);
        unsigned w[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int64_t m = mb * 32 + u.t0 + 2 * t;
            w[t] = pack2<T>(m < a.M ? k.code(2 * t, i) * s : 0.f, m + 1 < a.M ? k.code(2 * t + 1, i) * s : 0.f);
        }
        o[i] = make_uint2(w[0], w[1]);
    }
    store_operand(a.xt, kb, u, o, lds);
}

// float16: the largest magnitudes of dy (a block each of `parts`, its waves over units of 32 tokens x 64 channels) and of alpha (the first
// 64 blocks), every part written; and beside them, in the blocks behind, the input in operand order, which needs neither.  Without this
// launch, dx of a gradient of 1e-5 is off by 11 % at K = N = 4096.  It makes the backward pass 15 -> 18.5 us at 256 x 1024 x 1024, 37 -> 42
// at 1000 x 1003 x 2187, 265 -> 275 at 4096^3 and 3210 -> 3270 at 16384 x 8192 x 8192; bfloat16 needs none of it.
__global__ __launch_bounds__(256) void k_grad_range(GradArgs a)
{
    __shared__ __attribute__((aligned(16))) char smem[4 * 4096];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if ((int)blockIdx.x >= a.parts) {
        const int64_t unit = (int64_t)((int)blockIdx.x - a.parts) * 4 + wave;
        if (unit < a.x_units) x_unit<F16>(a, unit, smem + wave * 4096);
        return;
    }
    const int64_t units = (a.M + 31) / 32 * a.dz_strips;
    unsigned top = 0, al = 0;  // as bits: a NaN is larger than an infinity, and that than any number
    for (int64_t unit = (int64_t)wave * a.parts + blockIdx.x; unit < units; unit += 4 * a.parts) {
        const int64_t mb = unit / a.dz_strips;
        const Micro u = micro_of(mb, unit - mb * a.dz_strips);
        u32x4 v[kTok];
#pragma unroll
        for (int t = 0; t < kTok; ++t) v[t] = load_row((const unsigned short*)a.dy, a.lddy, mb * 32 + u.t0 + t, a.M, u.c, a.N);
#pragma unroll
        for (int t = 0; t < kTok; ++t)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const unsigned b = (v[t][i >> 1] >> (16 * (i & 1))) & 0x7fffu;
                top = b > top ? b : top;
            }
    }
    if (blockIdx.x < 64 && a.alpha.ptr)
        for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < a.N; n += 64 * 256) {
            const unsigned b = __float_as_uint(a.alpha.ptr[n]) & 0x7fffffffu;
            al = b > al ? b : al;
        }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const unsigned o = (unsigned)__shfl_xor((int)top, d), p = (unsigned)__shfl_xor((int)al, d);
        top = o > top ? o : top;
        al = p > al ? p : al;
    }
    unsigned* tops = (unsigned*)smem;  // [2][4]
    if (lane == 0) tops[wave] = top, tops[4 + wave] = al;
    __syncthreads();
    if (threadIdx.x >= 2 || (threadIdx.x == 1 && blockIdx.x >= 64)) return;
    unsigned m = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) m = tops[threadIdx.x * 4 + w] > m ? tops[threadIdx.x * 4 + w] : m;
    a.range[threadIdx.x * kRangeParts + blockIdx.x] = m;
}

// The gradient before the activation, dz = dy act'(z^), as the two products take it: row-major, times an alpha per output (dx), and in
// operand order (dw); its sums over a run of tokens (dbias), in fp32 throughout; and the layer's input from its checkpoint in operand order.
// Both forms of dz are rounded to T here, for the matrix cores take 16-bit operands: one rounding of u a term beside the one of the
// result.  (dz without an activation is dy and is not rounded, and one alpha for all outputs is left to the product's epilogue.)
template <class T, bool UNITS>
__global__ __launch_bounds__(256) void k_linear_grad(GradArgs a)
{
    __shared__ __attribute__((aligned(16))) char smem[4 * 4096];
    char* lds = smem + (threadIdx.x >> 6) * 4096;  // of this wave
    int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit < a.dz_units) {
        const int64_t run = unit / a.dz_strips, strip = unit - run * a.dz_strips, tb0 = run * a.per;
        if (a.act == kActNone)
            grad_unit<T, kActNone, UNITS>(a, tb0, strip, lds);
        else if (a.act == kActRelu)
            grad_unit<T, kActRelu, UNITS>(a, tb0, strip, lds);
        else if (a.act == kActGelu)
            grad_unit<T, kActGelu, UNITS>(a, tb0, strip, lds);
        else
            grad_unit<T, kActSilu, UNITS>(a, tb0, strip, lds);
        return;
    }
    unit -= a.dz_units;
    if (unit >= a.x_units) return;
    x_unit<T>(a, unit, lds);
}

}  // namespace

hipError_t launch_checkpoint_pack(const CkptArgs& a, hipStream_t st)
{
    const int64_t strips = (a.C + kStrip - 1) / kStrip, blocks = ((a.M + 31) / 32 * strips + 3) / 4;
    if (a.f16)
        k_ckpt_pack<F16><<<(unsigned)blocks, 256, 0, st>>>(a, (int)strips);
    else
        k_ckpt_pack<BF16><<<(unsigned)blocks, 256, 0, st>>>(a, (int)strips);
    return hipGetLastError();
}

hipError_t launch_checkpoint_unpack(const CkptArgs& a, hipStream_t st)
{
    const int64_t strips = (a.C + kStrip - 1) / kStrip, blocks = ((a.M + 31) / 32 * strips + 3) / 4;
    if (a.f16)
        k_ckpt_unpack<F16><<<(unsigned)blocks, 256, 0, st>>>(a, (int)strips);
    else
        k_ckpt_unpack<BF16><<<(unsigned)blocks, 256, 0, st>>>(a, (int)strips);
    return hipGetLastError();
}

hipError_t launch_linear_grad(GradArgs a, int f16, hipStream_t st)
{
    const int64_t tbs = operand_blocks(a.M);
    a.dz_strips = a.dzt || a.dza || a.part ? (a.N + kStrip - 1) / kStrip : 0;
    a.dz_units = (tbs + a.per - 1) / a.per * a.dz_strips;
    a.x_strips = a.xt ? (a.K + kStrip - 1) / kStrip : 0;
    a.x_units = tbs * a.x_strips;
    if (a.range) {
        const int64_t want = (a.M + 31) / 32 * a.dz_strips / 4;  // a unit a wave, up to 4096 waves
        a.parts = want >= kRangeParts ? kRangeParts : want <= 256 ? 256 : (int)((want + 255) / 256 * 256);
        k_grad_range<<<(unsigned)(a.parts + (a.x_units + 3) / 4), 256, 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.x_units = 0;
    }
    const int64_t blocks = (a.dz_units + a.x_units + 3) / 4;
    if (!blocks) return hipSuccess;
    if (f16 && a.range)
        k_linear_grad<F16, true><<<(unsigned)blocks, 256, 0, st>>>(a);
    else if (f16)
        k_linear_grad<F16, false><<<(unsigned)blocks, 256, 0, st>>>(a);
    else
        k_linear_grad<BF16, false><<<(unsigned)blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace rtn
