// Microscaled 4-bit packing (Mx4Shape), along the rows or along rows and columns in one pass, and back.  One pass over memory each.
#include "mx4_math.h"
#include "rtn_kernels.h"

namespace rtn {

namespace {

// The larger of the four lanes of a quad, in all of them
__device__ __forceinline__ unsigned quad_larger(unsigned a)
{
    a = larger(a, (unsigned)__builtin_amdgcn_update_dpp(0, (int)a, 0xB1, 0xf, 0xf, true));  // lanes 1 0 3 2
    return larger(a, (unsigned)__builtin_amdgcn_update_dpp(0, (int)a, 0x4E, 0xf, 0xf, true));  // lanes 2 3 0 1
}
__device__ __forceinline__ unsigned largest8(const float (&v)[8])
{
    Largest a;
#pragma unroll
    for (int i = 0; i < 8; i += 2) a.take(v[i], v[i + 1]);
    return a.bits();
}

// Eight values that are all there
template <class T>
__device__ __forceinline__ void load_whole(const char* p, float (&v)[8])
{
    if constexpr (std::is_same_v<T, F32>) {
        __builtin_memcpy(v, p, 32);
    } else {
        const u32x4 q = load16(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = half_of<T>(q[i >> 1], i & 1);
    }
}

template <class T>
__device__ __forceinline__ float load_one(const void* p, int64_t i)
{
    if constexpr (std::is_same_v<T, F32>)
        return ((const float*)p)[i];
    else
        return T::to_float(((const unsigned short*)p)[i]);
}

// Along the rows alone.  A block has 64 rows x 128 columns, a wave 16 rows, a lane 8 columns of a row: four lanes have a group, 16 read
// 256 bytes of a row (of 16-bit values), and the maximum is over a quad of lanes.
// 16384 x 8192 of bfloat16: 64 us, 5.3 TB/s of what is read and written, stochastic 77, bound by the vector unit; a few rows 3.6 us, the launch
// and one round of loads.
template <class T, bool RANDOM>
__global__ __launch_bounds__(256) void k_mx4_rows(Mx4PackArgs a)
{
    __shared__ unsigned scales[64];
    const Mx4Shape s(a.R, a.C);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, p = lane & 3, g = (lane >> 2) & 3;
    const int64_t kb = (int64_t)blockIdx.x % s.kb, rg = (int64_t)blockIdx.x / s.kb, rb = rg * 4 + wave;
    const int64_t c = kb * 128 + g * 32 + p * 8, groups = (a.C + 31) / 32;
    const uint64_t seed = RANDOM ? *a.seed : 0;
    float v[4][8];
    const bool whole = kb * 128 + 128 <= a.C && rg * 64 + 64 <= a.R;
    if (whole) {
        const char* x = (const char*)a.x + ((rb * 16 + (lane >> 4)) * a.ldx + c) * kBytesOf<T>;
#pragma unroll
        for (int i = 0; i < 4; ++i) load_whole<T>(x + i * 4 * a.ldx * kBytesOf<T>, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = rb * 16 + i * 4 + (lane >> 4);
        if (whole) break;
        if (r < a.R) {
            load_values<T>((const char*)a.x + r * a.ldx * kBytesOf<T>, c, a.C, v[i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 4 + (lane >> 4), e = mx4_scale(quad_larger(largest8(v[i])), RANDOM);
        const Mx4Random rnd = {seed, (uint64_t)((rb * 16 + row) * groups + kb * 4 + g), 0};
        const unsigned q = RANDOM ? mx4_stochastic(v[i], e, rnd.bits(p)) : mx4_nearest(v[i], e);
        if (rb < s.rb) *(unsigned*)((char*)a.out + (rb * s.kb + kb) * 1024 + (row + 16 * g) * 16 + p * 4) = q;
        if (p == 0) ((unsigned char*)scales)[(row + 16 * g) * 4 + wave] = (unsigned char)e;
    }
    __syncthreads();
    if (wave == 0) *(unsigned*)((char*)a.out + s.codes() + (rg * s.kb + kb) * 256 + lane * 4) = scales[lane];
}

// phi'(z) of gelu or silu for the gradient that is packed: to fp32's accuracy, since a packed value next to the border of two codes takes the one or
// the other.  z may be an infinity (float16 rounds what is beyond its range to one): the factor that is z itself is held to where the other
// one is 0 already, so that the slopes there are 0 and 1.  (A NaN comes through erfcf and expf.)
template <int ACT>
__device__ __forceinline__ float exact_slope(float z)
{
    const float held = __builtin_amdgcn_fmed3f(z, -128.f, 128.f);
    if constexpr (ACT == kActGelu) {
        return 0.5f * erfcf(z * -0.70710678f) + held * 0.39894228f * expf(-0.5f * z * z);
    } else {
        static_assert(ACT == kActSilu, "");
        const float s = 1.f / (1.f + expf(-z));
        return s * (1.f + held * (1.f - s));
    }
}
// dy phi'(z).  Where a relu is off dy is dropped, not multiplied: 0 times an infinity or NaN is no 0, and one NaN takes its groups' other 31 values
// in both packings with it.
template <int ACT>
__device__ __forceinline__ float act_gradient(float dy, float z)
{
    if constexpr (ACT == kActRelu)
        return z > 0.f ? dy : z == z ? 0.f : z;
    else
        return dy * exact_slope<ACT>(z);
}

// Along the rows and along the columns.  A block has 64 rows x 64 columns: the rows' groups as above, straight from the registers; the
// columns' through LDS as fp32, after which a lane has one group of 32 rows.  Two blocks beside or below each other fill a piece of
// 1 KiB of codes and 256 bytes of scales, each in whole 128-byte lines; the last of an odd number fills its neighbour's half with zeros.
// The sums of the columns (the bias gradient) come on the way, 64 rows each.
// To nearest bound by memory, 4096 x 4096 of bfloat16 13.6 us, of float32 16 us (5.3 TB/s); stochastic by the vector unit, whose random numbers
// are 40 instructions for 8 values and direction: 16384 x 8192 153 us, 93 % of its issue slots.  (Blocks of 128 x 128: 256 x 1024 17.5 us
// instead of 7.7, for want of blocks.)  Behind an activation z is read too and its slope formed for every element: relu 172 us, silu 260, gelu
// 393 to 424, whose erfcf and expf are the most of that; at 4096 x 4096 silu 40, gelu 58.
template <class T, int ACT, bool RANDOM>
__global__ __launch_bounds__(128, 4) void k_mx4_both(Mx4PackArgs a)
{
    __shared__ __attribute__((aligned(16))) float tile[64][64];
    __shared__ unsigned srow[32], scol[32];
    __shared__ float sums[64];
    const Mx4Shape s(a.R, a.C), st(a.C, a.R);
    const unsigned tid = threadIdx.x, p = tid & 3, g = (tid >> 2) & 1, rr = tid >> 3, c8 = (tid & 7) * 8, tc = tid & 63, half = tid >> 6;
    const unsigned cbs = (unsigned)((a.C + 63) / 64), rbs = (unsigned)((a.R + 63) / 64), tb = blockIdx.x / cbs, cb = blockIdx.x - tb * cbs;
    const uint64_t seed = RANDOM ? *a.seed : 0;
    float v[4][8];
    if (cb * 64 + 64 <= a.C && tb * 64 + 64 <= a.R) {
        const char* x = (const char*)a.x + (((int64_t)tb * 64 + rr) * a.ldx + cb * 64 + c8) * kBytesOf<T>;
#pragma unroll
        for (int i = 0; i < 4; ++i) load_whole<T>(x + i * 16 * a.ldx * kBytesOf<T>, v[i]);
        if constexpr (ACT != kActNone) {
            const char* zs = (const char*)a.z + (((int64_t)tb * 64 + rr) * a.ldz + cb * 64 + c8) * kBytesOf<T>;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float z[8];
                load_whole<T>(zs + i * 16 * a.ldz * kBytesOf<T>, z);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = act_gradient<ACT>(v[i][e], z[e]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float4* t = (float4*)&tile[i * 16 + rr][c8];
            t[0] = make_float4(v[i][0], v[i][1], v[i][2], v[i][3]), t[1] = make_float4(v[i][4], v[i][5], v[i][6], v[i][7]);
        }
        __syncthreads();
    } else {  // at the matrix' ends: through LDS one by one
#pragma unroll 1
        for (unsigned i = half; i < 64; i += 2) {
            const int64_t r = (int64_t)tb * 64 + i, c = (int64_t)cb * 64 + tc;
            float f = 0.f;
            if (r < a.R && c < a.C) {
                f = load_one<T>(a.x, r * a.ldx + c);
                if constexpr (ACT != kActNone) f = act_gradient<ACT>(f, load_one<T>(a.z, r * a.ldz + c));
            }
            tile[i][tc] = f;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4* t = (const float4*)&tile[i * 16 + rr][c8];
            const float4 l = t[0], h = t[1];
            v[i][0] = l.x, v[i][1] = l.y, v[i][2] = l.z, v[i][3] = l.w, v[i][4] = h.x, v[i][5] = h.y, v[i][6] = h.z, v[i][7] = h.w;
        }
    }
    if (a.out) {
        const unsigned gr = (cb & 1) * 2 + g;  // the group in its block of 128 columns
        char* out = (char*)a.out + (tb * 4 * s.kb + (cb >> 1)) * 1024;
        uint64_t group = ((uint64_t)tb * 64 + rr) * (uint64_t)((a.C + 31) / 32) + cb * 2 + g;
#pragma unroll
        for (unsigned i = 0; i < 4; ++i) {
            const int e = mx4_scale(quad_larger(largest8(v[i])), RANDOM);
            const Mx4Random rnd = {seed, group, 0};
            const unsigned q = RANDOM ? mx4_stochastic(v[i], e, rnd.bits((int)p)) : mx4_nearest(v[i], e);
            if (tb * 4 + i < s.rb) *(unsigned*)(out + i * s.kb * 1024 + ((rr + 16 * gr) * 16 + p * 4)) = q;
            if (p == 0) ((unsigned char*)srow)[(rr + 16 * g) * 4 + i] = (unsigned char)e;
            group += 16 * (uint64_t)((a.C + 31) / 32);
        }
    }
    const unsigned kt = tb >> 1;  // the block of 128 rows
    if (a.out_t || a.part) {
        float w[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) w[i] = tile[half * 32 + i][tc];
        if (a.part) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) sum += w[i];
            if (half) sums[tc] = sum;
            __syncthreads();
            if (!half && cb * 64 + tc < a.C) a.part[tb * a.C + cb * 64 + tc] = sum + sums[tc];
        }
        if (a.out_t) {
            Largest m;
#pragma unroll
            for (int i = 0; i < 32; i += 2) m.take(w[i], w[i + 1]);
            const int e = mx4_scale(m.bits(), RANDOM);
            const unsigned gt = (tb & 1) * 2 + half, b = cb * 4 + (tc >> 4);
            const Mx4Random rnd = {seed, ((uint64_t)cb * 64 + tc) * (uint64_t)((a.R + 31) / 32) + tb * 2 + half, 1};
            unsigned q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) q[j] = RANDOM ? mx4_stochastic(w + 8 * j, e, rnd.bits(j)) : mx4_nearest(w + 8 * j, e);
            if (b < st.rb) *(uint4*)((char*)a.out_t + (b * st.kb + kt) * 1024 + ((tc & 15) + 16 * gt) * 16) = make_uint4(q[0], q[1], q[2], q[3]);
            ((unsigned char*)scol)[((tc & 15) + 16 * half) * 4 + (tc >> 4)] = (unsigned char)e;
        }
    }
    __syncthreads();
    const unsigned l = tid & 31, i = tid >> 5;
    // the second half of a block of 128 columns or rows that has none: codes and scales of groups that are not there
    const bool lone_c = cb == cbs - 1 && !(cb & 1), lone_r = tb == rbs - 1 && !(tb & 1);
    if (a.out) {
        unsigned* scales = (unsigned*)((char*)a.out + s.codes() + (tb * s.kb + (cb >> 1)) * 256) + l;
        if (i == 0) scales[(cb & 1) * 32] = srow[l];
        if (lone_c) {
            if (i == 1) scales[32] = 0;
            if (tb * 4 + i < s.rb) *(uint4*)((char*)a.out + ((tb * 4 + i) * s.kb + (cb >> 1)) * 1024 + 512 + l * 16) = make_uint4(0, 0, 0, 0);
        }
    }
    if (a.out_t) {
        unsigned* scales = (unsigned*)((char*)a.out_t + st.codes() + (cb * st.kb + kt) * 256) + l;
        if (i == 2) scales[(tb & 1) * 32] = scol[l];
        if (lone_r) {
            if (i == 3) scales[32] = 0;
            if (cb * 4 + i < st.rb) *(uint4*)((char*)a.out_t + ((cb * 4 + i) * st.kb + kt) * 1024 + 512 + l * 16) = make_uint4(0, 0, 0, 0);
        }
    }
}

// A quad of lanes has a group, 16 lanes 256 bytes of a row.  16384 x 8192 to bfloat16: 54 us, 6.3 TB/s.
template <class T>
__global__ __launch_bounds__(256) void k_mx4_unpack(Mx4UnpackArgs a)
{
    const Mx4Shape s(a.R, a.C);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, p = lane & 3, g = (lane >> 2) & 3;
    const int64_t kb = (int64_t)blockIdx.x % s.kb, rg = (int64_t)blockIdx.x / s.kb, rb = rg * 4 + wave;
    if (rb >= s.rb) return;
    const int64_t c = kb * 128 + g * 32 + p * 8;
    unsigned q[4], e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int l = i * 4 + (lane >> 4) + 16 * g;
        q[i] = *(const unsigned*)((const char*)a.packed + (rb * s.kb + kb) * 1024 + l * 16 + p * 4);
        e[i] = *((const unsigned char*)a.packed + s.codes() + (rg * s.kb + kb) * 256 + l * 4 + wave);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = rb * 16 + i * 4 + (lane >> 4);
        if (r >= a.R || c >= a.C) continue;
        float v[8];
        mx4_values(q[i], v);
        const float f = mx4_factor((int)e[i]);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= f;
        if constexpr (std::is_same_v<T, F32>) {
            float* y = (float*)a.y + r * a.ldy + c;
            if (c + 8 <= a.C) {
                __builtin_memcpy(y, v, 32);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < a.C) y[k] = v[k];
            }
        } else {
            unsigned short* y = (unsigned short*)a.y + r * a.ldy + c;
            if (c + 8 <= a.C) {
                store16(y, u32x4{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])});
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < a.C) y[k] = T::from_float(v[k]);
            }
        }
    }
}

// out[c] = sum over runs of part[run][c]: 64 columns a block, its 16 waves share the runs
template <class T>
__global__ __launch_bounds__(1024) void k_mx4_sums(const float* part, int64_t runs, int64_t C, unsigned short* out)
{
    __shared__ float lds[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.f;
    if (c < C)
        for (int64_t r = wave; r < runs; r += 16) s += part[r * C + c];
    lds[wave][lane] = s;
    __syncthreads();
    if (wave || c >= C) return;
    for (int v = 1; v < 16; ++v) s += lds[v][lane];
    out[c] = T::from_float(s);
}

template <class T>
hipError_t run_rows(const Mx4PackArgs& a, unsigned grid, hipStream_t st)
{
    if (a.seed)
        k_mx4_rows<T, true><<<grid, 256, 0, st>>>(a);
    else
        k_mx4_rows<T, false><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}
template <class T, int ACT>
hipError_t run_both(const Mx4PackArgs& a, unsigned grid, hipStream_t st)
{
    if (a.seed)
        k_mx4_both<T, ACT, true><<<grid, 128, 0, st>>>(a);
    else
        k_mx4_both<T, ACT, false><<<grid, 128, 0, st>>>(a);
    return hipGetLastError();
}
template <class T>
hipError_t run_both(const Mx4PackArgs& a, unsigned grid, hipStream_t st)
{
    switch (a.act) {
        case kActNone: return run_both<T, kActNone>(a, grid, st);
        case kActRelu: return run_both<T, kActRelu>(a, grid, st);
        case kActGelu: return run_both<T, kActGelu>(a, grid, st);
        default: return run_both<T, kActSilu>(a, grid, st);
    }
}

}  // namespace

int64_t mx4_sum_runs(int64_t R) { return (R + 63) / 64; }

hipError_t launch_mx4_pack(const Mx4PackArgs& a, hipStream_t st)
{
    const Mx4Shape s(a.R, a.C);
    if (!a.out_t && !a.part && a.act == kActNone) {
        const int64_t n = s.rg * s.kb;
        if (n > 0x7fffffff) return hipErrorInvalidValue;
        return a.type == 2 ? run_rows<F32>(a, (unsigned)n, st) : a.type == 1 ? run_rows<F16>(a, (unsigned)n, st) : run_rows<BF16>(a, (unsigned)n, st);
    }
    const int64_t n = (a.C + 63) / 64 * ((a.R + 63) / 64);
    if (n > 0x7fffffff) return hipErrorInvalidValue;
    if (a.type == 2) return run_both<F32, kActNone>(a, (unsigned)n, st);
    return a.type == 1 ? run_both<F16>(a, (unsigned)n, st) : run_both<BF16>(a, (unsigned)n, st);
}

hipError_t launch_mx4_unpack(const Mx4UnpackArgs& a, hipStream_t st)
{
    const Mx4Shape s(a.R, a.C);
    const int64_t n = s.rg * s.kb;
    if (n > 0x7fffffff) return hipErrorInvalidValue;
    if (a.type == 2)
        k_mx4_unpack<F32><<<(unsigned)n, 256, 0, st>>>(a);
    else if (a.type == 1)
        k_mx4_unpack<F16><<<(unsigned)n, 256, 0, st>>>(a);
    else
        k_mx4_unpack<BF16><<<(unsigned)n, 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_mx4_sums(const float* part, int64_t R, int64_t C, void* out, int f16, hipStream_t st)
{
    const unsigned grid = (unsigned)((C + 63) / 64);
    if (f16)
        k_mx4_sums<F16><<<grid, 1024, 0, st>>>(part, mx4_sum_runs(R), C, (unsigned short*)out);
    else
        k_mx4_sums<BF16><<<grid, 1024, 0, st>>>(part, mx4_sum_runs(R), C, (unsigned short*)out);
    return hipGetLastError();
}

}  // namespace rtn
