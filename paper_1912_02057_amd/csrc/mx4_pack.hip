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
    unsigned a = magnitude(v[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) a = larger(a, magnitude(v[i]));
    return a;
}

// Along the rows alone.  A block has 64 rows x 128 columns, a wave 16 rows, a lane 8 columns of a row: four lanes have a group, 16 read
// 256 bytes of a row (of 16-bit values), and the maximum is over a quad of lanes.
template <class T>
__global__ __launch_bounds__(256) void k_mx4_rows(Mx4PackArgs a)
{
    __shared__ unsigned scales[64];
    const Mx4Shape s(a.R, a.C);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, p = lane & 3, g = (lane >> 2) & 3;
    const int64_t kb = (int64_t)blockIdx.x % s.kb, rg = (int64_t)blockIdx.x / s.kb, rb = rg * 4 + wave;
    const int64_t c = kb * 128 + g * 32 + p * 8, groups = (a.C + 31) / 32;
    const uint64_t seed = a.seed ? *a.seed : 0;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = rb * 16 + i * 4 + (lane >> 4);
        if (r < a.R) {
            load_values<T>((const char*)a.x + r * a.ldx * kBytesOf<T>, c, a.C, v[i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 4 + (lane >> 4), e = mx4_scale(quad_larger(largest8(v[i])), a.seed != nullptr);
        const Mx4Random rnd = {seed, (uint64_t)((rb * 16 + row) * groups + kb * 4 + g), 0};
        const unsigned q = a.seed ? mx4_stochastic(v[i], e, rnd.bits(p)) : mx4_nearest(v[i], e);
        if (rb < s.rb) *(unsigned*)((char*)a.out + (rb * s.kb + kb) * 1024 + (row + 16 * g) * 16 + p * 4) = q;
        if (p == 0) ((unsigned char*)scales)[(row + 16 * g) * 4 + wave] = (unsigned char)e;
    }
    __syncthreads();
    if (wave == 0) *(unsigned*)((char*)a.out + s.codes() + (rg * s.kb + kb) * 256 + lane * 4) = scales[lane];
}

// phi'(z) for the gradient that is packed: to fp32's accuracy, since a packed value next to the border of two codes takes the one or
// the other.
template <int ACT>
__device__ __forceinline__ float exact_slope(float z)
{
    if constexpr (ACT == kActGelu) {
        return 0.5f * erfcf(z * -0.70710678f) + z * 0.39894228f * expf(-0.5f * z * z);
    } else if constexpr (ACT == kActSilu) {
        const float s = 1.f / (1.f + expf(-z));
        return s * (1.f + z * (1.f - s));
    } else {
        return act_slope<ACT>(z);
    }
}

// Along the rows and along the columns.  A block has 128 rows x 128 columns, 64 rows at a time: the rows' groups as above, straight from
// the registers; the columns' through LDS as fp32, after which a lane has one group of 32 rows.  Both scales are whole 256-byte
// pieces.  The sums of the columns (the bias gradient) come on the way; a block then has `per` tiles below each other.
template <class T, int ACT>
__global__ __launch_bounds__(256) void k_mx4_both(Mx4PackArgs a)
{
    __shared__ __attribute__((aligned(16))) float tile[64][128];
    __shared__ unsigned srow[2][64], scol[2][64];
    __shared__ float sums[128];
    const Mx4Shape s(a.R, a.C), st(a.C, a.R);
    const int tid = threadIdx.x, p = tid & 3, g = (tid >> 2) & 3, rr = tid >> 4, tc = tid & 127, half = tid >> 7;
    const int64_t cbs = s.kb, cb = (int64_t)blockIdx.x % cbs, run = (int64_t)blockIdx.x / cbs;
    const int64_t c = cb * 128 + (tid & 15) * 8, groups = (a.C + 31) / 32, groups_t = (a.R + 31) / 32;
    const uint64_t seed = a.seed ? *a.seed : 0;
    float sum = 0.f;
    for (int64_t tb = run * a.per; tb < (run + 1) * a.per && tb < st.kb; ++tb) {
#pragma unroll 1
        for (int sub = 0; sub < 2; ++sub) {
            const int64_t row0 = tb * 128 + sub * 64;
            float v[4][8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t r = row0 + i * 16 + rr;
                if (r < a.R) {
                    load_values<T>((const char*)a.x + r * a.ldx * kBytesOf<T>, c, a.C, v[i]);
                    if constexpr (ACT != kActNone) {
                        float z[8];
                        load_values<T>((const char*)a.z + r * a.ldz * kBytesOf<T>, c, a.C, z);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[i][e] = c + e < a.C ? v[i][e] * exact_slope<ACT>(z[e]) : 0.f;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float4* t = (float4*)&tile[i * 16 + rr][(tid & 15) * 8];
                t[0] = make_float4(v[i][0], v[i][1], v[i][2], v[i][3]), t[1] = make_float4(v[i][4], v[i][5], v[i][6], v[i][7]);
            }
            if (a.out) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int64_t rb = row0 / 16 + i;
                    const int e = mx4_scale(quad_larger(largest8(v[i])), a.seed != nullptr);
                    const Mx4Random rnd = {seed, (uint64_t)((rb * 16 + rr) * groups + cb * 4 + g), 0};
                    const unsigned q = a.seed ? mx4_stochastic(v[i], e, rnd.bits(p)) : mx4_nearest(v[i], e);
                    if (rb < s.rb) *(unsigned*)((char*)a.out + (rb * s.kb + cb) * 1024 + (rr + 16 * g) * 16 + p * 4) = q;
                    if (p == 0) ((unsigned char*)srow[sub])[(rr + 16 * g) * 4 + i] = (unsigned char)e;
                }
            }
            __syncthreads();
            if (a.out_t || a.part) {
                float w[32];
                unsigned m = 0;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    w[i] = tile[half * 32 + i][tc];
                    m = larger(m, magnitude(w[i]));
                }
                if (a.part) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) sum += w[i];
                }
                if (a.out_t) {
                    const int e = mx4_scale(m, a.seed != nullptr), gt = sub * 2 + half;
                    const Mx4Random rnd = {seed, (uint64_t)((cb * 128 + tc) * groups_t + tb * 4 + gt), 1};
                    unsigned q[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) q[j] = a.seed ? mx4_stochastic(w + 8 * j, e, rnd.bits(j)) : mx4_nearest(w + 8 * j, e);
                    const int64_t b = cb * 8 + (tc >> 4);
                    if (b < st.rb) *(uint4*)((char*)a.out_t + (b * st.kb + tb) * 1024 + ((tc & 15) + 16 * gt) * 16) = make_uint4(q[0], q[1], q[2], q[3]);
                    ((unsigned char*)scol[tc >> 6])[((tc & 15) + 16 * gt) * 4 + ((tc >> 4) & 3)] = (unsigned char)e;
                }
            }
            __syncthreads();
        }
        const int which = (tid >> 6) & 1, l = tid & 63;
        if (tid < 128) {
            const int64_t rg = tb * 2 + which;
            if (a.out && rg < s.rg) *(unsigned*)((char*)a.out + s.codes() + (rg * s.kb + cb) * 256 + l * 4) = srow[which][l];
        } else {
            const int64_t rg = cb * 2 + which;
            if (a.out_t && rg < st.rg) *(unsigned*)((char*)a.out_t + st.codes() + (rg * st.kb + tb) * 256 + l * 4) = scol[which][l];
        }
        // (the next tile's scales are written behind a barrier that these reads come before)
    }
    if (a.part) {
        if (half) sums[tc] = sum;
        __syncthreads();
        if (!half && cb * 128 + tc < a.C) a.part[run * a.C + cb * 128 + tc] = sum + sums[tc];
    }
}

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

// out[c] = sum over runs of part[run][c], in their order
template <class T>
__global__ __launch_bounds__(256) void k_mx4_sums(const float* part, int64_t runs, int64_t C, unsigned short* out)
{
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= C) return;
    float s = 0.f;
    for (int64_t r = 0; r < runs; ++r) s += part[r * C + c];
    out[c] = T::from_float(s);
}

template <class T>
hipError_t run_both(const Mx4PackArgs& a, unsigned grid, hipStream_t st)
{
    switch (a.act) {
        case kActNone: k_mx4_both<T, kActNone><<<grid, 256, 0, st>>>(a); break;
        case kActRelu: k_mx4_both<T, kActRelu><<<grid, 256, 0, st>>>(a); break;
        case kActGelu: k_mx4_both<T, kActGelu><<<grid, 256, 0, st>>>(a); break;
        default: k_mx4_both<T, kActSilu><<<grid, 256, 0, st>>>(a); break;
    }
    return hipGetLastError();
}

}  // namespace

// Tiles below each other of a block that forms the sums of its columns: few enough partial sums (4 bytes for every 256 or more of the values)
// while the blocks fill the chip.
int64_t mx4_sum_tiles(int64_t R, int64_t C)
{
    const int64_t tiles = (R + 127) / 128 * ((C + 127) / 128), per = tiles / 2048;
    return per < 1 ? 1 : per > 8 ? 8 : per;
}
int64_t mx4_sum_runs(int64_t R, int64_t C) { return ((R + 127) / 128 + mx4_sum_tiles(R, C) - 1) / mx4_sum_tiles(R, C); }

hipError_t launch_mx4_pack(Mx4PackArgs a, hipStream_t st)
{
    const Mx4Shape s(a.R, a.C);
    if (!a.out_t && !a.part && a.act == kActNone) {
        const int64_t n = s.rg * s.kb;
        if (n > 0x7fffffff) return hipErrorInvalidValue;
        if (a.type == 2)
            k_mx4_rows<F32><<<(unsigned)n, 256, 0, st>>>(a);
        else if (a.type == 1)
            k_mx4_rows<F16><<<(unsigned)n, 256, 0, st>>>(a);
        else
            k_mx4_rows<BF16><<<(unsigned)n, 256, 0, st>>>(a);
        return hipGetLastError();
    }
    a.per = a.part ? mx4_sum_tiles(a.R, a.C) : 1;
    const int64_t n = s.kb * (((a.R + 127) / 128 + a.per - 1) / a.per);
    if (n > 0x7fffffff) return hipErrorInvalidValue;
    if (a.type == 2) {
        k_mx4_both<F32, kActNone><<<(unsigned)n, 256, 0, st>>>(a);
        return hipGetLastError();
    }
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
    const unsigned grid = (unsigned)((C + 255) / 256);
    if (f16)
        k_mx4_sums<F16><<<grid, 256, 0, st>>>(part, mx4_sum_runs(R, C), C, (unsigned short*)out);
    else
        k_mx4_sums<BF16><<<grid, 256, 0, st>>>(part, mx4_sum_runs(R, C), C, (unsigned short*)out);
    return hipGetLastError();
}

}  // namespace rtn
