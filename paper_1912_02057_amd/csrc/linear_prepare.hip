// Ternary codes -> the two-bit operand order of the linear layer's products (WeightShape), for the forward product
// (rows n, columns k) and the backward one (rows k, columns n), in one pass over the codes.
#include "../../include/rtn.h"
#include "linear_math.h"
#include "rtn_kernels.h"

namespace rtn {

namespace {

constexpr int kPitch = 72;  // bytes of a row of an LDS tile

// code of two bits: bit 0 non-zero, bit 1 sign; that is t & 3
template <int FMT>
__device__ __forceinline__ int code_bits(const LinearPrepArgs& a, int64_t n, int64_t k)
{
    if constexpr (FMT == RTN_CODE_I8) return ((const int8_t*)a.codes)[n * a.Kpad + k] & 3;
    if constexpr (FMT == RTN_CODE_FP4) {
        const int v = ((const uint8_t*)a.codes)[n * (a.Kpad >> 1) + (k >> 1)] >> (4 * (k & 1));
        return (v >> 1 & 1) | (v >> 2 & 2);
    }
    const uint64_t* mask = (const uint64_t*)a.codes;
    const int64_t words = a.Kpad >> 6, at = n * words + (k >> 6);
    const int m = (int)(mask[at] >> (k & 63) & 1), plus = (int)(mask[a.N * words + at] >> (k & 63) & 1);
    return m | (m & (plus ^ 1)) << 1;
}

// Four codes of a dword (c0 .. c3, two bits each) at register r, r + 1 of a word: c0 and c2 in the low half, c1 and c3 in the high.
__device__ __forceinline__ unsigned place(unsigned d, int r)
{
    const unsigned lo = __builtin_amdgcn_perm(0, d, 0x0c010c00u), hi = __builtin_amdgcn_perm(0, d, 0x0c030c02u);
    return lo << (14 - 2 * r) | hi << (12 - 2 * r);
}

// TILES 64 x 64 tiles of codes beside each other per block, through LDS as they are and transposed (4 x 4 bytes a thread); waves 0
// and 1 write the forward order, 2 and 3 the transposed one.  Bound by its bytes, 1 read and 1/2 written per weight.
constexpr int kTiles = 2;
template <int FMT>
__global__ __launch_bounds__(256) void k_linear_prepare(LinearPrepArgs a)
{
    __shared__ __attribute__((aligned(16))) uint8_t tiles[kTiles][2][64 * kPitch];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t kt = (a.K + 64 * kTiles - 1) / (64 * kTiles);
    const int64_t nb = blockIdx.x / kt, kb = (blockIdx.x - nb * kt) * kTiles;
    const int64_t n0 = nb * 64;
    {
        const int row = tid >> 2, c0 = (tid & 3) * 16;
        const int64_t n = n0 + row;
        unsigned w[kTiles][4];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int64_t k0 = (kb + t) * 64 + c0;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (FMT == RTN_CODE_I8 && n < a.N && k0 < a.Kpad) v = *(const uint4*)((const int8_t*)a.codes + n * a.Kpad + k0);
            w[t][0] = v.x, w[t][1] = v.y, w[t][2] = v.z, w[t][3] = v.w;
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int64_t k0 = (kb + t) * 64 + c0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                unsigned u = w[t][i] & 0x03030303u;
                if constexpr (FMT != RTN_CODE_I8) {
                    u = 0;
                    for (int j = 0; j < 4; ++j)
                        if (n < a.N && k0 + 4 * i + j < a.K) u |= (unsigned)code_bits<FMT>(a, n, k0 + 4 * i + j) << (8 * j);
                } else if (k0 + 4 * i + 4 > a.K) {  // whatever lies past the row's end
                    const int64_t left = a.K - (k0 + 4 * i);
                    u = left <= 0 ? 0u : u & (0xffffffffu >> (32 - 8 * (int)left));
                }
                *(unsigned*)(tiles[t][0] + row * kPitch + c0 + 4 * i) = u;
            }
        }
    }
    __syncthreads();
    if (a.out_t) {
        const int r4 = (tid >> 4) * 4, c4 = (tid & 15) * 4;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            unsigned d[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) d[i] = *(const unsigned*)(tiles[t][0] + (r4 + i) * kPitch + c4);
            const unsigned a0 = __builtin_amdgcn_perm(d[1], d[0], 0x05010400u), a1 = __builtin_amdgcn_perm(d[1], d[0], 0x07030602u);
            const unsigned b0 = __builtin_amdgcn_perm(d[3], d[2], 0x05010400u), b1 = __builtin_amdgcn_perm(d[3], d[2], 0x07030602u);
            uint8_t* o = tiles[t][1] + c4 * kPitch + r4;
            *(unsigned*)o = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
            *(unsigned*)(o + kPitch) = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
            *(unsigned*)(o + 2 * kPitch) = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
            *(unsigned*)(o + 3 * kPitch) = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
        }
        __syncthreads();
    }
    const bool trans = wave >= 2;
    uint2* out = (uint2*)(trans ? a.out_t : a.out);
    if (!out) return;
    const int rsub = (wave & 1) * 32 + (lane & 31), h = lane >> 5;
    const WeightShape ws(trans ? a.K : a.N, trans ? a.N : a.K);
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const int64_t rblk = (trans ? kb + t : nb) * 2 + (wave & 1), cblk = trans ? nb : kb + t;
        if (rblk >= ws.rb || cblk >= ws.cb) continue;
        const uint8_t* row = tiles[t][trans] + rsub * kPitch + 8 * h;
        unsigned word[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint2 p = *(const uint2*)(row + 32 * s), q = *(const uint2*)(row + 32 * s + 16);
            word[s] = place(p.x, 0) | place(p.y, 2) | place(q.x, 4) | place(q.y, 6);
        }
        out[(rblk * ws.cb + cblk) * 64 + lane] = make_uint2(word[0], word[1]);
    }
}

}  // namespace

hipError_t launch_linear_prepare(const LinearPrepArgs& a, int fmt, hipStream_t st)
{
    const int64_t tiles = ((a.N + 63) / 64) * ((a.K + 64 * kTiles - 1) / (64 * kTiles));
    if (fmt == RTN_CODE_I8)
        k_linear_prepare<RTN_CODE_I8><<<(unsigned)tiles, 256, 0, st>>>(a);
    else if (fmt == RTN_CODE_FP4)
        k_linear_prepare<RTN_CODE_FP4><<<(unsigned)tiles, 256, 0, st>>>(a);
    else
        k_linear_prepare<RTN_CODE_BITPLANE><<<(unsigned)tiles, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace rtn
