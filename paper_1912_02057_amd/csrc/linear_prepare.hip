// Ternary codes -> the two-bit operand order of the linear layer's products (WeightShape), for the forward product
// (rows n, columns k) and the backward one (rows k, columns n), in one pass over the codes.
#include "../../include/rtn.h"
#include "linear_math.h"
#include "rtn_kernels.h"

namespace rtn {

namespace {

constexpr int kPitch = 68;  // bytes of a row of the LDS tile

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

// One 64 x 64 tile of codes per block, through LDS; waves 0 and 1 write the forward order, 2 and 3 the transposed one.
template <int FMT>
__global__ __launch_bounds__(256) void k_linear_prepare(LinearPrepArgs a)
{
    __shared__ uint8_t tile[64 * kPitch];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t kt = (a.K + 63) / 64;
    const int64_t nb = blockIdx.x / kt, kb = blockIdx.x - nb * kt;
    const int64_t n0 = nb * 64, k0 = kb * 64;
    {
        const int row = tid >> 2, c0 = (tid & 3) * 16;
        const int64_t n = n0 + row;
        if (FMT == RTN_CODE_I8 && n < a.N && k0 + 64 <= a.Kpad) {  // rows are whole 64-byte steps, the padding codes are 0
            const uint4 v = *(const uint4*)((const int8_t*)a.codes + n * a.Kpad + k0 + c0);
            unsigned* t = (unsigned*)(tile + row * kPitch + c0);
            const bool whole = k0 + c0 + 16 <= a.K;
            const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                unsigned u = w[i] & 0x03030303u;
                const int64_t left = a.K - (k0 + c0 + 4 * i);  // codes of this row from here on
                if (!whole && left < 4) u = left <= 0 ? 0u : u & (0xffffffffu >> (32 - 8 * (int)left));
                t[i] = u;
            }
        } else {
            for (int i = 0; i < 16; ++i) {
                const int64_t k = k0 + c0 + i;
                tile[row * kPitch + c0 + i] = n < a.N && k < a.K ? (uint8_t)code_bits<FMT>(a, n, k) : (uint8_t)0;
            }
        }
    }
    __syncthreads();
    const bool trans = wave >= 2;
    uint2* out = (uint2*)(trans ? a.out_t : a.out);
    if (!out) return;
    const int rsub = (wave & 1) * 32 + (lane & 31), h = lane >> 5;
    const int64_t rows = trans ? a.K : a.N, cols = trans ? a.N : a.K;
    const WeightShape ws(rows, cols);
    const int64_t rblk = (trans ? kb : nb) * 2 + (wave & 1), cblk = trans ? nb : kb;
    if (rblk >= ws.rb) return;
    unsigned word[2] = {0, 0};
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int r = 0; r < 8; ++r)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int c = (2 * s + (r >> 2)) * 16 + 8 * h + 2 * (r & 3) + half;
                const unsigned bits = trans ? tile[c * kPitch + rsub] : tile[rsub * kPitch + c];
                word[s] |= bits << (16 * half + 14 - 2 * r);
            }
    out[(rblk * ws.cb + cblk) * 64 + lane] = make_uint2(word[0], word[1]);
}

}  // namespace

hipError_t launch_linear_prepare(const LinearPrepArgs& a, int fmt, hipStream_t st)
{
    const int64_t tiles = ((a.N + 63) / 64) * ((a.K + 63) / 64);
    if (fmt == RTN_CODE_I8)
        k_linear_prepare<RTN_CODE_I8><<<(unsigned)tiles, 256, 0, st>>>(a);
    else if (fmt == RTN_CODE_FP4)
        k_linear_prepare<RTN_CODE_FP4><<<(unsigned)tiles, 256, 0, st>>>(a);
    else
        k_linear_prepare<RTN_CODE_BITPLANE><<<(unsigned)tiles, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace rtn
