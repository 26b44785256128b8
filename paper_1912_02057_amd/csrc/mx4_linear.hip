// Products of packed 4-bit matrices on the scaled FP4 matrix instruction: y = act(a w^T + bias) + residual, and the gradients of a layer.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 32 values and their scale from each lane, which is how they are packed (Mx4Shape): a block of
// 16 rows x 128 columns is 1 KiB in a row, lane by lane.  Products of codes and scales are exact; sums are the instruction's
// fp32 accumulators.  The weights are its first operand, so that a lane has four consecutive outputs of one token.
#include "mx4_math.h"
#include "choice.h"
#include "lds_limit.h"
#include "tmm_kernel.h"

namespace rtn {

namespace {

struct Mx4Params {
    const int8_t *a, *w;  // packed tokens and weights
    int M, N;
    int nk, arb, wrb;     // blocks of 128 columns; blocks of 16 rows of a and w
    int64_t ldr, ldy, ldz;
    const unsigned short *bias, *res;
    void* y;
    unsigned short* z;
    int act, y_f32;
    int res_once;         // the residual is read with the non-temporal hint
    int tilesM, ntiles, band_tiles;
    FastDiv div_band, div_lastband;
};

template <class F>
__device__ __forceinline__ void with_act(int act, F&& f)
{
    if (act == kActNone)
        f(std::integral_constant<int, kActNone>{});
    else if (act == kActRelu)
        f(std::integral_constant<int, kActRelu>{});
    else if (act == kActGelu)
        f(std::integral_constant<int, kActGelu>{});
    else
        f(std::integral_constant<int, kActSilu>{});
}

// Operand bytes of SEL in the lanes' scale registers
template <int SA, int SB>
__device__ __forceinline__ f32x4 mx4_mfma(u32x4 a, unsigned sa, u32x4 b, unsigned sb, f32x4 c)
{
    const v8i va = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, vb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, c, 4, 4, SA, (int)sa, SB, (int)sb);
}

// 32 x 32 x 64 with the sums held in place: as a function of 16 or more of them the compiler would rather write each product's result elsewhere
// and copy it back.  What reads `c` otherwise has to come behind mx4_settle().
template <int SA, int SB>
__device__ __forceinline__ void mx4_mfma_inplace(u32x4 a, unsigned sa, u32x4 b, unsigned sb, f32x16& c)
{
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0] cbsz:4 blgp:4"
                 : "+a"(c)
                 : "v"(a), "v"(b), "v"(sa), "v"(sb), "n"(SA & 1), "n"(SB & 1), "n"(SA >> 1), "n"(SB >> 1));
#endif
}
// The wait states between a matrix instruction and a vector instruction that reads its result (at most 20), which the compiler does not count for
// statements like the above; what reads the sums comes behind them, since they pass through the statement.
template <int TN, int TM>
__device__ __forceinline__ void mx4_settle(f32x16 (&c)[TN][TM])
{
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) asm volatile("" : "+a"(c[i][j]));
#endif
}

// What four outputs need beside their sums, fetched before the products: conditional loads behind them would each be waited for.
struct Extra {
    uint2 bias, res;
    static __device__ __forceinline__ uint2 four(const unsigned short* q, int left)
    {
        uint2 v = make_uint2(0, 0);
        if (left >= 4)
            __builtin_memcpy(&v, q, 8);
        else
            for (int i = 0; i < left; ++i) (i & 2 ? v.y : v.x) |= (unsigned)q[i] << (16 * (i & 1));
        return v;
    }
    __device__ __forceinline__ void fetch(const Mx4Params& p, int m, int n)
    {
        bias = res = make_uint2(0, 0);
        if (m >= p.M || n >= p.N) return;
        if (p.bias) bias = four(p.bias + n, p.N - n);
        if (p.res) res = four(p.res + m * p.ldr + n, p.N - n);
    }
};
// Outputs n .. n + 3 of token m from their sums
template <class T>
__device__ __forceinline__ void finish4(const Mx4Params& p, int m, int n, float4 sum, const Extra& x)
{
    if (m >= p.M || n >= p.N) return;
    const int left = p.N - n;
    float z[4] = {sum.x, sum.y, sum.z, sum.w};
    auto pick = [](const uint2& v, int i) { return half_of<T>(i & 2 ? v.y : v.x, i & 1); };
    if (p.bias) {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] += pick(x.bias, i);
    }
    auto put = [&](unsigned short* o) {
        const uint2 q = make_uint2(pack2<T>(z[0], z[1]), pack2<T>(z[2], z[3]));
        if (left >= 4)
            __builtin_memcpy(o, &q, 8);
        else
            for (int i = 0; i < left; ++i) o[i] = (unsigned short)((i & 2 ? q.y : q.x) >> (16 * (i & 1)));
    };
    if (p.z) put(p.z + m * p.ldz + n);
    with_act(p.act, [&](auto which) {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = act_value<decltype(which)::value>(z[i]);
    });
    if (p.res) {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] += pick(x.res, i);
    }
    if (p.y_f32) {
        float* y = (float*)p.y + m * p.ldy + n;
        if (left >= 4) {
            __builtin_memcpy(y, z, 16);
        } else {
            if (left > 0) y[0] = z[0];
            if (left > 1) y[1] = z[1];
            if (left > 2) y[2] = z[2];
        }
    } else {
        put((unsigned short*)p.y + m * p.ldy + n);
    }
}
// Item i of a block's outputs, four each, RB * 4 items a token, summed over the waves' parts in LDS
template <class T, int RB, int WAVES, int TOKENS, int PITCH>
struct Items {
    static constexpr int COUNT = TOKENS * RB * 4, PER = (COUNT + WAVES * 64 - 1) / (WAVES * 64);
    Extra x[PER];
    __device__ __forceinline__ void fetch(const Mx4Params& p, int m0, int n0)
    {
#pragma unroll
        for (int o = 0; o < PER; ++o) {
            const int i = threadIdx.x + o * WAVES * 64;
            x[o].fetch(p, i < COUNT ? m0 + i / (RB * 4) : p.M, n0 + i % (RB * 4) * 4);
        }
    }
    __device__ __forceinline__ void finish(const Mx4Params& p, int m0, int n0, const float* part)
    {
#pragma unroll
        for (int o = 0; o < PER; ++o) {
            const int i = threadIdx.x + o * WAVES * 64, t = i / (RB * 4), n = i % (RB * 4) * 4;
            if (i >= COUNT) break;
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int v = 0; v < WAVES; ++v) {
                const float4 q = *(const float4*)(part + (v * TOKENS + t) * PITCH + n);
                s.x += q.x, s.y += q.y, s.z += q.z, s.w += q.w;
            }
            finish4<T>(p, m0 + t, n0 + n, s, x[o]);
        }
    }
};

// The same of eight outputs whose bias is added and whose residual is there
template <class T>
__device__ __forceinline__ void finish_row(const Mx4Params& p, int m, int n, float (&z)[8], const u32x4& res)
{
    if (m >= p.M || n >= p.N) return;
    const int left = p.N - n;
    auto put = [&](unsigned short* o) {
        if (left >= 8) {
            store16(o, u32x4{pack2<T>(z[0], z[1]), pack2<T>(z[2], z[3]), pack2<T>(z[4], z[5]), pack2<T>(z[6], z[7])});
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) o[i] = T::from_float(z[i]);
        }
    };
    if (p.z) put(p.z + m * p.ldz + n);
    with_act(p.act, [&](auto which) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = act_value<decltype(which)::value>(z[i]);
    });
    if (p.res) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] += half_of<T>(res[i >> 1], i & 1);
    }
    if (p.y_f32) {
        float* y = (float*)p.y + m * p.ldy + n;
        if (left >= 8) {
            __builtin_memcpy(y, z, 32);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) y[i] = z[i];
        }
    } else {
        put((unsigned short*)p.y + m * p.ldy + n);
    }
}

template <int TB, int RB, int WAVES>
struct SplitMx4 {
    static constexpr int PITCH = RB * 16 + 4, LDS = WAVES * TB * 16 * PITCH * 4;
};

// Small grids: a block has 16 TB tokens x 16 RB outputs, its waves share the columns, every WAVES-th block of 128 each, and the operands go
// straight into registers, two blocks in flight.  The waves' sums are added up in LDS, in their order.  Bound by the latency of its loads:
// 24 tokens of 8192 x 8192 in 7.0 to 8.0 us, 4.5 to 5.1 TB/s of weights; 1000 x 1003 x 2187 8.5 us.
template <class T, int TB, int RB, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_mx4_split(Mx4Params p)
{
    using L = SplitMx4<TB, RB, WAVES>;
    static_assert(TB <= 4 && RB <= 4 && (TB & (TB - 1)) == 0 && (RB & (RB - 1)) == 0, "a block's scales are in one register");
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tn = (int)blockIdx.x / p.tilesM, tm = (int)blockIdx.x - tn * p.tilesM;
    const int rb0 = tn * RB, tb0 = tm * TB, nk = p.nk;
    const int64_t a_scales = (int64_t)p.arb * nk * 1024, w_scales = (int64_t)p.wrb * nk * 1024;
    const int8_t *ac[TB], *wc[RB];
#pragma unroll
    for (int t = 0; t < TB; ++t) ac[t] = p.a + (int64_t)(tb0 + t < p.arb ? tb0 + t : p.arb - 1) * nk * 1024 + lane * 16;
#pragma unroll
    for (int r = 0; r < RB; ++r) wc[r] = p.w + (int64_t)(rb0 + r < p.wrb ? rb0 + r : p.wrb - 1) * nk * 1024 + lane * 16;
    const int8_t *as = p.a + a_scales + (int64_t)(tb0 >> 2) * nk * 256 + lane * 4, *ws = p.w + w_scales + (int64_t)(rb0 >> 2) * nk * 256 + lane * 4;
    const int ash = 8 * (tb0 & 3), wsh = 8 * (rb0 & 3);
    Items<T, RB, WAVES, TB * 16, L::PITCH> items;
    items.fetch(p, tb0 * 16, rb0 * 16);

    f32x4 acc[RB][TB];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int t = 0; t < TB; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    struct Step {
        u32x4 a[TB], w[RB];
        unsigned sa, sw;
    };
    auto load = [&](Step& s, int kb) {
#pragma unroll
        for (int r = 0; r < RB; ++r) s.w[r] = load16(wc[r] + (int64_t)kb * 1024);
#pragma unroll
        for (int t = 0; t < TB; ++t) s.a[t] = load16(ac[t] + (int64_t)kb * 1024);
        s.sw = *(const unsigned*)(ws + (int64_t)kb * 256);
        s.sa = *(const unsigned*)(as + (int64_t)kb * 256);
    };
    auto products = [&](const Step& s) {
        const unsigned sw = s.sw >> wsh, sa = s.sa >> ash;
        for_each_index(
            [&](auto ri) {
                for_each_index(
                    [&](auto ti) {
                        constexpr int r = decltype(ri)::value, t = decltype(ti)::value;
                        acc[r][t] = mx4_mfma<r, t>(s.w[r], sw, s.a[t], sa, acc[r][t]);
                    },
                    std::make_integer_sequence<int, TB>{});
            },
            std::make_integer_sequence<int, RB>{});
    };
    if (wave < nk) {
        Step s[2];
        load(s[0], wave);
        int kb = wave;
        for (; kb + WAVES < nk; kb += 2 * WAVES) {
            load(s[1], kb + WAVES);
            products(s[0]);
            if (kb + 2 * WAVES < nk) load(s[0], kb + 2 * WAVES);
            products(s[1]);
        }
        if (kb < nk) products(s[0]);
    }
    float* part = (float*)smem + wave * TB * 16 * L::PITCH;
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int r = 0; r < RB; ++r)
            *(float4*)(part + (t * 16 + (lane & 15)) * L::PITCH + r * 16 + 4 * (lane >> 4)) = make_float4(acc[r][t][0], acc[r][t][1], acc[r][t][2], acc[r][t][3]);
    __syncthreads();
    items.finish(p, tb0 * 16, rb0 * 16, (const float*)smem);
}

template <class T, int TB, int RB, int WAVES>
hipError_t run_split(Mx4Params& p, hipStream_t st)
{
    using L = SplitMx4<TB, RB, WAVES>;
    static_assert(L::LDS <= 160 * 1024, "");
    p.tilesM = (p.M + 16 * TB - 1) / (16 * TB);
    const int64_t nt = (int64_t)p.tilesM * ((p.N + 16 * RB - 1) / (16 * RB));
    if (nt > 0x7fffff00) return hipErrorInvalidValue;
    static LdsLimit limit;
    const hipError_t e = limit.raise((const void*)&k_mx4_split<T, TB, RB, WAVES>, L::LDS);
    if (e != hipSuccess) return e;
    k_mx4_split<T, TB, RB, WAVES><<<(unsigned)nt, WAVES * 64, L::LDS, st>>>(p);
    return hipGetLastError();
}

// The packing of a lane's group of 32 16-bit values, as mx4_scale and mx4_nearest do it: its codes and its scale byte.  The conversion from
// 16 bits takes two values an instruction.
template <class T>
__device__ __forceinline__ u32x4 pack_group(const u32x4 (&v)[4], unsigned& scale)
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i >> 2][i & 3] & 0x7fff7fffu));
    const int s = mx4_scale(__float_as_uint(T::to_float(m[0] > m[1] ? m[0] : m[1])), false);
    const float f = mx4_factor(s);
    u32x4 q = {0, 0, 0, 0};
    scale = (unsigned)s;
    if (s == 255) return q;
    auto pair = [&](unsigned old, unsigned w, auto sel) {
        if constexpr (std::is_same_v<T, BF16>)
            return (unsigned)__builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2, w), f, decltype(sel)::value);
        else
            return (unsigned)__builtin_amdgcn_cvt_scalef32_pk_fp4_f16(old, __builtin_bit_cast(f16x2, w), f, decltype(sel)::value);
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned c = pair(0, v[i][0], std::integral_constant<int, 0>{});
        c = pair(c, v[i][1], std::integral_constant<int, 1>{});
        c = pair(c, v[i][2], std::integral_constant<int, 2>{});
        q[i] = pair(c, v[i][3], std::integral_constant<int, 3>{});
    }
    return q;
}

// A few tokens (at most 16) in 16 bits: a block has 16 RB outputs, its waves share the columns, every WAVES-th block of 128 each.  A lane's part of
// the token operand is one group of 32 values, so it packs them itself on the way into the instruction.
// Bound by latencies: launch, a round of loads per two blocks of a wave, the sum over the waves (4096 x 4096, one token: 4.7 us, 8192 x 8192 7.6
// from packed tokens: 5.0 TB/s of weights).  What an output needs beside its sum is fetched first: loaded behind the products, where a
// condition stands before each, it took 18.9 us.  ROW16: rows of whole 16-byte units, loaded without a branch.
template <class T, int RB, int WAVES, bool ROW16>
__global__ __launch_bounds__(WAVES * 64) void k_mx4_few(Mx4Params p, const unsigned short* x, int64_t ldx, int K)
{
    constexpr int PITCH = RB * 16 + 4;
    __shared__ __attribute__((aligned(16))) float part[WAVES][16][PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, c = lane >> 4;
    // blocks that share a piece of scales (four blocks of rows) on one XCD, whose L2 then fetches it once
    const int chunk = (int)(gridDim.x >> 3), rb0 = ((int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3)) * RB, nk = p.nk;
    if (rb0 >= p.wrb) return;
    Items<T, RB, WAVES, 16, PITCH> items;
    items.fetch(p, 0, rb0 * 16);
    const int8_t* wc[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) wc[r] = p.w + (int64_t)(rb0 + r < p.wrb ? rb0 + r : p.wrb - 1) * nk * 1024 + lane * 16;
    const int8_t* ws = p.w + ((int64_t)p.wrb * 4 + (rb0 >> 2)) * nk * 256 + lane * 4;
    const int wsh = 8 * (rb0 & 3);
    const unsigned short* row = x + (l16 < p.M ? l16 : 0) * ldx;
    const auto xr = __builtin_amdgcn_make_buffer_rsrc((void*)x, 0, ROW16 ? (int)(((p.M - 1) * ldx + K) * 2) : 0, 0x00020000);
    const int xoff = l16 < p.M ? (int)(l16 * ldx * 2) + c * 64 : (int)kOutside;  // (past the rows: zeros)
    f32x4 acc[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
    struct Step {
        u32x4 w[RB], x[4];
        unsigned sw;
    };
    auto load = [&](Step& s, int kb) {
#pragma unroll
        for (int r = 0; r < RB; ++r) s.w[r] = load16(wc[r] + (int64_t)kb * 1024);
        s.sw = *(const unsigned*)(ws + (int64_t)kb * 256);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (ROW16)
                s.x[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xr, (int)((unsigned)xoff + (unsigned)(kb * 256 + 16 * i)), 0, 0));
            else
                s.x[i] = l16 < p.M ? load_row8(row, kb * 128 + 32 * c + 8 * i, K) : u32x4{0, 0, 0, 0};
        }
    };
    auto products = [&](Step& s, int kb) {
        if (ROW16 && kb == nk - 1) {  // what follows the row's end is another row's
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (kb * 128 + 32 * c + 8 * i >= K) s.x[i] = u32x4{0, 0, 0, 0};
        }
        const unsigned sw = s.sw >> wsh;
        unsigned sx;
        const u32x4 q = pack_group<T>(s.x, sx);
        for_each_index(
            [&](auto ri) {
                constexpr int r = decltype(ri)::value;
                acc[r] = mx4_mfma<r, 0>(s.w[r], sw, q, sx, acc[r]);
            },
            std::make_integer_sequence<int, RB>{});
    };
    if (wave < nk) {
        Step s[2];
        load(s[0], wave);
        int kb = wave;
        for (; kb + WAVES < nk; kb += 2 * WAVES) {
            load(s[1], kb + WAVES);
            products(s[0], kb);
            if (kb + 2 * WAVES < nk) load(s[0], kb + 2 * WAVES);
            products(s[1], kb + WAVES);
        }
        if (kb < nk) products(s[0], kb);
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) *(float4*)&part[wave][l16][r * 16 + 4 * c] = make_float4(acc[r][0], acc[r][1], acc[r][2], acc[r][3]);
    __syncthreads();
    items.finish(p, 0, rb0 * 16, &part[0][0][0]);
}

template <class T, int RB, int WAVES>
hipError_t run_few(const Mx4Params& p, const Mx4LinArgs& a, hipStream_t st)
{
    const int blocks = (p.wrb + RB - 1) / RB;
    const unsigned grid = (unsigned)((blocks + 7) / 8 * 8);
    if (a.K % 8 == 0 && a.ldx % 8 == 0 && ((uintptr_t)a.x & 15) == 0 && (a.M * a.ldx + a.K) * 2 < (int64_t)kOutside)
        k_mx4_few<T, RB, WAVES, true><<<grid, WAVES * 64, 0, st>>>(p, (const unsigned short*)a.x, a.ldx, (int)a.K);
    else
        k_mx4_few<T, RB, WAVES, false><<<grid, WAVES * 64, 0, st>>>(p, (const unsigned short*)a.x, a.ldx, (int)a.K);
    return hipGetLastError();
}

// ---- tiles of a full grid
typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2)));  // wherever it starts
template <int BM, int BN, int NS_, int WM>
struct TileMx4 {
    static constexpr int NS = NS_;                                 // stages of 128 columns
    static constexpr int WAVES = 2 * WM, WN = BN / 2, TM = BM / 32 / WM, TN = BN / 64;  // a wave's outputs; its blocks of 32 tokens, of 32 outputs
    // codes of the weights and the tokens, then their scales, 1 KiB each
    static constexpr int CODES = (BM + BN) * 64, STAGE = CODES + 2 * 1024, PER = (BM + BN) / 16 / WAVES, DPS = PER + 1;
    static constexpr int OTHER = BN / 16 % PER;                    // from this one on, a wave's loads may be of the tokens
    static constexpr int PITCH = WN * 4 + 16, WAVE = 32 * PITCH;   // 32 tokens of a wave in the epilogue
    static constexpr int LDS = NS * STAGE > WAVES * WAVE ? NS * STAGE : WAVES * WAVE, BLOCKS = LDS <= 80 * 1024 ? 2 : 1;
};

// A block of 2 WM waves owns BM tokens x BN outputs, a wave half of the outputs of a WM-th of the tokens.  Ring of NS stages of 128 columns, as packed
// (1 KiB a block of 16 rows, so loads and reads of it are in a row), and their scales.  One barrier a step, before the second of its two
// 64-column slices; fragments are read one slice ahead, and the loads of the stage that the barrier frees are spread over the second.  The
// instruction is 32 x 32 x 64: one wave a SIMD issues 16 x 16 x 128 at two thirds of its rate (registers only, random codes: 5.3
// PFLOP/s against 6.5, which is what the power limit leaves).  Lane l has row l & 31 of 32, so 16 lanes have one block of rows and 16 the
// next: a lane's scales are shifted so that both stand in the byte the instruction picks.
// Over several rounds two blocks of 128 x 256 share a CU, so that one's epilogue passes beside the other's products: 16384 x 8192 x 8192 492 us,
// with a residual 513 to 537 (4.1 to 4.3 PFLOP/s).  Bound by the power limit and by waits: the clock falls to 1.4 to 1.6 GHz, and of its cycles the
// matrix cores are busy 59 to 64 %, where a loop of products alone has none idle at 1.56 GHz.  Of 822 thousand cycles 132 are outside the loop (what
// is left at no columns, from 8192 and 16384 of them) and 166 are in it, waiting at its counters, barriers and LDS reads.  In a
// single round there is nothing to pass beside, and a block of 256 x 256 with eight waves loads a third less: 4096 x 4096 x 4096 36 to 38 us (38
// to 40), 2048 x 8192 x 8192 63 (68); over several, with a residual, 553 (528) at 16384 x 8192 x 8192.
template <class T, int BM, int BN, int NS, int WM>
__global__ __launch_bounds__(128 * WM, (TileMx4<BM, BN, NS, WM>::BLOCKS * WM / 2)) void k_mx4_tile(Mx4Params p)
{
    using L = TileMx4<BM, BN, NS, WM>;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, h = lane >> 5, wn = wave / WM, wm = wave % WM, nk = p.nk;
    int tm, tn;
    {
        const int chunk = (int)(gridDim.x >> 3), bid = (int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3);
        if (bid >= p.ntiles) return;
        band_tile(bid, p.tilesM, p.band_tiles, [&](int n) { return (int)fastdiv((uint32_t)n, p.div_band); },
                  [&](int n) { return (int)fastdiv((uint32_t)n, p.div_lastband); }, tm, tn);
    }
    tm = __builtin_amdgcn_readfirstlane(tm), tn = __builtin_amdgcn_readfirstlane(tn);  // (scalars, also where band_tile is a call)
    const int m0 = tm * BM, n0 = tn * BN;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;

    // ---- direct loads of a stage: a wave has its share of the blocks of 16 rows, the weights' before the tokens', and the scales of either
    // (all even waves write the same, and all odd ones, so that all count alike)
    const int wb0 = n0 / 16, ab0 = m0 / 16;
    auto code_base = [&](bool of_w) { return buffer_base(of_w ? p.w + (int64_t)wb0 * nk * 1024 : p.a + (int64_t)ab0 * nk * 1024); };
    const v4i codes[2] = {code_base(wave * L::PER < BN / 16), code_base(wave * L::PER + L::OTHER < BN / 16)};
    const v4i scales = wave & 1 ? buffer_base(p.a + ((int64_t)p.arb * 4 + (ab0 >> 2)) * nk * 256) : buffer_base(p.w + ((int64_t)p.wrb * 4 + (wb0 >> 2)) * nk * 256);
    unsigned off[L::PER], soff;
#pragma unroll
    for (int i = 0; i < L::PER; ++i) {
        const int b = wave * L::PER + i, local = b < BN / 16 ? b : b - BN / 16, last = b < BN / 16 ? p.wrb - 1 - wb0 : p.arb - 1 - ab0;
        off[i] = (unsigned)(local < last ? local : last) * (unsigned)(nk * 1024) + (unsigned)(lane * 16);
    }
    {
        // (four pieces of 256 bytes; those beyond the tile or the matrix repeat the last one: a branch in the loop would cost more)
        const int last = (wave & 1 ? (p.arb - 1) / 4 - ab0 / 4 : (p.wrb - 1) / 4 - wb0 / 4), g = lane >> 4;
        soff = (unsigned)(g < last ? g : last) * (unsigned)(nk * 256) + (unsigned)((lane & 15) * 16);
    }
    auto load_one = [&](auto index, int step, unsigned stage) {
        constexpr int i = decltype(index)::value;
        if constexpr (i < L::PER)
            dma_buf<i * 1024>(codes[L::OTHER && i >= L::OTHER], off[i], (unsigned)step * 1024u, stage + (unsigned)(wave * L::PER * 1024));
        else
            dma_buf<L::CODES>(scales, soff, (unsigned)step * 256u, stage + (unsigned)((wave & 1) * 1024));
    };
    auto issue = [&](int step, int slot) {
        for_each_index([&](auto index) { load_one(index, step, lds0 + (unsigned)(slot * L::STAGE)); }, std::make_integer_sequence<int, L::DPS>{});
    };

    f32x16 acc[L::TN][L::TM];
#pragma unroll
    for (int i = 0; i < L::TN; ++i)
#pragma unroll
        for (int j = 0; j < L::TM; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    constexpr int ST = (L::TN + 1) / 2, SM = (L::TM + 1) / 2, READS = ST + SM + L::TN + L::TM, NM = L::TN * L::TM;
    struct Frags {
        u32x4 w[L::TN], a[L::TM];
        unsigned sw[ST], sa[SM];
    } f[2];
    const int flane = (l32 >> 4) * 1024 + h * 256 + (l32 & 15) * 16, slane = h * 64 + (l32 & 15) * 4, shift = 8 * (l32 >> 4);
    // read `index` of a slice's fragments
    auto read_one = [&](auto index, auto slice, Frags& q, const char* stage) {
        constexpr int i = decltype(index)::value, s = decltype(slice)::value;
        if constexpr (i < ST)
            q.sw[i] = *(const unsigned*)(stage + L::CODES + (wn * ST + i) * 256 + s * 128 + slane);
        else if constexpr (i < ST + SM)
            q.sa[i - ST] = *(const unsigned*)(stage + L::CODES + 1024 + (wm * SM + i - ST) * 256 + s * 128 + slane);
        else if constexpr (i < ST + SM + L::TN)
            q.w[i - ST - SM] = *(const u32x4*)(stage + (wn * L::TN + i - ST - SM) * 2048 + s * 512 + flane);
        else
            q.a[i - ST - SM - L::TN] = *(const u32x4*)(stage + (BN / 32 + wm * L::TM + i - ST - SM - L::TN) * 2048 + s * 512 + flane);
    };

    for (int s = 0; s < L::NS && s < nk; ++s) issue(s, s);
    wait_groups<L::DPS>((nk < L::NS ? nk : L::NS) - 1);
    block_barrier();
    const std::integral_constant<int, 0> zero{};
    const std::integral_constant<int, 1> one{};
    for_each_index([&](auto index) { read_one(index, zero, f[0], smem); }, std::make_integer_sequence<int, READS>{});

    int slot = 0;
    // STEADY: step + NS exists, so that it is loaded and no count depends on the step; behind the last of those nothing is left to load
    auto one_step = [&](auto steady, int step) {
        constexpr bool STEADY = decltype(steady)::value;
        const int next = slot + 1 == L::NS ? 0 : slot + 1;
        const unsigned fill = lds0 + (unsigned)(slot * L::STAGE);
        auto slice = [&](auto index) {
            constexpr int s = decltype(index)::value;
            Frags &cur = f[s], &nxt = f[s ^ 1];
            if constexpr (s == 1) {
                // all of this step's fragments are in registers, of all waves behind the barrier: its slot is free, and step + 1 has landed
                if constexpr (STEADY) {
                    wait_vm<(L::NS - 2) * L::DPS>();
                } else {
                    const int later = nk - 2 - step;
                    wait_groups<L::DPS>(later < L::NS - 2 ? later : L::NS - 2);
                }
                wait_lgkm0();
                block_barrier();
            } else {
                wait_lgkm0();
            }
#pragma unroll
            for (int i = 0; i < ST; ++i) cur.sw[i] >>= shift, pin(cur.sw[i]);
#pragma unroll
            for (int i = 0; i < SM; ++i) cur.sa[i] >>= shift, pin(cur.sa[i]);
            asm volatile("s_nop 1");  // between a vector instruction's write and a matrix instruction that reads it, which the compiler does not see
            __builtin_amdgcn_sched_barrier(0);
            const char* stage = smem + (s ? next : slot) * L::STAGE;  // (behind the last step: what the slot holds, which nothing takes)
            constexpr int OPS = READS + (s && STEADY ? L::DPS : 0), PER = (READS + L::DPS + NM - 1) / NM;
            for_each_index(
                [&](auto mi) {
                    constexpr int n = decltype(mi)::value, i = n / L::TM, j = i & 1 ? L::TM - 1 - n % L::TM : n % L::TM;
                    mx4_mfma_inplace<2 * (i & 1), 2 * (j & 1)>(cur.w[i], cur.sw[i / 2], cur.a[j], cur.sa[j / 2], acc[i][j]);
                    for_each_index(
                        [&](auto oi) {
                            constexpr int o = n * PER + decltype(oi)::value;
                            if constexpr (o < READS)
                                read_one(std::integral_constant<int, o>{}, std::integral_constant<int, s ^ 1>{}, nxt, stage);
                            else if constexpr (o < OPS)
                                load_one(std::integral_constant<int, o - READS>{}, step + L::NS, fill);
                        },
                        std::make_integer_sequence<int, PER>{});
                    __builtin_amdgcn_sched_barrier(0);
                },
                std::make_integer_sequence<int, NM>{});
        };
        slice(zero);
        slice(one);
        slot = next;
    };
    int step = 0;
    for (; step + L::NS < nk; ++step) one_step(std::true_type{}, step);
    for (; step < nk; ++step) one_step(std::false_type{}, step);

    mx4_settle(acc);
    // ---- epilogue: 32 tokens of the wave at a time through LDS, after which a lane has 8 outputs of a token, in TPL passes.  With one wave on a
    // SIMD its time is its instructions, each some five cycles: a tile that lies inside the matrix has no address or bound to compute per
    // row (scalar bases, one offset a lane), and the activation is picked once.
    __syncthreads();
    constexpr int CL = L::WN / 8, RPP = 64 / CL, TPL = 32 / RPP;
    char* zs = smem + wave * L::WAVE;
    const int nw = n0 + wn * L::WN, mw = m0 + wm * (BM / WM), n8 = nw + (lane % CL) * 8, t0 = lane / CL;
    if (nw >= p.N || mw >= p.M) return;
    float bi[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) bi[i] = p.bias && n8 + i < p.N ? T::to_float(p.bias[n8 + i]) : 0.f;
    auto put = [&](auto index) __attribute__((always_inline)) {
        constexpr int j = decltype(index)::value;
#pragma unroll
        for (int i = 0; i < L::TN; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)  // outputs 8 q + 4 h .. + 3 of token l32
                *(float4*)(zs + l32 * L::PITCH + (i * 32 + 8 * q + 4 * h) * 4) =
                    make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
        wait_lgkm0();
        // (the next round's writes to `zs` are this wave's own and come after its reads)
    };
    auto read_z = [&](int t, float(&z)[8]) __attribute__((always_inline)) {
        const float* q = (const float*)(zs + (t * RPP + t0) * L::PITCH + (lane % CL) * 32);
        const float4 a = *(const float4*)q, b = *(const float4*)(q + 4);
        z[0] = a.x + bi[0], z[1] = a.y + bi[1], z[2] = a.z + bi[2], z[3] = a.w + bi[3];
        z[4] = b.x + bi[4], z[5] = b.y + bi[5], z[6] = b.z + bi[6], z[7] = b.w + bi[7];
    };
    constexpr int64_t kFar = 1 << 26;  // a pitch up to which a lane's offset is 32 bits
    const bool whole = mw + BM / WM <= p.M && nw + L::WN <= p.N && p.ldy < kFar && p.ldr < kFar && p.ldz < kFar;
    const unsigned col = (unsigned)(lane % CL) * 8;
    const unsigned vy = ((unsigned)t0 * (unsigned)p.ldy + col) * (p.y_f32 ? 4u : 2u), vr = ((unsigned)t0 * (unsigned)p.ldr + col) * 2u,
                   vz = ((unsigned)t0 * (unsigned)p.ldz + col) * 2u;
    auto row = [](auto* base, int64_t ld, int m, int n, int bytes) { return (char*)base + ((int64_t)m * ld + n) * bytes; };
    // the residual of all rounds at once where a block is alone on its CU, so that one latency is exposed; else of a round
    constexpr int AHEAD = L::BLOCKS == 1 ? L::TM : 1;
    u32x4 res[AHEAD][TPL];
    auto fetch = [&](int k, u32x4(&r)[TPL]) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < TPL; ++t) {
            const u32x4_any* q = (const u32x4_any*)(row(p.res, p.ldr, mw + k * 32 + t * RPP, nw, 2) + vr);
            r[t] = p.res_once ? __builtin_nontemporal_load(q) : *q;
        }
    };
    if (AHEAD > 1 && p.res && whole)
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) fetch(k, res[k]);
    for_each_index(
        [&](auto index) __attribute__((always_inline)) {
            constexpr int k = decltype(index)::value, at = AHEAD > 1 ? k : 0;
            if (mw + k * 32 >= p.M) return;
            if (AHEAD == 1 && p.res && whole) fetch(k, res[0]);
            put(index);
            if (!whole) {
#pragma unroll 1
                for (int t = 0; t < TPL; ++t) {
                    const int m = mw + k * 32 + t * RPP + t0;
                    float z[8];
                    read_z(t, z);
                    finish_row<T>(p, m, n8, z, p.res && m < p.M ? load_row8(p.res + m * p.ldr, n8, p.N) : u32x4{0, 0, 0, 0});
                }
                return;
            }
            with_act(p.act, [&](auto which) __attribute__((always_inline)) {
#pragma unroll
                for (int t = 0; t < TPL; ++t) {
                    const int m = mw + k * 32 + t * RPP;
                    float z[8];
                    read_z(t, z);
                    auto packed = [&] { return u32x4{pack2<T>(z[0], z[1]), pack2<T>(z[2], z[3]), pack2<T>(z[4], z[5]), pack2<T>(z[6], z[7])}; };
                    if (p.z) store16(row(p.z, p.ldz, m, nw, 2) + vz, packed());
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[i] = act_value<decltype(which)::value>(z[i]);
                    if (p.res) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) z[i] += half_of<T>(res[at][t][i >> 1], i & 1);
                    }
                    if (p.y_f32) {
                        char* y = row(p.y, p.ldy, m, nw, 4) + vy;
                        const u32x4_any lo = {__float_as_uint(z[0]), __float_as_uint(z[1]), __float_as_uint(z[2]), __float_as_uint(z[3])},
                                        hi = {__float_as_uint(z[4]), __float_as_uint(z[5]), __float_as_uint(z[6]), __float_as_uint(z[7])};
                        *(u32x4_any*)y = lo, *(u32x4_any*)(y + 16) = hi;
                    } else {
                        store16(row(p.y, p.ldy, m, nw, 2) + vy, packed());
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            });
        },
        std::make_integer_sequence<int, L::TM>{});
}

template <class T, int BM, int BN, int NS, int WM>
hipError_t run_tile(Mx4Params& p, hipStream_t st)
{
    using L = TileMx4<BM, BN, NS, WM>;
    p.tilesM = (p.M + BM - 1) / BM;
    const int tilesN = (p.N + BN - 1) / BN;
    const int64_t nt = (int64_t)p.tilesM * tilesN;
    if (nt > 0x7fffff00) return hipErrorInvalidValue;
    p.ntiles = (int)nt;
    p.band_tiles = 8 * tilesN;
    p.div_band = make_fastdiv((uint32_t)p.band_tiles);
    p.div_lastband = make_fastdiv((uint32_t)(p.tilesM % 8 ? p.tilesM % 8 : 8));
    static LdsLimit limit;
    const hipError_t e = limit.raise((const void*)&k_mx4_tile<T, BM, BN, NS, WM>, L::LDS);
    if (e != hipSuccess) return e;
    k_mx4_tile<T, BM, BN, NS, WM><<<(unsigned)((nt + 7) / 8 * 8), 128 * WM, L::LDS, st>>>(p);
    return hipGetLastError();
}

template <class T>
hipError_t run(Mx4Params& p, const Mx4LinArgs& a, hipStream_t st)
{
    if (!p.a) return a.N <= 4096 ? run_few<T, 1, 8>(p, a, st) : run_few<T, 2, 8>(p, a, st);
    switch (mx4_form(a.M, a.N, a.K)) {
        case Mx4Form::kSplit16: return run_split<T, 1, 1, 8>(p, st);
        case Mx4Form::kSplit16x32: return run_split<T, 1, 2, 8>(p, st);
        case Mx4Form::kSplit32: return run_split<T, 2, 2, 8>(p, st);
        case Mx4Form::kSplit32x64: return run_split<T, 2, 4, 8>(p, st);
        case Mx4Form::kSplit64: return run_split<T, 4, 4, 8>(p, st);
        case Mx4Form::kSplit64x4: return run_split<T, 4, 4, 4>(p, st);
        case Mx4Form::kTile128: return run_tile<T, 128, 128, 4, 2>(p, st);
        case Mx4Form::kTile256: return run_tile<T, 256, 256, 4, 4>(p, st);
        default: return run_tile<T, 128, 256, 3, 2>(p, st);
    }
}

__global__ __launch_bounds__(256) void k_mx4_zero(unsigned short* out, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) out[i] = 0;
}
hipError_t zero(void* out, int64_t n, hipStream_t st)
{
    const int64_t blocks = (n + 255) / 256;
    k_mx4_zero<<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, st>>>((unsigned short*)out, n);
    return hipGetLastError();
}

int64_t up256(int64_t n) { return (n + 255) / 256 * 256; }

}  // namespace

bool mx4_packs_x(int64_t M, int64_t, int64_t) { return M > kMx4FewTokens; }

hipError_t launch_mx4_linear(const Mx4LinArgs& a, hipStream_t st)
{
    Mx4Params p = {};
    p.M = (int)a.M, p.N = (int)a.N;
    const Mx4Shape as(a.M, a.K), ws(a.N, a.K);
    p.nk = (int)ws.kb, p.arb = (int)as.rb, p.wrb = (int)ws.rb;
    p.w = (const int8_t*)a.w;
    p.a = (const int8_t*)a.a;
    p.ldr = a.ldr, p.ldy = a.ldy, p.ldz = a.ldz;
    p.bias = (const unsigned short*)a.bias, p.res = (const unsigned short*)a.res;
    p.y = a.y, p.z = (unsigned short*)a.z;
    p.act = a.act, p.y_f32 = a.y_f32;
    // A residual that the memory-side cache would not keep anyway leaves the operands there: 16384 x 8192 x 8192 531 -> 513 us, but
    // 4096 x 4096 x 4096 (32 MiB) 44 -> 47.  (The same hint on the stores changes nothing.)
    p.res_once = a.M * a.N >= (int64_t)1 << 25;
    if (!a.a && mx4_packs_x(a.M, a.N, a.K)) {
        Mx4PackArgs k = {};
        k.x = a.x, k.R = a.M, k.C = a.K, k.ldx = a.ldx, k.out = a.workspace, k.type = a.f16;
        const hipError_t e = launch_mx4_pack(k, st);
        if (e != hipSuccess) return e;
        p.a = (const int8_t*)a.workspace;
    }
    return a.f16 ? run<F16>(p, a, st) : run<BF16>(p, a, st);
}

// dz packed along its rows for dx, along its columns for dw, and the partial sums of dbias
size_t mx4_backward_workspace(int64_t M, int64_t N, int64_t)
{
    if (M == 0) return 0;
    return (size_t)(up256(Mx4Shape(M, N).bytes()) + up256(Mx4Shape(N, M).bytes()) + mx4_sum_runs(M) * N * 4);
}

hipError_t launch_mx4_backward(const Mx4BwdArgs& a, hipStream_t st)
{
    hipError_t e;
    if (a.M == 0) {
        if (a.dw && (e = zero(a.dw, a.N * a.K * (a.dw_f32 ? 2 : 1), st)) != hipSuccess) return e;
        return a.dbias ? zero(a.dbias, a.N, st) : hipSuccess;
    }
    char *dz = a.workspace, *dzt = dz + up256(Mx4Shape(a.M, a.N).bytes());
    float* part = (float*)(dzt + up256(Mx4Shape(a.N, a.M).bytes()));
    Mx4PackArgs k = {};
    k.x = a.dy, k.R = a.M, k.C = a.N, k.ldx = a.lddy, k.z = a.z, k.ldz = a.ldz, k.act = a.act, k.type = a.f16, k.seed = a.seed;
    k.out = a.dx ? dz : nullptr, k.out_t = a.dw ? dzt : nullptr, k.part = a.dbias ? part : nullptr;
    if ((e = launch_mx4_pack(k, st)) != hipSuccess) return e;
    if (a.dbias && (e = launch_mx4_sums(part, a.M, a.N, a.dbias, a.f16, st)) != hipSuccess) return e;
    Mx4LinArgs l = {};
    l.f16 = a.f16;
    if (a.dx) {
        l.a = dz, l.w = a.wt, l.M = a.M, l.N = a.K, l.K = a.N, l.y = a.dx, l.ldy = a.lddx;
        if ((e = launch_mx4_linear(l, st)) != hipSuccess) return e;
    }
    if (a.dw) {
        l.a = dzt, l.w = a.xt, l.M = a.N, l.N = a.K, l.K = a.M, l.y = a.dw, l.ldy = a.K, l.y_f32 = a.dw_f32;
        if ((e = launch_mx4_linear(l, st)) != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace rtn
