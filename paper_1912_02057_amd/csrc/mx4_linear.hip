// Products of packed 4-bit matrices on the scaled FP4 matrix instruction: y = act(a w^T + bias) + residual, and the gradients of a layer.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 32 values and their scale from each lane, which is how they are packed (Mx4Shape): a block of
// 16 rows x 128 columns is 1 KiB in a row, lane by lane.  Products of codes and scales are exact; sums are the instruction's
// fp32 accumulators.  The weights are its first operand, so that a lane has four consecutive outputs of one token.
#include "mx4_math.h"
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

// Outputs n .. n + V - 1 of token m from their sums
template <class T, int V>
__device__ __forceinline__ void finish(const Mx4Params& p, int m, int n, float (&z)[V])
{
    if (m >= p.M || n >= p.N) return;
    const int left = p.N - n;
    if (p.bias) {
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] += i < left ? T::to_float(p.bias[n + i]) : 0.f;
    }
    auto put = [&](unsigned short* o) {
        if (left >= V) {
            unsigned q[V / 2];
#pragma unroll
            for (int i = 0; i < V; i += 2) q[i / 2] = pack2<T>(z[i], z[i + 1]);
            __builtin_memcpy(o, q, V * 2);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < left) o[i] = T::from_float(z[i]);
        }
    };
    if (p.z) put(p.z + m * p.ldz + n);
    with_act(p.act, [&](auto which) {
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = act_value<decltype(which)::value>(z[i]);
    });
    if (p.res) {
        const unsigned short* r = p.res + m * p.ldr + n;
        if (left >= V) {
            unsigned short q[V];
            __builtin_memcpy(q, r, V * 2);
#pragma unroll
            for (int i = 0; i < V; ++i) z[i] += T::to_float(q[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < left) z[i] += T::to_float(r[i]);
        }
    }
    if (p.y_f32) {
        float* y = (float*)p.y + m * p.ldy + n;
        if (left >= V) {
            __builtin_memcpy(y, z, V * 4);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
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
// straight into registers.  The waves' sums are added up in LDS, in their order.
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
        s.sw = *(const unsigned*)(ws + (int64_t)kb * 256) >> wsh;
        s.sa = *(const unsigned*)(as + (int64_t)kb * 256) >> ash;
    };
    auto products = [&](const Step& s) {
        for_each_index(
            [&](auto ri) {
                for_each_index(
                    [&](auto ti) {
                        constexpr int r = decltype(ri)::value, t = decltype(ti)::value;
                        acc[r][t] = mx4_mfma<r, t>(s.w[r], s.sw, s.a[t], s.sa, acc[r][t]);
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
    for (int item = tid; item < TB * 16 * RB * 4; item += WAVES * 64) {
        const int t = item / (RB * 4), n = item % (RB * 4) * 4;
        float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < WAVES; ++v) {
            const float4 q = *(const float4*)((const float*)smem + (v * TB * 16 + t) * L::PITCH + n);
            z[0] += q.x, z[1] += q.y, z[2] += q.z, z[3] += q.w;
        }
        finish<T, 4>(p, tb0 * 16 + t, rb0 * 16 + n, z);
    }
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

template <class T>
hipError_t run(Mx4Params& p, hipStream_t st)
{
    return run_split<T, 2, 2, 8>(p, st);
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

bool mx4_packs_x(int64_t, int64_t, int64_t) { return true; }

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
    if (!a.a) {
        Mx4PackArgs k = {};
        k.x = a.x, k.R = a.M, k.C = a.K, k.ldx = a.ldx, k.out = a.workspace, k.type = a.f16;
        const hipError_t e = launch_mx4_pack(k, st);
        if (e != hipSuccess) return e;
        p.a = (const int8_t*)a.workspace;
    }
    return a.f16 ? run<F16>(p, st) : run<BF16>(p, st);
}

// dz packed along its rows for dx, along its columns for dw, and the partial sums of dbias
size_t mx4_backward_workspace(int64_t M, int64_t N, int64_t)
{
    if (M == 0) return 0;
    return (size_t)(up256(Mx4Shape(M, N).bytes()) + up256(Mx4Shape(N, M).bytes()) + mx4_sum_runs(M, N) * N * 4);
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
