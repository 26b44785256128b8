// Gradients of the ternary linear layer from 8-bit checkpoints of its input and of the value before its activation.
//
//   dz = dy act'(z^)     dbias = sum_m dz     dx = (dz alpha) t     dw = dz^T x^
//
// One pass (k_linear_grad) writes dz as each product takes it; dx is the forward product on the transposed prepared weights;
// dw, which contracts over tokens, has a kernel of its own here: both operands lie in the order the matrix instruction takes
// them, so its loads and fragment reads are consecutive.
#include "linear_math.h"
#include "tmm_kernel.h"

namespace rtn {

namespace {

// dbias[n] = sum of the runs' partial sums: four strands of every fourth run, each in order, then the strands in order.  A block of
// 256 threads has 64 outputs; `sums` 256 floats of LDS.
__host__ __device__ inline int bias_blocks(const BiasSum& b) { return b.out ? (int)((b.N + 63) / 64) : 0; }
template <class T>
__device__ __forceinline__ void bias_sum(const BiasSum& b, int block, float* sums)
{
    if (block >= bias_blocks(b)) return;
    const int c = threadIdx.x & 63, g = threadIdx.x >> 6;
    const int64_t n = (int64_t)block * 64 + c;
    float s = 0.f;
    if (n < b.N) {
#pragma unroll 8
        for (int64_t r = g; r < b.runs; r += 4) s += b.part[r * b.N + n];
    }
    sums[g * 64 + c] = s;
    __syncthreads();
    if (g || n >= b.N) return;
#pragma unroll
    for (int i = 1; i < 4; ++i) s += sums[i * 64 + c];
    ((unsigned short*)b.out)[n] = T::from_float(s);
}

struct WgParams {
    const char *x, *d;  // x^ and dz in operand order
    int N, K, steps;    // steps of 64 tokens,
    int per, splits;    // of which a block takes `per`; split s > 0 writes N K floats behind split 0's
    int64_t xpitch, dpitch;  // bytes from one block of tokens to the next
    int tilesN, ntiles, band_tiles;
    FastDiv div_band, div_lastband;
    void* dw;
    const float* unit;  // nullable: of the sums
    BiasSum bias;       // blocks behind the tiles'
};

template <int BN, int BK>
struct WgTile {
    static constexpr int WN = BN / 2, WK = BK / 2, TN = WN / 32, TK = WK / 32, NM = TN * TK, SLOTS = 5;
    // a slot: a block of 32 tokens, x^ before dz; a wave's loads of 1 KiB
    static constexpr int XBYTES = BK * 64, SLOT = XBYTES + BN * 64, XDMA = BK / 64, DDMA = BN / 64, DPS = XDMA + DDMA;
    static constexpr int ZPITCH = WK * 4 + 16, ZBYTES = 32 * ZPITCH;
    static constexpr int LDS = SLOTS * SLOT > 4 * ZBYTES ? SLOTS * SLOT : 4 * ZBYTES;
};

template <class T>
__global__ __launch_bounds__(256) void k_bias_sum(BiasSum b)
{
    __shared__ float sums[256];
    bias_sum<T>(b, blockIdx.x, sums);
}

// A block of 4 waves (2 x 2) owns BN x BK of dw.  A step is 64 tokens, two slots of a ring of five; fragments are read one
// 16-token slice ahead, so that before the last slice of a step nothing is left to read of its slots.  Behind the one barrier
// there they are filled again, over the next four slices: first with the second half of the step after next, which then has half
// a step to land, then with the first half of the one after that.
template <class T, int BN, int BK, bool F32>
__global__ __launch_bounds__(256, BN * BK >= 256 * 256 ? 1 : 2) void k_wgrad(WgParams p)
{
    using L = WgTile<BN, BK>;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn = wave >> 1, wk = wave & 1, l32 = lane & 31, h = lane >> 5;
    int tn, tk, split;
    {
        // each XCD has a run of the tiles, then of the sums
        const int blocks = p.ntiles * p.splits, chunk = (blocks + 7) >> 3, at = (int)(blockIdx.x >> 3);
        int bid = (int)(blockIdx.x & 7) * chunk + at;
        if (at >= chunk) {
            bias_sum<T>(p.bias, (at - chunk) * 8 + (int)(blockIdx.x & 7), (float*)smem);
            return;
        }
        if (bid >= blocks) return;
        split = bid / p.ntiles;
        bid -= split * p.ntiles;
        band_tile(bid, p.tilesN, p.band_tiles, [&](int n) { return (int)fastdiv((uint32_t)n, p.div_band); },
                  [&](int n) { return (int)fastdiv((uint32_t)n, p.div_lastband); }, tn, tk);
    }
    const int n0 = tn * BN, k0 = tk * BK, step0 = split * p.per, nk = p.steps - step0 < p.per ? p.steps - step0 : p.per, nh = 2 * nk;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    const int8_t* xg = (const int8_t*)p.x + (int64_t)(k0 / 32) * 2048 + wave * L::XDMA * 1024 + 2 * step0 * p.xpitch;
    const int8_t* dg = (const int8_t*)p.d + (int64_t)(n0 / 32) * 2048 + wave * L::DDMA * 1024 + 2 * step0 * p.dpitch;
    const unsigned voff = (unsigned)lane * 16u;
    // load i of token block q into its slot at LDS address `base`
    auto load_one = [&](auto index, int q, unsigned base) {
        constexpr int i = decltype(index)::value;
        if constexpr (i < L::XDMA)
            dma16_base<i * 1024>(xg + q * p.xpitch, voff + i * 1024, base + (unsigned)(wave * L::XDMA * 1024));
        else
            dma16_base<L::XBYTES + (i - L::XDMA) * 1024>(dg + q * p.dpitch, voff + (i - L::XDMA) * 1024, base + (unsigned)(wave * L::DDMA * 1024));
    };
    auto slot_of = [&](int q) { return q >= 2 * L::SLOTS ? q - 2 * L::SLOTS : q >= L::SLOTS ? q - L::SLOTS : q; };

    f32x16 acc[L::TK][L::TN];
#pragma unroll
    for (int i = 0; i < L::TK; ++i)
#pragma unroll
        for (int j = 0; j < L::TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    u32x4 xf[2][L::TK], df[2][L::TN];
    const int xbase = wk * L::TK * 2048 + lane * 16, dbase = L::XBYTES + wn * L::TN * 2048 + lane * 16;

    // blocks 0 .. 4, of which the first step's two are waited for
    const int first = nh < L::SLOTS ? nh : L::SLOTS;
    for (int q = 0; q < first; ++q)
        for_each_index([&](auto index) { load_one(index, q, lds0 + (unsigned)(q * L::SLOT)); }, std::make_integer_sequence<int, L::DPS>{});
    wait_groups<L::DPS>(first - 2);
    block_barrier();
#pragma unroll
    for (int i = 0; i < L::TK; ++i) xf[0][i] = *(const u32x4*)(smem + xbase + i * 2048);
#pragma unroll
    for (int i = 0; i < L::TN; ++i) df[0][i] = *(const u32x4*)(smem + dbase + i * 2048);

    const std::true_type yes{};
    const std::false_type no{};
    int s0 = 0;  // slot of the step's first block
    // Whether slice 0, slices 1 and 2, and slice 3 load anything: the rest of block 2 step + 3, block 2 step + 4, the first half of
    // block 2 step + 5.
    auto one_step = [&](auto fill0, auto fill12, auto fill3, int step) {
        auto slice = [&](auto index) {
            constexpr int j = decltype(index)::value, cur = j & 1, nxt = cur ^ 1;
            constexpr bool FILL = j == 0 ? decltype(fill0)::value : j == 3 ? decltype(fill3)::value : decltype(fill12)::value;
            if constexpr (j == 3) {
                // the next step has landed, but for the first half of the one behind it; this wave has read all of the present one
                if constexpr (FILL)
                    wait_vm<L::DPS>();
                else
                    wait_vm<0>();
                wait_lgkm0();
                block_barrier();
            }
            // the slot the next slice is read from
            const char* stage = smem + slot_of(s0 + (j == 0 ? 0 : j == 3 ? 2 : 1)) * L::SLOT + ((j + 1) & 1) * 1024;
            // the loads of four slices from a barrier on: part 0 (slice 3) to 3 (slice 2 of the next step), two of a block
            constexpr int part = (j + 1) & 3, DN = L::DPS / 2;
            const int q = 2 * step + (j == 3 ? 5 : 3) + (part >> 1);
            const unsigned base = lds0 + (unsigned)(slot_of(s0 + (j == 3 ? 0 : 3) + (part >> 1)) * L::SLOT);
            for_each_index(
                [&](auto mi) {
                    constexpr int n = decltype(mi)::value, i = n / L::TN, k = i & 1 ? L::TN - 1 - n % L::TN : n % L::TN;  // one operand changes at a time
                    acc[i][k] = T::mfma(xf[cur][i], df[cur][k], acc[i][k]);
                    // the next slice's fragments, early in this one's products
                    constexpr int NF = L::TK + L::TN, PER = (NF + L::NM - 1) / L::NM;
#pragma unroll
                    for (int f = n * PER; f < (n + 1) * PER && f < NF; ++f) {
                        if (f < L::TK)
                            xf[nxt][f < L::TK ? f : 0] = *(const u32x4*)(stage + xbase + f * 2048);
                        else
                            df[nxt][f < L::TK ? 0 : f - L::TK] = *(const u32x4*)(stage + dbase + (f - L::TK) * 2048);
                    }
                    if constexpr (FILL) {
                        constexpr int EVERY = L::NM / DN > 0 ? L::NM / DN : 1, DPER = (DN + L::NM - 1) / L::NM;
                        if constexpr (n % EVERY == EVERY - 1)
                            for_each_index(
                                [&](auto di) {
                                    constexpr int d = n / EVERY * DPER + decltype(di)::value;
                                    if constexpr (d < DN) load_one(std::integral_constant<int, (part & 1) * DN + d>{}, q, base);
                                },
                                std::make_integer_sequence<int, DPER>{});
                    }
                    __builtin_amdgcn_sched_barrier(0);
                },
                std::make_integer_sequence<int, L::NM>{});
        };
        slice(std::integral_constant<int, 0>{});
        slice(std::integral_constant<int, 1>{});
        slice(std::integral_constant<int, 2>{});
        slice(std::integral_constant<int, 3>{});
        s0 = slot_of(s0 + 2);
    };
    // (the first step finds blocks 3 and 4 loaded; the last block is 2 nk - 1)
    int step = 0;
    if (nk > 2) {
        one_step(no, no, yes, step++);
        for (; step < nk - 2; ++step) one_step(yes, yes, yes, step);
        one_step(yes, no, no, step++);
    }
    for (; step < nk; ++step) one_step(no, no, no, step);

    __syncthreads();
    constexpr int CL = L::WK / 8, TPL = CL / 2;
    char* zs = smem + wave * L::ZBYTES;
    const int k8 = k0 + wk * L::WK + (lane % CL) * 8, t0 = (lane / CL) * TPL;
    const float unit = p.unit ? *p.unit : 1.f;
#pragma unroll 1
    for (int k = 0; k < L::TN; ++k) {
        auto put = [&](auto index) {
            constexpr int kk = decltype(index)::value;
            if (kk != k) return;
#pragma unroll
            for (int i = 0; i < L::TK; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(float4*)(zs + l32 * L::ZPITCH + (i * 32 + q * 8 + h * 4) * 4) =
                        make_float4(acc[i][kk][4 * q], acc[i][kk][4 * q + 1], acc[i][kk][4 * q + 2], acc[i][kk][4 * q + 3]);
        };
        for_each_index(put, std::make_integer_sequence<int, L::TN>{});
        wait_lgkm0();
        const int nt = n0 + wn * L::WN + k * 32;
        if (nt >= p.N || k8 >= p.K) continue;
#pragma unroll
        for (int t = 0; t < TPL; ++t) {
            const int n = nt + t0 + t;
            const float* row = (const float*)(zs + (t0 + t) * L::ZPITCH + (lane % CL) * 32);
            const float4 a = *(const float4*)row, b = *(const float4*)(row + 4);
            if (n >= p.N) continue;
            const float v[8] = {a.x * unit, a.y * unit, a.z * unit, a.w * unit, b.x * unit, b.y * unit, b.z * unit, b.w * unit};
            if constexpr (F32) {
                float* o = (float*)p.dw + ((int64_t)split * p.N + n) * p.K + k8;
                if (k8 + 8 <= p.K) {
                    __builtin_memcpy(o, v, 32);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (k8 + i < p.K) o[i] = v[i];
                }
            } else {
                unsigned short* o = (unsigned short*)p.dw + (int64_t)n * p.K + k8;
                if (k8 + 8 <= p.K) {
                    const u32x4 q = {pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])};
                    __builtin_memcpy(o, &q, 16);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (k8 + i < p.K) o[i] = T::from_float(v[i]);
                }
            }
        }
    }
}

template <class T, int BN, int BK, bool F32>
hipError_t run_tile(WgParams& p, hipStream_t st)
{
    using L = WgTile<BN, BK>;
    p.tilesN = (p.N + BN - 1) / BN;
    const int tilesK = (p.K + BK - 1) / BK;
    const int64_t nt = (int64_t)p.tilesN * tilesK;
    const int64_t blocks = (nt * p.splits + 7) / 8 * 8 + bias_blocks(p.bias);
    if (blocks > 0x7fffff00) return hipErrorInvalidValue;
    p.ntiles = (int)nt;
    p.band_tiles = 8 * tilesK;
    p.div_band = make_fastdiv((uint32_t)p.band_tiles);
    p.div_lastband = make_fastdiv((uint32_t)(p.tilesN % 8 ? p.tilesN % 8 : 8));
    static LdsLimit limit;
    const hipError_t e = limit.raise((const void*)&k_wgrad<T, BN, BK, F32>, L::LDS);
    if (e != hipSuccess) return e;
    k_wgrad<T, BN, BK, F32><<<(unsigned)((blocks + 7) / 8 * 8), 256, L::LDS, st>>>(p);
    return hipGetLastError();
}

template <class T, bool F32>
hipError_t run(WgParams& p, int tile, hipStream_t st)
{
    if (tile == 256) return run_tile<T, 256, 256, F32>(p, st);
    if (tile == 128) return run_tile<T, 128, 128, F32>(p, st);
    return run_tile<T, 64, 64, F32>(p, st);
}

// dw = the sum of the splits, in their order
template <class T, bool F32>
__global__ __launch_bounds__(256) void k_wgrad_sum(const float* part, int splits, int64_t n, void* out)
{
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * 1024) {
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        const int m = n - i < 4 ? (int)(n - i) : 4;
        for (int s = 0; s < splits; ++s) {
            const float* q = part + s * n + i;
            if (m == 4) {
                float w[4];
                __builtin_memcpy(w, q, 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += w[e];
            } else {
                for (int e = 0; e < m; ++e) v[e] += q[e];
            }
        }
        for (int e = 0; e < m; ++e) {
            if constexpr (F32)
                ((float*)out)[i + e] = v[e];
            else
                ((unsigned short*)out)[i + e] = T::from_float(v[e]);
        }
    }
}

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

struct BwdWork {
    int64_t dza, dzt, xt, part, range, dwpart, total;
    BwdWork(int64_t M, int64_t N, int64_t K)
    {
        dza = 0;
        dzt = dza + round_up(M * round_up(N, 64) * 2, 256);
        xt = dzt + operand_bytes(M, N);
        part = xt + operand_bytes(M, K);
        const int64_t tb = operand_blocks(M), per = grad_blocks_per_run(M, N);
        range = part + round_up((tb + per - 1) / per * N * 4, 256);
        dwpart = range + round_up(kRangeBytes, 256);
        const WgradForm f = wgrad_form(M, N, K);
        total = dwpart + (f.splits > 1 ? round_up(f.splits * N * K * 4, 256) : 0);
    }
};

hipError_t launch_bias_sum(const BiasSum& b, int f16, hipStream_t st)
{
    if (f16)
        k_bias_sum<F16><<<(unsigned)bias_blocks(b), 256, 0, st>>>(b);
    else
        k_bias_sum<BF16><<<(unsigned)bias_blocks(b), 256, 0, st>>>(b);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_wgrad(const WgradArgs& a, hipStream_t st)
{
    const WgradForm f = wgrad_form(a.M, a.N, a.K);
    WgParams p = {};
    p.x = a.xt, p.d = a.dzt;
    p.N = (int)a.N, p.K = (int)a.K, p.steps = (int)((a.M + 63) / 64);
    p.splits = f.splits, p.per = (p.steps + f.splits - 1) / f.splits;
    p.xpitch = (a.K + 31) / 32 * 2048, p.dpitch = (a.N + 31) / 32 * 2048;
    p.dw = f.splits > 1 ? a.part : a.dw;
    p.unit = a.unit;
    p.bias = a.bias;
    hipError_t e;
    if (a.dw_f32 || f.splits > 1)
        e = a.f16 ? run<F16, true>(p, f.tile, st) : run<BF16, true>(p, f.tile, st);
    else
        e = a.f16 ? run<F16, false>(p, f.tile, st) : run<BF16, false>(p, f.tile, st);
    if (e != hipSuccess || f.splits == 1) return e;
    const int64_t n = a.N * a.K, blocks = (n + 1023) / 1024;
    const unsigned grid = (unsigned)(blocks < 4096 ? blocks : 4096);
    if (a.dw_f32)
        k_wgrad_sum<BF16, true><<<grid, 256, 0, st>>>(a.part, f.splits, n, a.dw);
    else if (a.f16)
        k_wgrad_sum<F16, false><<<grid, 256, 0, st>>>(a.part, f.splits, n, a.dw);
    else
        k_wgrad_sum<BF16, false><<<grid, 256, 0, st>>>(a.part, f.splits, n, a.dw);
    return hipGetLastError();
}

size_t linear_backward_workspace(int64_t M, int64_t N, int64_t K) { return (size_t)BwdWork(M, N, K).total; }

hipError_t launch_linear_backward(const LinearBwdArgs& a, hipStream_t st)
{
    const BwdWork w(a.M, a.N, a.K);
    // a gradient that is dy itself, with one factor for all outputs, is multiplied where it lies
    const bool direct = a.act == kActNone && !a.alpha.ptr;
    GradArgs g = {};
    g.dy = a.dy, g.zq = a.zq, g.xq = a.xq;
    g.M = a.M, g.N = a.N, g.K = a.K, g.lddy = a.lddy, g.lda = round_up(a.N, 64);
    g.alpha = a.alpha, g.act = a.act;
    g.per = grad_blocks_per_run(a.M, a.N);
    g.dza = a.dx && !direct ? a.workspace + w.dza : nullptr;
    g.dzt = a.dw ? a.workspace + w.dzt : nullptr;
    g.xt = a.dw ? a.workspace + w.xt : nullptr;
    g.part = a.dbias ? (float*)(a.workspace + w.part) : nullptr;
    // float16 operands that dz is rounded to, or multiplied by alpha for, are brought into the type's range
    const float* unit = nullptr;
    if (a.f16 && a.M && (g.dza || (g.dzt && a.act != kActNone))) {
        g.range = (unsigned*)(a.workspace + w.range);
        unit = (const float*)(g.range + kRangeParts + 64);
    }
    hipError_t e;
    if (a.M && (e = launch_linear_grad(g, a.f16, st)) != hipSuccess) return e;
    if (a.dx && a.M) {
        LinearArgs l = {};
        l.x = direct ? a.dy : g.dza;
        l.ldx = direct ? a.lddy : g.lda;
        l.w = a.wt;
        l.M = a.M, l.N = a.K, l.K = direct ? a.N : g.lda;
        l.alpha.s = a.alpha.ptr ? 1.f : a.alpha.s;
        l.unit = unit ? unit + 1 : nullptr;
        l.y = a.dx, l.ldy = a.lddx;
        l.f16 = a.f16;
        l.workspace = a.workspace + w.dza;
        if ((e = launch_linear(l, st)) != hipSuccess) return e;
    }
    BiasSum bias = {};
    if (a.dbias) bias = {g.part, (operand_blocks(a.M) + g.per - 1) / g.per, a.N, a.dbias};
    if (a.dw) return launch_linear_wgrad(WgradArgs{g.dzt, g.xt, a.M, a.N, a.K, a.dw, a.f16, a.dw_f32, a.act != kActNone ? unit : nullptr, (float*)(a.workspace + w.dwpart), bias}, st);
    return a.dbias ? launch_bias_sum(bias, a.f16, st) : hipSuccess;
}

}  // namespace rtn
