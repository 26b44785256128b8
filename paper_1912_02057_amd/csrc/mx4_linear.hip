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

// The same with the sums held in place: with 64 of them the compiler would rather write each product's result elsewhere and copy it back, 220
// copies a step.  What reads `c` otherwise has to come behind mx4_settle().
template <int SA, int SB>
__device__ __forceinline__ void mx4_mfma_inplace(u32x4 a, unsigned sa, u32x4 b, unsigned sb, f32x4& c)
{
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0] cbsz:4 blgp:4"
                 : "+a"(c)
                 : "v"(a), "v"(b), "v"(sa), "v"(sb), "n"(SA & 1), "n"(SB & 1), "n"(SA >> 1), "n"(SB >> 1));
#endif
}
// The wait states between a matrix instruction and a vector instruction that reads its result (at most 19 for 16 passes), which the compiler does
// not count for statements like the above.
__device__ __forceinline__ void mx4_settle() { asm volatile("s_nop 15\n\ts_nop 7" ::: "memory"); }

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

// ---- tiles of a full grid
template <int BM, int BN>
struct TileMx4 {
    static constexpr int NS = 4;                                   // stages of 128 columns
    static constexpr int WN = BN / 2, TM = BM / 32, TN = BN / 32;  // a wave's outputs; its blocks of 16 tokens, of 16 outputs
    static constexpr int CODES = (BM + BN) * 64, STAGE = CODES + 4 * 1024, PER = (BM + BN) / 64, DPS = PER + 1;  // (a wave's scales: 1 KiB)
    static constexpr int PITCH = WN * 4 + 16, WAVE = 16 * PITCH;   // 16 tokens of a wave in the epilogue
    static constexpr int LDS = NS * STAGE > 4 * WAVE ? NS * STAGE : 4 * WAVE;
};

template <class T, int BM, int BN>
__global__ __launch_bounds__(256) void k_mx4_tile(Mx4Params p)
{
    using L = TileMx4<BM, BN>;
    static_assert(BM == BN, "a wave loads blocks of one operand");
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn = wave >> 1, wm = wave & 1, nk = p.nk;
    int tm, tn;
    {
        const int chunk = (int)(gridDim.x >> 3), bid = (int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3);
        if (bid >= p.ntiles) return;
        band_tile(bid, p.tilesM, p.band_tiles, [&](int n) { return (int)fastdiv((uint32_t)n, p.div_band); },
                  [&](int n) { return (int)fastdiv((uint32_t)n, p.div_lastband); }, tm, tn);
    }
    const int m0 = tm * BM, n0 = tn * BN;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;

    // ---- direct loads of a stage: waves 0 and 1 the weights' blocks, 2 and 3 the tokens', each half of them and their scales
    const bool mine_w = wave < 2;
    const int8_t* base = mine_w ? p.w : p.a;
    const int blocks = mine_w ? p.wrb : p.arb, b0 = (mine_w ? n0 : m0) / 16, first = (wave & 1) * L::PER;
    const v4i codes = buffer_base(base + (int64_t)b0 * nk * 1024), scales = buffer_base(base + ((int64_t)blocks * 4 + (b0 >> 2)) * nk * 256);
    unsigned off[L::PER], soff;
#pragma unroll
    for (int i = 0; i < L::PER; ++i) {
        const int b = first + i, last = blocks - 1 - b0;
        off[i] = (unsigned)(b < last ? b : last) * (unsigned)(nk * 1024) + (unsigned)(lane * 16);
    }
    {
        // (PER / 4 pieces of 256 bytes; the lanes beyond repeat them, since a branch in the loop would cost more than what they load)
        const int g = first / 4 + (lane >> 4) % (L::PER / 4), last = (blocks - 1) / 4 - b0 / 4;
        soff = (unsigned)(g < last ? g : last) * (unsigned)(nk * 256) + (unsigned)((lane & 15) * 16);
    }
    auto load_one = [&](auto index, int step, unsigned stage) {
        constexpr int i = decltype(index)::value;
        if constexpr (i < L::PER) {
            dma_buf<i * 1024>(codes, off[i], (unsigned)step * 1024u, stage + (unsigned)(wave * L::PER * 1024));
        } else {
            dma_buf<L::CODES>(scales, soff, (unsigned)step * 256u, stage + (unsigned)(wave * 1024));
        }
    };
    auto issue = [&](int step, int slot) {
        for_each_index([&](auto index) { load_one(index, step, lds0 + (unsigned)(slot * L::STAGE)); }, std::make_integer_sequence<int, L::DPS>{});
    };

    f32x4 acc[L::TN][L::TM];
#pragma unroll
    for (int i = 0; i < L::TN; ++i)
#pragma unroll
        for (int j = 0; j < L::TM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // Fragments: the tokens' and the scales of this step and the next; the weights' alone, each read again when its row of products is done.
    u32x4 w[L::TN];
    struct Frags {
        u32x4 a[L::TM];
        unsigned sw[L::TN / 4], sa[L::TM / 4];
    } f[2];
    constexpr int READS = L::TM + L::TN / 4 + L::TM / 4;
    static_assert(READS + L::DPS <= L::TN * L::TM, "one between two products");
    auto read_w = [&](auto index, const char* stage) {
        constexpr int i = decltype(index)::value;
        w[i] = *(const u32x4*)(stage + (wn * L::TN + i) * 1024 + lane * 16);
    };
    auto read_one = [&](auto index, Frags& q, const char* stage) {
        constexpr int i = decltype(index)::value, S = L::TN / 4 + L::TM / 4;
        if constexpr (i < L::TN / 4)
            q.sw[i] = *(const unsigned*)(stage + L::CODES + wn * 1024 + i * 256 + lane * 4);
        else if constexpr (i < S)
            q.sa[i - L::TN / 4] = *(const unsigned*)(stage + L::CODES + (2 + wm) * 1024 + (i - L::TN / 4) * 256 + lane * 4);
        else
            q.a[i - S] = *(const u32x4*)(stage + (BN / 16 + wm * L::TM + i - S) * 1024 + lane * 16);
    };

    for (int s = 0; s < L::NS && s < nk; ++s) issue(s, s);
    wait_groups<L::DPS>((nk < L::NS ? nk : L::NS) - 1);
    block_barrier();
    for_each_index([&](auto index) { read_one(index, f[0], smem); }, std::make_integer_sequence<int, READS>{});
    for_each_index([&](auto index) { read_w(index, smem); }, std::make_integer_sequence<int, L::TN>{});

    int slot = 0;
    // STEADY: step + NS exists, so that it is loaded and no count depends on the step
    auto one_step = [&](auto steady, auto parity, int step) {
        constexpr bool STEADY = decltype(steady)::value;
        Frags &cur = f[decltype(parity)::value], &nxt = f[decltype(parity)::value ^ 1];
        // this step's fragments are in registers, of all waves behind the barrier: its slot is free, and step + 1 has landed
        if constexpr (STEADY) {
            wait_vm<(L::NS - 2) * L::DPS>();
        } else {
            const int later = nk - 2 - step;
            wait_groups<L::DPS>(later < L::NS - 2 ? later : L::NS - 2);
        }
        wait_lgkm0();
        block_barrier();
        const int next = slot + 1 == L::NS ? 0 : slot + 1;
        const char* stage = smem + next * L::STAGE;
        const unsigned fill = lds0 + (unsigned)(slot * L::STAGE);
        for_each_index(
            [&](auto mi) {
                constexpr int n = decltype(mi)::value, i = n / L::TM, j = i & 1 ? L::TM - 1 - n % L::TM : n % L::TM;
                mx4_mfma_inplace<(i & 3), (j & 3)>(w[i], cur.sw[i / 4], cur.a[j], cur.sa[j / 4], acc[i][j]);
                // (behind the last step: what the slot holds, which nothing takes)
                if constexpr (n < READS) {
                    read_one(mi, nxt, stage);
                } else if constexpr (STEADY && n - READS < L::DPS) {
                    load_one(std::integral_constant<int, n - READS>{}, step + L::NS, fill);
                }
                if constexpr (n % L::TM == L::TM - 1) read_w(std::integral_constant<int, i>{}, stage);
                __builtin_amdgcn_sched_barrier(0);
            },
            std::make_integer_sequence<int, L::TN * L::TM>{});
        if (!STEADY && step + L::NS < nk) issue(step + L::NS, slot);
        slot = next;
    };
    const std::true_type yes{};
    const std::false_type no{};
    const std::integral_constant<int, 0> even{};
    const std::integral_constant<int, 1> odd{};
    int step = 0;
    for (; step + 1 + L::NS < nk; step += 2) {
        one_step(yes, even, step);
        one_step(yes, odd, step + 1);
    }
    for (; step < nk; step += 2) {
        one_step(no, even, step);
        if (step + 1 < nk) one_step(no, odd, step + 1);
    }

    mx4_settle();
    // ---- epilogue: 16 tokens of the wave at a time through LDS, after which a lane has 8 outputs of a token, in TPL passes
    __syncthreads();
    constexpr int CL = L::WN / 8, TPL = 16 * CL / 64;
    char* zs = smem + wave * L::WAVE;
    const int nw = n0 + wn * L::WN, n8 = nw + (lane % CL) * 8, t0 = lane / CL;
    if (nw >= p.N) return;
    u32x4 res[TPL];
    auto fetch = [&](int k) {
#pragma unroll
        for (int t = 0; t < TPL; ++t) {
            const int m = m0 + wm * (BM / 2) + k * 16 + t * (64 / CL) + t0;
            res[t] = m < p.M ? load_row8(p.res + m * p.ldr, n8, p.N) : u32x4{0, 0, 0, 0};
        }
    };
    float bi[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) bi[i] = p.bias && n8 + i < p.N ? T::to_float(p.bias[n8 + i]) : 0.f;
    if (p.res) fetch(0);
#pragma unroll 1
    for (int k = 0; k < L::TM; ++k) {
        const int mt = m0 + wm * (BM / 2) + k * 16;
        if (mt >= p.M) break;
        for_each_index(
            [&](auto index) {
                constexpr int j = decltype(index)::value;
                if (j != k) return;
#pragma unroll
                for (int i = 0; i < L::TN; ++i)
                    *(float4*)(zs + (lane & 15) * L::PITCH + (i * 16 + 4 * (lane >> 4)) * 4) = make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
            },
            std::make_integer_sequence<int, L::TM>{});
        u32x4 now[TPL];
#pragma unroll
        for (int t = 0; t < TPL; ++t) now[t] = res[t];
        if (p.res && k + 1 < L::TM) fetch(k + 1);
        wait_lgkm0();
#pragma unroll
        for (int t = 0; t < TPL; ++t) {
            const int row = t * (64 / CL) + t0;
            const float* q = (const float*)(zs + row * L::PITCH + (lane % CL) * 32);
            const float4 a = *(const float4*)q, b = *(const float4*)(q + 4);
            float z[8] = {a.x + bi[0], a.y + bi[1], a.z + bi[2], a.w + bi[3], b.x + bi[4], b.y + bi[5], b.z + bi[6], b.w + bi[7]};
            finish_row<T>(p, mt + row, n8, z, now[t]);
        }
        // (the next round's writes to `zs` are this wave's own and come after its reads)
    }
}

template <class T, int BM, int BN>
hipError_t run_tile(Mx4Params& p, hipStream_t st)
{
    using L = TileMx4<BM, BN>;
    p.tilesM = (p.M + BM - 1) / BM;
    const int tilesN = (p.N + BN - 1) / BN;
    const int64_t nt = (int64_t)p.tilesM * tilesN;
    if (nt > 0x7fffff00) return hipErrorInvalidValue;
    p.ntiles = (int)nt;
    p.band_tiles = 8 * tilesN;
    p.div_band = make_fastdiv((uint32_t)p.band_tiles);
    p.div_lastband = make_fastdiv((uint32_t)(p.tilesM % 8 ? p.tilesM % 8 : 8));
    static LdsLimit limit;
    const hipError_t e = limit.raise((const void*)&k_mx4_tile<T, BM, BN>, L::LDS);
    if (e != hipSuccess) return e;
    k_mx4_tile<T, BM, BN><<<(unsigned)((nt + 7) / 8 * 8), 256, L::LDS, st>>>(p);
    return hipGetLastError();
}

template <class T>
hipError_t run(Mx4Params& p, hipStream_t st)
{
    auto blocks = [&](int64_t m, int64_t n) { return (p.M + m - 1) / m * ((p.N + n - 1) / n); };
    if (blocks(256, 256) >= 192) return run_tile<T, 256, 256>(p, st);
    if (blocks(128, 128) >= 192) return run_tile<T, 128, 128>(p, st);
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
