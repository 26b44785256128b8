// Ternary linear layer of 16-bit activations: y = act(alpha (x t^T) + bias) + residual, on the bf16 / fp16 matrix cores.
//
// The weights are two bits each in the order the matrix instruction takes them (WeightShape); a register of two weights is
// a shift and an AND away from its word (-2, 0, +2; the halves are made up for in alpha).  Products with them are exact; sums
// are the instruction's fp32 accumulators, along the columns in one order per form, and y is rounded once.
//
// Three kernels, chosen by the sizes (linear_form): k_linear_few for a token or a few, bound by the weights' bytes and their
// widening; k_linear_split for grids that do not fill the chip, bound by the latency of its loads and by the bytes of x that
// pass through a CU; k_linear, tiles of a full grid, bound by the power limit of the matrix cores.
#include "linear_math.h"
#include "tmm_kernel.h"

namespace rtn {

namespace {

struct LinParams {
    const int8_t* x;
    const int8_t* w;
    int M, N, K;
    int64_t ldx, ldr, ldy;  // elements
    int nk;                 // 64-column steps = column blocks of the prepared weights
    int rb;                 // row blocks of the prepared weights
    int tilesM, ntiles, band_tiles;
    FastDiv div_band, div_lastband;
    Param alpha;
    const float* unit;      // nullable: a factor of alpha
    const unsigned short *bias, *res;
    unsigned short* y;
    int8_t* zq;
    int act;
};

// What the sums are multiplied by beside alpha: the weights' operands are twice the weights.
__device__ __forceinline__ float sum_unit(const LinParams& p) { return p.unit ? 0.5f * *p.unit : 0.5f; }

// The parameters of 8 consecutive outputs (0 past the end).
template <class T>
__device__ __forceinline__ void load_affine(const LinParams& p, int n, float (&al)[8], float (&bi)[8])
{
    const float unit = sum_unit(p);
    if (n + 8 <= p.N) {
        if (p.alpha.ptr) {
            __builtin_memcpy(al, p.alpha.ptr + n, 32);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) al[i] = p.alpha.s;
        }
        u32x4 b = {0, 0, 0, 0};
        if (p.bias) b = load16(p.bias + n);
#pragma unroll
        for (int i = 0; i < 8; ++i) al[i] *= unit, bi[i] = half_of<T>(b[i >> 1], i & 1);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool in = n + i < p.N;
            al[i] = in ? unit * (p.alpha.ptr ? p.alpha.ptr[n + i] : p.alpha.s) : 0.f;
            bi[i] = in && p.bias ? T::to_float(p.bias[n + i]) : 0.f;
        }
    }
}

// Eight outputs, of which the first `left` exist, rounded
template <class T>
__device__ __forceinline__ void store_row8(unsigned short* y, int left, const float (&v)[8])
{
    if (left >= 8) {
        store16(y, u32x4{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])});
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) y[i] = T::from_float(v[i]);
    }
}
// act(z) + residual of outputs n .. n + 7 of row m -> y
template <class T, int ACT>
__device__ __forceinline__ void finish_row(const LinParams& p, int m, int n, const float (&z)[8])
{
    if (m >= p.M || n >= p.N) return;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = act_value<ACT>(z[i]);
    if (p.res) {
        const u32x4 q = load_row8(p.res + m * p.ldr, n, p.N);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += half_of<T>(q[i >> 1], i & 1);
    }
    store_row8<T>(p.y + m * p.ldy + n, p.N - n, v);
}

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

// Scales of 8 channels from the largest magnitudes (as bits) of their groups
template <class T>
struct CkptScale {
    unsigned ex[2];
    float inv[8];
    bool clamp;
    CkptScale() = default;
    __device__ __forceinline__ CkptScale(const unsigned (&am)[8])
    {
        bool end = false;
        ex[0] = ex[1] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = ckpt_exponent<T>(__uint_as_float(am[i]));
            ex[i >> 2] |= (unsigned)e << (8 * (i & 3));
            inv[i] = ckpt_inverse(e);
            end |= e == T::kMostExp + 127;
        }
        clamp = __any(end);
    }
};
template <class T>
__device__ __forceinline__ void store_scales(const LinParams& p, int mt, int n, const CkptScale<T>& s)
{
    const CkptShape cs(p.M, p.N);
    *(uint2*)(p.zq + cs.codes() + ((int64_t)(mt >> 5) * cs.cb + (n >> 3)) * 8) = make_uint2(s.ex[0], s.ex[1]);
}
// The codes of R tokens from mt + t0 on
template <class T, int R>
__device__ __forceinline__ void store_codes(const LinParams& p, int mt, int t0, int n, const float (&z)[R][8], const CkptScale<T>& s)
{
    const CkptShape cs(p.M, p.N);
    int8_t* out = p.zq + ((int64_t)(mt >> 5) * cs.cb + (n >> 3)) * 256 + t0 * 8;
    unsigned w[R * 2];
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
        for (int q = 0; q < 2; ++q)
            w[2 * t + q] = ckpt_codes(z[t][4 * q], z[t][4 * q + 1], z[t][4 * q + 2], z[t][4 * q + 3], s.inv[4 * q], s.inv[4 * q + 1],
                                      s.inv[4 * q + 2], s.inv[4 * q + 3], s.clamp);
    if constexpr (R > 1) {
#pragma unroll
        for (int i = 0; i < R; i += 2) *(uint4*)(out + 8 * i) = make_uint4(w[2 * i], w[2 * i + 1], w[2 * i + 2], w[2 * i + 3]);
    } else {
        *(uint2*)out = make_uint2(w[0], w[1]);
    }
}

// Eight two-bit codes of a lane (registers 4 (slice & 1) .. + 3 of the word) -> operand.
template <int SLICE>
__device__ __forceinline__ u32x4 expand(uint2 word)
{
    const unsigned w = SLICE & 2 ? word.y : word.x;
    constexpr int r = 4 * (SLICE & 1);
    return u32x4{(w << 2 * r) & kCodeMask, (w << (2 * r + 2)) & kCodeMask, (w << (2 * r + 4)) & kCodeMask, (w << (2 * r + 6)) & kCodeMask};
}

template <int BM, int BN, int NS>
struct LinTile {
    static constexpr int WN = BN / 4, TM = BM / 32, TN = WN / 32, NM = TM * TN;
    static constexpr int ABYTES = BM * 128, STAGE = ABYTES + BN * 16, XDMA = BM / 32, DPS = XDMA + 1;
    static constexpr int ZPITCH = WN * 4 + 16, ZBYTES = 32 * ZPITCH;  // a wave's 32 rows of fp32 in the epilogue
    static constexpr int LDS = NS * STAGE > 4 * ZBYTES ? NS * STAGE : 4 * ZBYTES;
};

// A block of 4 waves owns BM tokens x BN outputs, a wave all the tokens of a quarter of the outputs, so that no weight is widened
// twice: large products are bound by the power limit (clock 1.5 to 1.7 GHz while the matrix cores are busy 88 % of it), and with the
// waves 2 x 2 instead the redundant vector operations cost 3 %: 16384 x 8192 x 8192 1540 us against 1490.  Two blocks share a CU, so one's
// epilogue passes beside the other's products (one block of 256 x 256: 1660 us).  Ring of NS stages of 64 columns: x rows of 128 bytes, 16-byte
// chunk c of row r at place c ^ (r >> 1 & 7), so that 16 rows' fragments hit all banks; then the weights' words.  One barrier per
// step, before the last of its four 16-column slices, and fragments are read one slice ahead.  x is the instruction's first
// operand: it takes 4 % less time at the power limit with the ternary values as the second (1490 -> 1430 us).  Per step of 64 columns a wave has 32 matrix
// instructions (128 x 256), 64 vector operations that widen weights, 16 + 2 fragment reads and 5 direct loads, spread between
// them.  16384 x 8192 x 8192: 1397 us, 1574 TFLOP/s (a large library product of such values reaches 1665); 4096^3 with gelu
// 98 us, of which the launch, the first loads and the epilogue (33.5 MB of y, the activation on the vector ALU) are 13.
template <class T, int BM, int BN, int NS>
__global__ __launch_bounds__(256, 2) void k_linear(LinParams p)
{
    using L = LinTile<BM, BN, NS>;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, h = lane >> 5;

    int tm, tn;
    {
        const int chunk = (int)(gridDim.x >> 3), bid = (int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3);
        if (bid >= p.ntiles) return;
        band_tile(bid, p.tilesM, p.band_tiles, [&](int n) { return (int)fastdiv((uint32_t)n, p.div_band); },
                  [&](int n) { return (int)fastdiv((uint32_t)n, p.div_lastband); }, tm, tn);
    }
    const int m0 = tm * BM, n0 = tn * BN, nk = p.nk;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem;

    // ---- direct loads of a stage
    const v4i xr = buffer_base(p.x + (int64_t)m0 * p.ldx * 2), wr = buffer_base(p.w + (int64_t)(n0 / 32) * nk * 512);
    unsigned xoff[L::XDMA];
#pragma unroll
    for (int i = 0; i < L::XDMA; ++i) {
        const int row = (wave * L::XDMA + i) * 8 + (lane >> 3), last = p.M - 1 - m0;
        xoff[i] = (unsigned)(row < last ? row : last) * (unsigned)(p.ldx * 2) + (unsigned)(((lane & 7) ^ ((row >> 1) & 7)) * 16);
    }
    unsigned woff;
    {
        const int at = wave * BN * 4 + lane * 16, last = p.rb - 1 - n0 / 32, r = at >> 9;
        woff = (unsigned)(r < last ? r : last) * (unsigned)(nk * 512) + (unsigned)(at & 511);
    }
    const int ktail = p.K & 63;
    // load i of step `step`, into the stage at LDS address `base`; TAIL: it may be the last one, whose chunks past the rows' ends are zeros
    auto load_one = [&](auto index, auto may_end, int step, unsigned base) {
        constexpr int i = decltype(index)::value;
        if constexpr (i < L::XDMA) {
            unsigned v = xoff[i];
            if constexpr (decltype(may_end)::value) {
                const int row = (wave * L::XDMA + i) * 8 + (lane >> 3);
                if (ktail && step == nk - 1 && ((lane & 7) ^ ((row >> 1) & 7)) * 8 >= ktail) v = kOutside;
            }
            dma_buf<i * 1024>(xr, v, (unsigned)step * 128u, base + (unsigned)(wave * L::XDMA * 1024));
        } else {
            if (lane < BN / 4) dma_buf<L::ABYTES>(wr, woff, (unsigned)step * 512u, base + (unsigned)(wave * BN * 4));
        }
    };
    const std::true_type yes{};
    const std::false_type no{};
    auto issue = [&](int step, int slot) {
        for_each_index([&](auto index) { load_one(index, yes, step, lds0 + (unsigned)(slot * L::STAGE)); }, std::make_integer_sequence<int, L::DPS>{});
    };

    f32x16 acc[L::TN][L::TM];
#pragma unroll
    for (int i = 0; i < L::TN; ++i)
#pragma unroll
        for (int j = 0; j < L::TM; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    u32x4 xf[2][L::TM], wf[2][L::TN];
    uint2 words[L::TN];
    const int xbase = l32 * 128 + ((h ^ ((l32 >> 1) & 7)) * 16), wbase = L::ABYTES + wave * L::TN * 512 + lane * 8;

    for (int s = 0; s < NS - 1 && s < nk; ++s) issue(s, s);
    wait_groups<L::DPS>((nk < NS - 1 ? nk : NS - 1) - 1);
    block_barrier();
    int slot = 0;  // of the current step
#pragma unroll
    for (int i = 0; i < L::TN; ++i) words[i] = *(const uint2*)(smem + wbase + i * 512);
#pragma unroll
    for (int i = 0; i < L::TM; ++i) xf[0][i] = *(const u32x4*)(smem + xbase + i * 4096);
#pragma unroll
    for (int i = 0; i < L::TN; ++i) wf[0][i] = expand<0>(words[i]);

    // STEADY: at least NS steps follow, so one more is loaded and no count depends on the step
    auto one_step = [&](auto steady, int step) {
        constexpr bool STEADY = decltype(steady)::value;
        const int next = slot + 1 == NS ? 0 : slot + 1;
        const unsigned fill = lds0 + (unsigned)((slot == 0 ? NS - 1 : slot - 1) * L::STAGE);
        auto slice = [&](auto index) {
            constexpr int j = decltype(index)::value, cur = j & 1, nxt = cur ^ 1;
            if constexpr (j == 3) {
                // step + 1 has landed for this wave, then for all; and all are done with step - 1, whose slot is filled again
                if constexpr (STEADY) {
                    wait_vm<(NS - 3) * L::DPS>();
                } else {
                    const int later = nk - 2 - step;
                    wait_groups<L::DPS>(later < NS - 3 ? later : NS - 3);
                }
                block_barrier();
                if (!STEADY && step + NS - 1 < nk) issue(step + NS - 1, slot == 0 ? NS - 1 : slot - 1);
            }
            const char* stage = smem + (j == 3 ? next : slot) * L::STAGE;
            uint2 ahead[L::TN];
            constexpr int NF = (j == 3 ? L::TN : 0) + L::TM, FPER = (NF + L::NM - 1) / L::NM;  // fragment reads, front-loaded
            constexpr int ND = j == 3 && STEADY ? L::DPS : 0, DPER = (ND + L::NM - 1) / L::NM;
            auto read = [&](int f) {
                if (j == 3 && f < L::TN)
                    ahead[f < L::TN ? f : 0] = *(const uint2*)(stage + wbase + f * 512);
                else {
                    const int i = j == 3 ? f - L::TN : f;
                    xf[nxt][i] = *(const u32x4*)(stage + (xbase ^ (32 * ((j + 1) & 3))) + i * 4096);
                }
            };
            auto widen = [&](int e) {
                wf[nxt][e] = expand<(j + 1) & 3>(j == 3 ? ahead[e] : words[e]);
#pragma unroll
                for (int r = 0; r < 4; ++r) {  // here, not where they are used: they would all sit in front of the next slice
                    unsigned u = wf[nxt][e][r];
                    pin(u);
                    wf[nxt][e][r] = u;
                }
            };
            for_each_index(
                [&](auto mi) {
                    constexpr int n = decltype(mi)::value, i = n / L::TM, k = i & 1 ? L::TM - 1 - n % L::TM : n % L::TM;  // one operand changes at a time
                    acc[i][k] = T::mfma(xf[cur][k], wf[cur][i], acc[i][k]);
#pragma unroll
                    for (int f = n * FPER; f < (n + 1) * FPER && f < NF; ++f) read(f);
                    for_each_index(
                        [&](auto di) {
                            constexpr int d = n * DPER + decltype(di)::value;
                            if constexpr (d < ND) load_one(std::integral_constant<int, d>{}, no, step + NS - 1, fill);
                        },
                        std::make_integer_sequence<int, DPER>{});
                    // the next slice's weights, in the second half of this one's products
                    constexpr int first = L::NM / 2, left = L::NM - first, per = (L::TN + left - 1) / left, every = left / L::TN > 0 ? left / L::TN : 1;
                    if constexpr (n >= first && (n - first) % every == 0) {
#pragma unroll
                        for (int e = (n - first) / every * per; e < ((n - first) / every + 1) * per && e < L::TN; ++e) widen(e);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                },
                std::make_integer_sequence<int, L::NM>{});
            if constexpr (j == 3) {
#pragma unroll
                for (int i = 0; i < L::TN; ++i) words[i] = ahead[i];
            }
        };
        slice(std::integral_constant<int, 0>{});
        slice(std::integral_constant<int, 1>{});
        slice(std::integral_constant<int, 2>{});
        slice(std::integral_constant<int, 3>{});
        slot = next;
    };
    int step = 0;
    for (; step < nk - NS; ++step) one_step(yes, step);
    for (; step < nk; ++step) one_step(no, step);

    // ---- epilogue: 32 tokens of the wave's tile at a time through LDS, after which a lane has 8 outputs of TPL tokens
    __syncthreads();
    constexpr int CL = L::WN / 8, TPL = CL / 2;
    char* zs = smem + wave * L::ZBYTES;
    const int nw = n0 + wave * L::WN, n8 = nw + (lane % CL) * 8, t0 = (lane / CL) * TPL;
    if (nw >= p.N) return;
    const float unit = sum_unit(p);
    float al[L::TN], bi[L::TN];  // of the columns that this lane has in its accumulators
#pragma unroll
    for (int i = 0; i < L::TN; ++i) {
        const int n = nw + i * 32 + l32;
        al[i] = bi[i] = 0.f;
        if (n < p.N) {
            al[i] = unit * (p.alpha.ptr ? p.alpha.ptr[n] : p.alpha.s);
            if (p.bias) bi[i] = T::to_float(p.bias[n]);
        }
    }
    // the residual of the rows of a round, fetched before they pass through LDS
    u32x4 res[TPL];
    auto fetch = [&](int k) {
        const int mt = m0 + k * 32 + t0;
        const unsigned short* r = p.res + mt * p.ldr;
        if (mt + TPL <= p.M && nw + L::WN <= p.N) {
#pragma unroll
            for (int t = 0; t < TPL; ++t) res[t] = load16(r + t * p.ldr + n8);
        } else {
#pragma unroll
            for (int t = 0; t < TPL; ++t) res[t] = mt + t < p.M ? load_row8(r + t * p.ldr, n8, p.N) : u32x4{0, 0, 0, 0};
        }
    };
#pragma unroll 1
    for (int k = 0; k < L::TM; ++k) {
        const int mt = m0 + k * 32;  // first token
        if (mt >= p.M) break;
        if (p.res) fetch(k);
        auto put = [&](auto index) {
            constexpr int kk = decltype(index)::value;
            if (kk != k) return;
#pragma unroll
            for (int i = 0; i < L::TN; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)  // row 8 (r / 4) + 4 h + r % 4, column l32
                    *(float*)(zs + (8 * (r >> 2) + 4 * h + (r & 3)) * L::ZPITCH + (i * 32 + l32) * 4) = fmaf(acc[i][kk][r], al[i], bi[i]);
        };
        for_each_index(put, std::make_integer_sequence<int, L::TM>{});
        const bool whole = mt + 32 <= p.M && nw + L::WN <= p.N;
        wait_lgkm0();
        auto read_z = [&](int t, float(&z)[8]) {
            const float* row = (const float*)(zs + (t0 + t) * L::ZPITCH + (lane % CL) * 32);
            const float4 a = *(const float4*)row, b = *(const float4*)(row + 4);
            z[0] = a.x, z[1] = a.y, z[2] = a.z, z[3] = a.w, z[4] = b.x, z[5] = b.y, z[6] = b.z, z[7] = b.w;
            if (!whole) {  // (a checkpoint's tokens past the end are zeros)
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = mt + t0 + t < p.M ? z[i] : 0.f;
            }
        };
        CkptScale<T> scale;
        if (p.zq) {
            unsigned am[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < TPL; ++t) {
                float z[8];
                read_z(t, z);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const unsigned u = __float_as_uint(z[i]) & 0x7fffffffu;
                    am[i] = u > am[i] ? u : am[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int d = CL; d < 64; d *= 2) {
                    const unsigned o = (unsigned)__shfl_xor((int)am[i], d);
                    am[i] = o > am[i] ? o : am[i];
                }
            scale = CkptScale<T>(am);
            if (t0 == 0 && n8 < p.N) store_scales(p, mt, n8, scale);
        }
        unsigned short* y = p.y + (mt + t0) * p.ldy + n8;
        with_act(p.act, [&](auto which) {
            constexpr int ACT = decltype(which)::value;
#pragma unroll
            for (int r = 0; r < TPL; r += 2) {  // two rows at a time: more do not fit beside the accumulators
                float z[2][8];
                read_z(r, z[0]);
                read_z(r + 1, z[1]);
                if (p.zq && n8 < p.N) store_codes<T, 2>(p, mt, t0 + r, n8, z, scale);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[t][i] = act_value<ACT>(z[t][i]);
                    if (p.res) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) z[t][i] += half_of<T>(res[r + t][i >> 1], i & 1);
                    }
                    if (whole)
                        store16(y + (r + t) * p.ldy, u32x4{pack2<T>(z[t][0], z[t][1]), pack2<T>(z[t][2], z[t][3]), pack2<T>(z[t][4], z[t][5]), pack2<T>(z[t][6], z[t][7])});
                    else if (mt + t0 + r + t < p.M)
                        store_row8<T>(y + (r + t) * p.ldy, p.N - n8, z[t]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        });
        // (the next round's writes to `zs` are this wave's own and come after its reads)
    }
}

// A few tokens (at most 16): a block has 16 RB outputs, its waves share the columns, the weights are read once and x and weights
// go straight into registers.  v_mfma 16x16x32 takes row l & 15, columns 8 (l >> 4) .. + 7 from lane l, which lane
// (l & 15) + 16 half + 32 (l >> 4 & 1) of the 32-row order has, in the word's first four registers (slice 2 s) or its last.
// Bound by the widening of the weights, two vector operations for two of them, and for small layers by latencies: the launch, what the
// outputs need, then a round of loads for every BATCH steps of a wave, each waited for before the next is issued.
template <class T, int RB, int WAVES, int BATCH, bool ROW16>
__global__ __launch_bounds__(WAVES * 64) void k_linear_few(LinParams p)
{
    __shared__ float part[WAVES][kFewTokens][RB * 16 + 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, c = lane >> 4;
    const int n0 = blockIdx.x * 16 * RB;
    f32x4 acc[RB][2];  // the instruction's result is late for the next one on the same registers
#pragma unroll
    for (int r = 0; r < RB; ++r) acc[r][0] = acc[r][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bool mine = l16 < p.M;  // the other lanes' columns of the result are not looked at, whatever they hold
    const auto xr = __builtin_amdgcn_make_buffer_rsrc((void*)p.x, 0, (int)(((p.M - 1) * p.ldx + p.K) * 2), 0x00020000);
    const int xoff = (int)(l16 * p.ldx * 2) + c * 16;
    int woff[RB];
    const int rb0 = (int)(blockIdx.x * RB) >> 1, rbs = p.rb - rb0;  // (a block of 32 rows holds two of 16)
    const auto wr = __builtin_amdgcn_make_buffer_rsrc((void*)(p.w + (int64_t)rb0 * p.nk * 512), 0, rbs < (RB + 1) / 2 ? rbs * p.nk * 512 : (RB + 1) / 2 * p.nk * 512, 0x00020000);
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int r16 = (int)(blockIdx.x * RB) + r;  // (rows of no block read as zeros)
        woff[r] = ((r16 >> 1) - rb0) * p.nk * 512 + (l16 + 16 * (r16 & 1) + 32 * (c & 1)) * 8;
    }
    const int up = c & 2 ? 8 : 0;
    const unsigned short* xrow = (const unsigned short*)p.x + (int64_t)l16 * p.ldx;
    auto load_x = [&](int step, int s) {
        if constexpr (ROW16) {
            return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xr, xoff, step * 128 + 64 * s, 0));
        } else {
            return load_row8(xrow, step * 64 + 32 * s + 8 * c, p.K);
        }
    };
    // What the outputs need beside the sums: thread 16 RB m + i has output i of token m.  (Converted where they are loaded, so that a wave
    // that has outputs waits for them before its first weights.)
    constexpr int OUTS = 16 * RB, PER = (kFewTokens * OUTS + WAVES * 64 - 1) / (WAVES * 64);
    const float unit = sum_unit(p);
    float al[PER], bi[PER], re[PER];
#pragma unroll
    for (int o = 0; o < PER; ++o) {
        const int at = tid + o * WAVES * 64, om = at / OUTS, on = n0 + at % OUTS;
        al[o] = bi[o] = re[o] = 0.f;
        if (om >= p.M || on >= p.N) continue;
        al[o] = unit * (p.alpha.ptr ? p.alpha.ptr[on] : p.alpha.s);
        if (p.bias) bi[o] = T::to_float(p.bias[on]);
        if (p.res) re[o] = T::to_float(p.res[om * p.ldr + on]);
    }
    for (int s0 = wave; s0 < p.nk; s0 += WAVES * BATCH) {
        uint2 word[BATCH][RB];
        u32x4 xf[BATCH][2];
        // past the last step: that one again, with x of zero (weights of zero would make a NaN of an infinity in x)
        auto step_at = [&](int b) {
            const int step = s0 + b * WAVES;
            return step < p.nk ? step : p.nk - 1;
        };
#pragma unroll
        for (int b = 0; b < BATCH; ++b)
#pragma unroll
            for (int r = 0; r < RB; ++r)
                word[b][r] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(wr, woff[r], step_at(b) * 512, 0));
        if (mine)
#pragma unroll
            for (int b = 0; b < BATCH; ++b)
#pragma unroll
                for (int s = 0; s < 2; ++s) xf[b][s] = load_x(step_at(b), s);
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int left = p.K - (s0 + b * WAVES) * 64;  // columns from the step on; 0 or less behind the last one
            if (ROW16 ? left < 64 : left <= 0) {
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    if (32 * s + 8 * c >= left) xf[b][s] = u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                const uint2 w2 = make_uint2(word[b][r].x << up, word[b][r].y << up);
                acc[r][0] = T::mfma16(expand<0>(w2), xf[b][0], acc[r][0]);
                acc[r][1] = T::mfma16(expand<2>(w2), xf[b][1], acc[r][1]);
            }
        }
    }
    if (mine)
#pragma unroll
        for (int r = 0; r < RB; ++r)
            *(float4*)&part[wave][l16][r * 16 + 4 * c] = make_float4(acc[r][0][0] + acc[r][1][0], acc[r][0][1] + acc[r][1][1],
                                                                     acc[r][0][2] + acc[r][1][2], acc[r][0][3] + acc[r][1][3]);
    __syncthreads();
#pragma unroll
    for (int o = 0; o < PER; ++o) {
        const int at = tid + o * WAVES * 64, om = at / OUTS, i = at % OUTS;
        if (om >= p.M || n0 + i >= p.N) continue;
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) s += part[v][om][i];
        const float z = fmaf(s, al[o], bi[o]);
        with_act(p.act, [&](auto which) {
            p.y[om * p.ldy + n0 + i] = T::from_float(act_value<decltype(which)::value>(z) + re[o]);
        });
    }
}

template <int TT, int RB, int WAVES, int D>
struct SplitTile {
    static constexpr int XBYTES = TT * 4096, STAGE = XBYTES + RB * 512, DPS = TT * 4 + 1;
    static constexpr int ZPITCH = RB * 128 + 16, ZBYTES = TT * 32 * ZPITCH;
    static constexpr int WAVE = D * STAGE > ZBYTES ? D * STAGE : ZBYTES;
    static constexpr int LDS = WAVES * WAVE + TT * RB * 128;
};

// Small grids: a block has 32 TT tokens x 32 RB outputs and its waves share the columns, every WAVES-th step each, with rings
// of their own in LDS (D stages) and no barrier until their sums are added up in LDS.  ROW16: rows of whole 16-byte units, which
// direct loads bring there; any others come through registers, two steps ahead (1000 x 1003 x 2187 with gelu: 13.7 us, rows copied into
// such units first 15.5).
template <class T, int TT, int RB, int WAVES, int D, bool ROW16>
__global__ __launch_bounds__(WAVES * 64) void k_linear_split(LinParams p)
{
    using L = SplitTile<TT, RB, WAVES, D>;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, h = lane >> 5;
    const int nk = p.nk, tn = (int)blockIdx.x / p.tilesM, tm = (int)blockIdx.x - tn * p.tilesM;
    const int m0 = tm * 32 * TT, n0 = tn * 32 * RB;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)smem + (unsigned)(wave * L::WAVE);
    char* ring = smem + wave * L::WAVE;
    unsigned* amax = (unsigned*)(smem + WAVES * L::WAVE);  // [TT][32 RB]
    if (tid < TT * RB * 32) amax[tid] = 0;

    const v4i xr = buffer_base(p.x + (int64_t)m0 * p.ldx * 2), wr = buffer_base(p.w + (int64_t)(n0 / 32) * nk * 512);
    unsigned xoff[TT * 4];
#pragma unroll
    for (int i = 0; i < TT * 4; ++i) {
        const int row = i * 8 + (lane >> 3), last = p.M - 1 - m0;
        xoff[i] = (unsigned)(row < last ? row : last) * (unsigned)(p.ldx * 2) + (unsigned)(((lane & 7) ^ ((row >> 1) & 7)) * 16);
    }
    unsigned woff;
    {
        const int last = p.rb - 1 - n0 / 32, r = lane >> 5;
        woff = (unsigned)(r < last ? r : last) * (unsigned)(nk * 512) + (unsigned)((lane & 31) * 16);
    }
    const int ktail = p.K & 63;
    auto issue = [&](int step, int slot) {
        const unsigned base = lds0 + (unsigned)(slot * L::STAGE);
        const bool end = ktail && step == nk - 1;  // chunks past the rows' ends are zeros
        for_each_index(
            [&](auto index) {
                constexpr int i = decltype(index)::value;
                const int row = i * 8 + (lane >> 3);
                const unsigned v = end && ((lane & 7) ^ ((row >> 1) & 7)) * 8 >= ktail ? kOutside : xoff[i];
                dma_buf<i * 1024>(xr, v, (unsigned)step * 128u, base);
            },
            std::make_integer_sequence<int, TT * 4>{});
        if (lane < RB * 32) dma_buf<L::XBYTES>(wr, woff, (unsigned)step * 512u, base);
    };

    f32x16 acc[RB][TT];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    const int xbase = l32 * 128 + ((h ^ ((l32 >> 1) & 7)) * 16), wbase = L::XBYTES + lane * 8;
    const int count = wave < nk ? (nk - wave + WAVES - 1) / WAVES : 0;
    auto products = [&](const u32x4(&xf)[4][TT], const uint2(&words)[RB]) {
        for_each_index(
            [&](auto index) {
                constexpr int j = decltype(index)::value;
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const u32x4 wf = expand<j>(words[r]);
#pragma unroll
                    for (int t = 0; t < TT; ++t) acc[r][t] = T::mfma(wf, xf[j][t], acc[r][t]);
                }
            },
            std::make_integer_sequence<int, 4>{});
    };
    auto read_x = [&](const char* stage, u32x4(&xf)[4][TT]) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int t = 0; t < TT; ++t) xf[j][t] = *(const u32x4*)(stage + (xbase ^ (32 * j)) + t * 4096);
    };
    if constexpr (ROW16) {
        for (int i = 0; i < D && i < count; ++i) issue(wave + i * WAVES, i);
        int slot = 0;
        for (int i = 0; i < count; ++i) {
            wait_groups<L::DPS>(count - 1 - i < D - 1 ? count - 1 - i : D - 1);
            const char* stage = ring + slot * L::STAGE;
            uint2 words[RB];
            u32x4 xf[4][TT];
#pragma unroll
            for (int r = 0; r < RB; ++r) words[r] = *(const uint2*)(stage + wbase + r * 512);
            read_x(stage, xf);
            wait_lgkm0();
            if (i + D < count) issue(wave + (i + D) * WAVES, slot);
            products(xf, words);
            slot = slot + 1 == D ? 0 : slot + 1;
        }
    } else {
        constexpr int AHEAD = 2;  // steps
        u32x4 next[AHEAD][TT * 4];
        uint2 ahead[AHEAD][RB];
        auto load = [&](auto set, int step) {
            constexpr int a = decltype(set)::value;
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                const int last = p.rb - 1 - n0 / 32;
                ahead[a][r] = *((const uint2*)p.w + ((int64_t)(n0 / 32 + (r < last ? r : last)) * nk + step) * 64 + lane);
            }
#pragma unroll
            for (int i = 0; i < TT * 4; ++i) {
                const int row = i * 8 + (lane >> 3), last = p.M - 1 - m0, k = step * 64 + ((lane & 7) ^ ((row >> 1) & 7)) * 8;
                next[a][i] = load_row8((const unsigned short*)p.x + (int64_t)(m0 + (row < last ? row : last)) * p.ldx, k, p.K);
            }
        };
        auto one = [&](auto set, int i) {
            constexpr int a = decltype(set)::value;
            if (i >= count) return;
            uint2 words[RB];
            u32x4 xf[4][TT];
#pragma unroll
            for (int r = 0; r < RB; ++r) words[r] = ahead[a][r];
#pragma unroll
            for (int f = 0; f < TT * 4; ++f) *(u32x4*)(ring + f * 1024 + lane * 16) = next[a][f];
            if (i + AHEAD < count) load(set, wave + (i + AHEAD) * WAVES);
            wait_lgkm0();
            read_x(ring, xf);
            products(xf, words);
        };
        const std::integral_constant<int, 0> even{};
        const std::integral_constant<int, 1> odd{};
        if (count > 0) load(even, wave);
        if (count > 1) load(odd, wave + WAVES);
        for (int i = 0; i < count; i += AHEAD) {
            one(even, i);
            one(odd, i + 1);
        }
        wait_lgkm0();
    }
    // (this wave's ring is its own, and all of it has been read)
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(float4*)(ring + (t * 32 + l32) * L::ZPITCH + (r * 32 + q * 8 + h * 4) * 4) =
                    make_float4(acc[r][t][4 * q], acc[r][t][4 * q + 1], acc[r][t][4 * q + 2], acc[r][t][4 * q + 3]);
    __syncthreads();
    constexpr int GROUPS = RB * 4, ITEMS = TT * 32 * GROUPS, PER = (ITEMS + WAVES * 64 - 1) / (WAVES * 64);
    float z[PER][8];
#pragma unroll
    for (int o = 0; o < PER; ++o) {
        const int item = tid + o * WAVES * 64, g = item % GROUPS, t = item / GROUPS, n = n0 + g * 8;
        if (item >= ITEMS) break;
        float al[8], bi[8], s[8];
        load_affine<T>(p, n, al, bi);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = 0.f;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) {
            const float* row = (const float*)(smem + v * L::WAVE + t * L::ZPITCH + g * 32);
            const float4 a = *(const float4*)row, b = *(const float4*)(row + 4);
            s[0] += a.x, s[1] += a.y, s[2] += a.z, s[3] += a.w, s[4] += b.x, s[5] += b.y, s[6] += b.z, s[7] += b.w;
        }
        const bool in = m0 + t < p.M;
#pragma unroll
        for (int i = 0; i < 8; ++i) z[o][i] = in ? fmaf(s[i], al[i], bi[i]) : 0.f;
        with_act(p.act, [&](auto which) { finish_row<T, decltype(which)::value>(p, m0 + t, n, z[o]); });
        if (p.zq)
#pragma unroll
            for (int i = 0; i < 8; ++i) atomicMax(&amax[(t >> 5) * (32 * RB) + g * 8 + i], __float_as_uint(z[o][i]) & 0x7fffffffu);
    }
    if (!p.zq) return;
    __syncthreads();
#pragma unroll
    for (int o = 0; o < PER; ++o) {
        const int item = tid + o * WAVES * 64, g = item % GROUPS, t = item / GROUPS, n = n0 + g * 8;
        if (item >= ITEMS) break;
        const int mt = m0 + (t & ~31);
        unsigned am[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) am[i] = amax[(t >> 5) * (32 * RB) + g * 8 + i];
        float zz[1][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) zz[0][i] = z[o][i];
        const CkptScale<T> scale(am);
        if (mt >= p.M || n >= p.N) continue;
        store_codes<T, 1>(p, mt, t & 31, n, zz, scale);
        if ((t & 31) == 0) store_scales(p, mt, n, scale);
    }
}

// Rows of whole 64-column steps from any rows: the columns past K are zeros.
__global__ __launch_bounds__(256) void k_copy_rows(const unsigned short* x, int64_t ldx, int64_t M, int64_t K, int64_t ld, unsigned short* out)
{
    const int64_t per = ld / 8, n = M * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / per, k = (i - m * per) * 8;
        *(u32x4*)(out + m * ld + k) = load_row8(x + m * ldx, k, K);
    }
}

template <class T, int BM, int BN, int NS>
hipError_t run_tile(LinParams& p, hipStream_t st)
{
    using L = LinTile<BM, BN, NS>;
    p.tilesM = (p.M + BM - 1) / BM;
    const int tilesN = (p.N + BN - 1) / BN;
    const int64_t nt = (int64_t)p.tilesM * tilesN;
    if (nt > 0x7fffff00) return hipErrorInvalidValue;
    p.ntiles = (int)nt;
    p.band_tiles = 8 * tilesN;
    p.div_band = make_fastdiv((uint32_t)p.band_tiles);
    p.div_lastband = make_fastdiv((uint32_t)(p.tilesM % 8 ? p.tilesM % 8 : 8));
    static LdsLimit limit;
    const hipError_t e = limit.raise((const void*)&k_linear<T, BM, BN, NS>, L::LDS);
    if (e != hipSuccess) return e;
    k_linear<T, BM, BN, NS><<<(unsigned)((nt + 7) / 8 * 8), 256, L::LDS, st>>>(p);
    return hipGetLastError();
}

bool rows_of_16(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }
// Whether a tile's rows can be loaded straight into LDS: whole 16-byte units within the 32-bit offsets of up to 128 rows.
bool direct_rows(const void* x, int64_t ldx, int64_t K) { return rows_of_16(x, ldx) && K % 8 == 0 && 128 * ldx * 2 + K * 2 < (int64_t)kOutside; }

template <class T, int RB, int WAVES, int BATCH>
hipError_t run_few(const LinParams& p, hipStream_t st)
{
    const unsigned grid = (unsigned)((p.N + 16 * RB - 1) / (16 * RB));
    if (p.K % 8 == 0 && rows_of_16(p.x, p.ldx) && (p.M * p.ldx + p.K) * 2 < (int64_t)kOutside)
        k_linear_few<T, RB, WAVES, BATCH, true><<<grid, WAVES * 64, 0, st>>>(p);
    else
        k_linear_few<T, RB, WAVES, BATCH, false><<<grid, WAVES * 64, 0, st>>>(p);
    return hipGetLastError();
}

template <class T, int TT, int RB, int WAVES, int D, bool ROW16>
hipError_t run_split_rows(LinParams& p, hipStream_t st)
{
    using L = SplitTile<TT, RB, WAVES, D>;
    static_assert(L::LDS <= 160 * 1024, "");
    p.tilesM = (p.M + 32 * TT - 1) / (32 * TT);
    const int64_t nt = (int64_t)p.tilesM * ((p.N + 32 * RB - 1) / (32 * RB));
    if (nt > 0x7fffff00) return hipErrorInvalidValue;
    static LdsLimit limit;
    const hipError_t e = limit.raise((const void*)&k_linear_split<T, TT, RB, WAVES, D, ROW16>, L::LDS);
    if (e != hipSuccess) return e;
    k_linear_split<T, TT, RB, WAVES, D, ROW16><<<(unsigned)nt, WAVES * 64, L::LDS, st>>>(p);
    return hipGetLastError();
}

template <class T, int TT, int RB, int WAVES, int D>
hipError_t run_split(LinParams& p, hipStream_t st)
{
    return direct_rows(p.x, p.ldx, p.K) ? run_split_rows<T, TT, RB, WAVES, D, true>(p, st) : run_split_rows<T, TT, RB, WAVES, D, false>(p, st);
}

template <class T>
hipError_t run(const LinearArgs& a, LinParams p, hipStream_t st)
{
    const LinearForm form = linear_form(a.M, a.N, a.K, a.zq != nullptr);
    if (form == LinearForm::kFew) return a.N > kFewOutputs ? run_few<T, 2, 16, 2>(p, st) : run_few<T, 1, 16, 2>(p, st);
    if (linear_copies_x(a)) {
        const int64_t ld = (a.K + 63) / 64 * 64, blocks = (a.M * ld / 8 + 255) / 256;
        k_copy_rows<<<(unsigned)(blocks < 8192 ? blocks : 8192), 256, 0, st>>>((const unsigned short*)a.x, a.ldx, a.M, a.K, ld, (unsigned short*)a.workspace);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        p.x = (const int8_t*)a.workspace;
        p.ldx = ld;
        p.K = (int)ld;
    }
    switch (form) {
        case LinearForm::kSplit32: return run_split<T, 1, 1, 8, 2>(p, st);
        case LinearForm::kSplit32x64: return run_split<T, 1, 2, 8, 2>(p, st);
        case LinearForm::kSplit64: return run_split<T, 2, 2, 8, 2>(p, st);
        case LinearForm::kTile128: return run_tile<T, 128, 128, 4>(p, st);
        default: return run_tile<T, 128, 256, 4>(p, st);
    }
}

}  // namespace

bool linear_copies_x(const LinearArgs& a)
{
    const LinearForm form = linear_form(a.M, a.N, a.K, a.zq != nullptr);
    if (form == LinearForm::kFew || direct_rows(a.x, a.ldx, a.K)) return false;
    // The split forms take any rows, but over many steps that costs more than a copy.  us, without and with one: 216 x 6016 x 7223
    // 62 and 41, 1000 x 1003 x 2187 13.7 and 15.5.
    return form == LinearForm::kTile128 || form == LinearForm::kTile256 || a.K > 4096;
}

hipError_t launch_linear(const LinearArgs& a, hipStream_t st)
{
    LinParams p = {};
    p.x = (const int8_t*)a.x, p.w = (const int8_t*)a.w;
    p.M = (int)a.M, p.N = (int)a.N, p.K = (int)a.K;
    p.ldx = a.ldx, p.ldr = a.ldr, p.ldy = a.ldy;
    const WeightShape ws(a.N, a.K);
    p.nk = (int)ws.cb, p.rb = (int)ws.rb;
    p.alpha = a.alpha, p.unit = a.unit;
    p.bias = (const unsigned short*)a.bias, p.res = (const unsigned short*)a.res;
    p.y = (unsigned short*)a.y;
    p.zq = a.zq;
    p.act = a.act;
    return a.f16 ? run<F16>(a, p, st) : run<BF16>(a, p, st);
}

}  // namespace rtn
