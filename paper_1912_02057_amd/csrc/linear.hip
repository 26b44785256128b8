// Ternary linear layer of 16-bit activations: y = act(alpha (x t^T) + bias) + residual, on the bf16 / fp16 matrix cores.
//
// The weights are two bits each in the order the matrix instruction takes them (WeightShape); a register of two weights is
// a shift and an AND away from its word (-2, 0, +2; the halves are made up for in alpha), so 32 operand registers of a
// 64-step cost 64 vector operations beside 64 matrix instructions of 32 cycles.
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
    const unsigned short *bias, *res;
    unsigned short* y;
    int8_t* zq;
    int act;
    int vec_y, vec_r;       // rows of y / residual can be accessed 16 bytes at a time
};

// The parameters of 8 consecutive outputs (0 past the end).
template <class T>
__device__ __forceinline__ void load_affine(const LinParams& p, int n, float (&al)[8], float (&bi)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool in = n + i < p.N;
        al[i] = in ? 0.5f * (p.alpha.ptr ? p.alpha.ptr[n + i] : p.alpha.s) : 0.f;
        bi[i] = in && p.bias ? T::to_float(p.bias[n + i]) : 0.f;
    }
}

// act(z) + residual of row m, outputs n .. n + 7 -> y
template <class T, int ACT>
__device__ __forceinline__ void finish_row(const LinParams& p, int m, int n, const float (&z)[8])
{
    if (m >= p.M || n >= p.N) return;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = act_value<ACT>(z[i]);
    const bool whole = n + 8 <= p.N;
    if (p.res) {
        const unsigned short* r = p.res + m * p.ldr + n;
        if (p.vec_r && whole) {
            const u32x4 q = *(const u32x4*)r;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += half_of<T>(q[i >> 1], i & 1);
        } else {
            for (int i = 0; i < 8; ++i)
                if (n + i < p.N) v[i] += T::to_float(r[i]);
        }
    }
    unsigned short* y = p.y + m * p.ldy + n;
    if (p.vec_y && whole) {
        *(u32x4*)y = u32x4{pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7])};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (n + i < p.N) y[i] = T::from_float(v[i]);
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
    static constexpr int WM = BM / 2, WN = BN / 2, TM = WM / 32, TN = WN / 32, NM = TM * TN;
    static constexpr int ABYTES = BM * 128, STAGE = ABYTES + BN * 16, DPS = BM / 32 + 1;
    static constexpr int ZPITCH = WN * 4 + 16, ZBYTES = 32 * ZPITCH;  // a wave's 32 rows of fp32 in the epilogue
    static constexpr int LDS = NS * STAGE > 4 * ZBYTES ? NS * STAGE : 4 * ZBYTES;
};

// A block of 4 waves (2 x 2) owns BM tokens x BN outputs.  Ring of NS stages of 64 columns: x rows of 128 bytes, 16-byte
// chunk c of row r at place c ^ (r >> 1 & 7), so that 16 rows' fragments hit all banks; then the weights' words.  One barrier per
// step, before the last of its four 16-column slices, and fragments are read one slice ahead.
template <class T, int BM, int BN, int NS>
__global__ __launch_bounds__(256, BM * BN >= 256 * 256 ? 1 : 2) void k_linear(LinParams p)
{
    using L = LinTile<BM, BN, NS>;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1, l32 = lane & 31, h = lane >> 5;

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
    unsigned xoff[BM / 32];
#pragma unroll
    for (int i = 0; i < BM / 32; ++i) {
        const int row = (wave * (BM / 32) + i) * 8 + (lane >> 3), last = p.M - 1 - m0;
        xoff[i] = (unsigned)(row < last ? row : last) * (unsigned)(p.ldx * 2) + (unsigned)(((lane & 7) ^ ((row >> 1) & 7)) * 16);
    }
    unsigned woff;
    {
        const int at = wave * BN * 4 + lane * 16, last = p.rb - 1 - n0 / 32, r = at >> 9;
        woff = (unsigned)(r < last ? r : last) * (unsigned)(nk * 512) + (unsigned)(at & 511);
    }
    const int ktail = p.K & 63;
    auto issue = [&](int step, int slot) {
        const unsigned base = lds0 + (unsigned)(slot * L::STAGE), k2 = (unsigned)step * 128u;
        const bool tail = ktail && step == nk - 1;
        for_each_index(
            [&](auto index) {
                constexpr int i = decltype(index)::value;
                unsigned v = xoff[i];
                if (tail) {  // chunks past the row's end are zeros
                    const int row = (wave * (BM / 32) + i) * 8 + (lane >> 3);
                    if (((lane & 7) ^ ((row >> 1) & 7)) * 8 >= ktail) v = kOutside;
                }
                dma_buf<i * 1024, true>(xr, v, k2, base + (unsigned)(wave * (BM / 32) * 1024));
            },
            std::make_integer_sequence<int, BM / 32>{});
        if (lane < BN / 4) dma_buf<L::ABYTES, true>(wr, woff, (unsigned)step * 512u, base + (unsigned)(wave * BN * 4));
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
    const int xbase = (wm * L::WM + l32) * 128 + ((h ^ ((l32 >> 1) & 7)) * 16), wbase = L::ABYTES + wn * L::TN * 512 + lane * 8;

    int issued = 0;
    for (; issued < NS - 1 && issued < nk; ++issued) issue(issued, issued);
    wait_groups<L::DPS>(issued - 1);
    block_barrier();
    int slot = 0;  // of the current step
#pragma unroll
    for (int i = 0; i < L::TN; ++i) words[i] = *(const uint2*)(smem + wbase + i * 512);
#pragma unroll
    for (int i = 0; i < L::TM; ++i) xf[0][i] = *(const u32x4*)(smem + xbase + i * 4096);
#pragma unroll
    for (int i = 0; i < L::TN; ++i) wf[0][i] = expand<0>(words[i]);

    for (int step = 0; step < nk; ++step) {
        int next = slot + 1 == NS ? 0 : slot + 1;
        auto slice = [&](auto index) {
            constexpr int j = decltype(index)::value, cur = j & 1, nxt = cur ^ 1;
            if constexpr (j == 3) {
                // step + 1 has landed for this wave, then for all; and all are done with step - 1, whose slot is filled again
                const int later = nk - 2 - step;
                wait_groups<L::DPS>(later < NS - 3 ? later : NS - 3);
                block_barrier();
                if (issued < nk) {
                    issue(issued, slot == 0 ? NS - 1 : slot - 1);
                    ++issued;
                }
            }
            const char* stage = smem + (j == 3 ? next : slot) * L::STAGE;
            uint2 ahead[L::TN];
            if constexpr (j == 3) {
#pragma unroll
                for (int i = 0; i < L::TN; ++i) ahead[i] = *(const uint2*)(stage + wbase + i * 512);
            }
#pragma unroll
            for (int i = 0; i < L::TM; ++i) xf[nxt][i] = *(const u32x4*)(stage + (xbase ^ (32 * ((j + 1) & 3))) + i * 4096);
            __builtin_amdgcn_sched_barrier(0);
            for_each_index(
                [&](auto mi) {
                    constexpr int n = decltype(mi)::value, i = n / L::TM, k = n % L::TM;
                    acc[i][k] = T::mfma(wf[cur][i], xf[cur][k], acc[i][k]);
                    // the next slice's weights, in the second half of this one's products
                    constexpr int first = L::NM / 2, per = (L::NM - first) / L::TN > 0 ? (L::NM - first) / L::TN : 1;
                    if constexpr (n >= first && (n - first) % per == 0 && (n - first) / per < L::TN) {
                        constexpr int e = (n - first) / per;
                        wf[nxt][e] = expand<(j + 1) & 3>(j == 3 ? ahead[e] : words[e]);
                    }
                    if constexpr (L::NM > 2) __builtin_amdgcn_sched_barrier(0);
                },
                std::make_integer_sequence<int, L::NM>{});
            if constexpr (L::NM / 2 + L::TN > L::NM) {
#pragma unroll
                for (int e = 0; e < L::TN; ++e) wf[nxt][e] = expand<(j + 1) & 3>(j == 3 ? ahead[e] : words[e]);
            }
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
    }

    // ---- epilogue: 32 tokens of the wave's tile at a time through LDS, after which a lane has 8 outputs of TPL tokens
    __syncthreads();
    constexpr int CL = L::WN / 8, TPL = CL / 2;
    char* zs = smem + wave * L::ZBYTES;
    const int n8 = n0 + wn * L::WN + (lane % CL) * 8, t0 = (lane / CL) * TPL;
    float al[8], bi[8];
    load_affine<T>(p, n8, al, bi);
#pragma unroll 1
    for (int k = 0; k < L::TM; ++k) {
        auto put = [&](auto index) {
            constexpr int kk = decltype(index)::value;
            if (kk != k) return;
#pragma unroll
            for (int i = 0; i < L::TN; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(float4*)(zs + l32 * L::ZPITCH + (i * 32 + q * 8 + h * 4) * 4) =
                        make_float4(acc[i][kk][4 * q], acc[i][kk][4 * q + 1], acc[i][kk][4 * q + 2], acc[i][kk][4 * q + 3]);
        };
        for_each_index(put, std::make_integer_sequence<int, L::TM>{});
        const int mt = m0 + wm * L::WM + k * 32;  // first token
        float z[TPL][8];
        wait_lgkm0();
#pragma unroll
        for (int t = 0; t < TPL; ++t) {
            const float* row = (const float*)(zs + (t0 + t) * L::ZPITCH + (lane % CL) * 32);
            const float4 a = *(const float4*)row, b = *(const float4*)(row + 4);
            const float s[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) z[t][i] = fmaf(s[i], al[i], bi[i]);
        }
        if (mt >= p.M || n0 + wn * L::WN >= p.N) continue;
        if (p.zq) {
            const CkptShape cs(p.M, p.N);
            unsigned am[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                am[i] = 0;
#pragma unroll
                for (int t = 0; t < TPL; ++t) {
                    const unsigned u = mt + t0 + t < p.M ? __float_as_uint(z[t][i]) & 0x7fffffffu : 0u;
                    am[i] = u > am[i] ? u : am[i];
                }
#pragma unroll
                for (int d = CL; d < 64; d *= 2) {
                    const unsigned o = (unsigned)__shfl_xor((int)am[i], d);
                    am[i] = o > am[i] ? o : am[i];
                }
            }
            unsigned char ex[8];
            float inv[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = ckpt_exponent<T>(__uint_as_float(am[i]));
                ex[i] = (unsigned char)e;
                inv[i] = ckpt_inverse(e);
            }
            if (n8 < p.N) {
                const int64_t blk = (int64_t)(mt >> 5) * cs.cb + (n8 >> 3);
                int8_t* out = p.zq + blk * 256 + t0 * 8;
#pragma unroll
                for (int t = 0; t < TPL; ++t) {
                    unsigned w[2] = {0, 0};
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const unsigned q = mt + t0 + t < p.M ? ckpt_code(z[t][i], inv[i]) : 0u;
                        w[i >> 2] |= q << (8 * (i & 3));
                    }
                    *(uint2*)(out + t * 8) = make_uint2(w[0], w[1]);
                }
                if (t0 == 0) {
                    uint2 e2;
                    e2.x = ex[0] | ex[1] << 8 | ex[2] << 16 | (unsigned)ex[3] << 24;
                    e2.y = ex[4] | ex[5] << 8 | ex[6] << 16 | (unsigned)ex[7] << 24;
                    *(uint2*)(p.zq + cs.codes() + blk * 8) = e2;
                }
            }
        }
        auto rows = [&](auto which) {
#pragma unroll
            for (int t = 0; t < TPL; ++t) finish_row<T, decltype(which)::value>(p, mt + t0 + t, n8, z[t]);
        };
        if (p.act == kActNone)
            rows(std::integral_constant<int, kActNone>{});
        else if (p.act == kActRelu)
            rows(std::integral_constant<int, kActRelu>{});
        else if (p.act == kActGelu)
            rows(std::integral_constant<int, kActGelu>{});
        else
            rows(std::integral_constant<int, kActSilu>{});
        // (the next round's writes to `zs` are this wave's own and come after its reads)
    }
}

// Few tokens (at most 32 TT): a block has 32 outputs, its waves share the columns, the weights are read once and straight into
// registers.  Bound by the weights' bytes and, for small layers, by the latency of one load after the launch.
template <class T, int TT, int WAVES, bool VEC>
__global__ __launch_bounds__(WAVES * 64) void k_linear_few(LinParams p)
{
    __shared__ float part[WAVES][TT][32][33];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, h = lane >> 5;
    const int rb = blockIdx.x, n0 = rb * 32;
    f32x16 acc[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][r] = 0.f;
    const uint2* w = (const uint2*)p.w + (int64_t)rb * p.nk * 64 + lane;
    const unsigned short* xrow[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) xrow[t] = (const unsigned short*)p.x + (int64_t)(t * 32 + l32) * p.ldx;
    for (int step = wave; step < p.nk; step += WAVES) {
        const uint2 word = w[(int64_t)step * 64];
        auto slice = [&](auto index) {
            constexpr int j = decltype(index)::value;
            const int k = step * 64 + 16 * j + 8 * h;
            const u32x4 wf = expand<j>(word);
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                u32x4 xf = {0, 0, 0, 0};
                if (t * 32 + l32 < p.M) {
                    if constexpr (VEC) {
                        if (k < p.K) xf = *(const u32x4*)(xrow[t] + k);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (k + i < p.K) xf[i >> 1] |= (unsigned)xrow[t][k + i] << (16 * (i & 1));
                    }
                }
                acc[t] = T::mfma(wf, xf, acc[t]);
            }
        };
        slice(std::integral_constant<int, 0>{});
        slice(std::integral_constant<int, 1>{});
        slice(std::integral_constant<int, 2>{});
        slice(std::integral_constant<int, 3>{});
    }
#pragma unroll
    for (int t = 0; t < TT; ++t)
        if (t * 32 + l32 < p.M)
#pragma unroll
            for (int r = 0; r < 16; ++r) part[wave][t][l32][8 * (r >> 2) + 4 * h + (r & 3)] = acc[t][r];
    __syncthreads();
    for (int o = tid; o < p.M * 4; o += WAVES * 64) {  // 8 outputs of a token each
        const int m = o >> 2, c = (o & 3) * 8, n = n0 + c;
        float al[8], bi[8], z[8];
        load_affine<T>(p, n, al, bi);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < WAVES; ++v) s += part[v][m >> 5][m & 31][c + i];
            z[i] = fmaf(s, al[i], bi[i]);
        }
        if (p.act == kActNone)
            finish_row<T, kActNone>(p, m, n, z);
        else if (p.act == kActRelu)
            finish_row<T, kActRelu>(p, m, n, z);
        else if (p.act == kActGelu)
            finish_row<T, kActGelu>(p, m, n, z);
        else
            finish_row<T, kActSilu>(p, m, n, z);
    }
}

// Rows of whole 64-column steps from any rows: the columns past K are zeros.
__global__ __launch_bounds__(256) void k_copy_rows(const unsigned short* x, int64_t ldx, int64_t M, int64_t K, int64_t ld, unsigned short* out)
{
    const int64_t per = ld / 8, n = M * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / per, k = (i - m * per) * 8;
        const unsigned short* r = x + m * ldx + k;
        u32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (k + j < K) v[j >> 1] |= (unsigned)r[j] << (16 * (j & 1));
        *(u32x4*)(out + m * ld + k) = v;
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

template <class T, int TT, int WAVES>
hipError_t run_few(const LinParams& p, bool vec, hipStream_t st)
{
    const unsigned grid = (unsigned)((p.N + 31) / 32);
    if (vec)
        k_linear_few<T, TT, WAVES, true><<<grid, WAVES * 64, 0, st>>>(p);
    else
        k_linear_few<T, TT, WAVES, false><<<grid, WAVES * 64, 0, st>>>(p);
    return hipGetLastError();
}

bool rows_of_16(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

template <class T>
hipError_t run(const LinearArgs& a, LinParams p, hipStream_t st)
{
    const bool vec = rows_of_16(a.x, a.ldx) && a.K % 8 == 0;
    if (a.M <= kFewTokens && !a.zq) return p.nk >= 16 ? run_few<T, 1, 16>(p, vec, st) : run_few<T, 1, 4>(p, vec, st);
    if (linear_copies_x(a)) {
        const int64_t ld = (a.K + 63) / 64 * 64, blocks = (a.M * ld / 8 + 255) / 256;
        k_copy_rows<<<(unsigned)(blocks < 8192 ? blocks : 8192), 256, 0, st>>>((const unsigned short*)a.x, a.ldx, a.M, a.K, ld, (unsigned short*)a.workspace);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        p.x = (const int8_t*)a.workspace;
        p.ldx = ld;
        p.K = (int)ld;
    }
    const int64_t t256 = ((a.M + 255) / 256) * ((a.N + 255) / 256), t128 = ((a.M + 127) / 128) * ((a.N + 127) / 128);
    if (t256 >= 192) return run_tile<T, 256, 256, 4>(p, st);
    if (t128 >= 192) return run_tile<T, 128, 128, 4>(p, st);
    return run_tile<T, 64, 64, 4>(p, st);
}

}  // namespace

bool linear_copies_x(const LinearArgs& a)
{
    if (a.M <= kFewTokens && !a.zq) return false;
    return !rows_of_16(a.x, a.ldx) || a.K % 8 != 0 || 256 * a.ldx * 2 + a.K * 2 >= (int64_t)kOutside;
}

hipError_t launch_linear(const LinearArgs& a, hipStream_t st)
{
    LinParams p = {};
    p.x = (const int8_t*)a.x, p.w = (const int8_t*)a.w;
    p.M = (int)a.M, p.N = (int)a.N, p.K = (int)a.K;
    p.ldx = a.ldx, p.ldr = a.ldr, p.ldy = a.ldy;
    const WeightShape ws(a.N, a.K);
    p.nk = (int)ws.cb, p.rb = (int)ws.rb;
    p.alpha = a.alpha;
    p.bias = (const unsigned short*)a.bias, p.res = (const unsigned short*)a.res;
    p.y = (unsigned short*)a.y;
    p.zq = a.zq;
    p.act = a.act;
    p.vec_y = rows_of_16(a.y, a.ldy), p.vec_r = rows_of_16(a.res, a.ldr);
    return a.f16 ? run<F16>(a, p, st) : run<BF16>(a, p, st);
}

}  // namespace rtn
