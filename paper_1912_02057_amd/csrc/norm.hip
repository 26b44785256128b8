// Norms before and after a block of a language model, with the block's gate and residual scale, and their gradients:
//   y = scale x + gate (n(h) weight + bias)      u = n(y) next_weight + next_bias
// either line alone or both in one pass.  n is x / sqrt(mean x^2 + eps) or (x - mean) / sqrt(var + eps) of a row.
//
// All of them are one pass over memory: a row stays in the registers of W waves (PER pieces of 8 columns a lane) from its load to its
// stores, and statistics are sums over those registers, the variance of the centred values, in fp32.  A unit (W waves) walks
// consecutive rows, so that the vectors of the columns are read once.
#include "mx4_math.h"
#include "rtn_kernels.h"

namespace rtn {

namespace {

template <int W>
struct Unit {
    static constexpr int kRows = W == 1 ? 4 : 1, kThreads = W == 1 ? 256 : W * 64;  // units of a block
    static __device__ __forceinline__ int64_t index() { return W == 1 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : (int64_t)blockIdx.x; }
    static __device__ __forceinline__ int lane() { return W == 1 ? threadIdx.x & 63 : threadIdx.x; }
};

// Sums over a unit, in all its lanes.  `turn` alternates between two sets of LDS words, so that one barrier a sum is enough.
template <int W, int N>
__device__ __forceinline__ void unit_sums(float (&v)[N], float (*lds)[W][2], int& turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int d = 1; d < 64; d *= 2) v[i] += __shfl_xor(v[i], d);
    if constexpr (W > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) lds[turn][wave][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) v[i] += lds[turn][w][i];
        }
        turn ^= 1;
    }
}

template <int PER>
struct Cols {
    float v[PER][8];
};
template <int W, int PER>
struct Row {
    u32x4 q[PER];
    __device__ __forceinline__ void load(const void* base, int64_t ld, int64_t m, int64_t C)
    {
#pragma unroll
        for (int j = 0; j < PER; ++j) q[j] = load_row8((const unsigned short*)base + m * ld, (int64_t)(j * W * 64 + Unit<W>::lane()) * 8, C);
    }
    template <class T>
    __device__ __forceinline__ float get(int j, int i) const
    {
        return half_of<T>(q[j][i >> 1], i & 1);
    }
};
template <int W, int PER>
__device__ __forceinline__ void load_cols(Cols<PER>& c, const float* p, int64_t C, float otherwise)
{
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int64_t k = (int64_t)(j * W * 64 + Unit<W>::lane()) * 8;
        if (p) {
            load_values<F32>(p, k, C, c.v[j]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) c.v[j][i] = otherwise;
        }
    }
}
// (rounded and returned as rounded)
template <class T, int W, int PER>
__device__ __forceinline__ void store_row(void* base, int64_t ld, int64_t m, int64_t C, Cols<PER>& v)
{
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int64_t k = (int64_t)(j * W * 64 + Unit<W>::lane()) * 8;
        unsigned short* y = (unsigned short*)base + m * ld + k;
        const u32x4 q = {pack2<T>(v.v[j][0], v.v[j][1]), pack2<T>(v.v[j][2], v.v[j][3]), pack2<T>(v.v[j][4], v.v[j][5]), pack2<T>(v.v[j][6], v.v[j][7])};
#pragma unroll
        for (int i = 0; i < 8; ++i) v.v[j][i] = half_of<T>(q[i >> 1], i & 1);
        if (k + 8 <= C) {
            store16(y, q);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < C) y[i] = (unsigned short)(i & 1 ? q[i >> 1] >> 16 : q[i >> 1] & 0xffffu);
        }
    }
}
template <int W>
__device__ __forceinline__ bool inside(int j, int i, int64_t C) { return (int64_t)(j * W * 64 + Unit<W>::lane()) * 8 + i < C; }

// v -> n(v), and 1 / sqrt(..).  A mean in fp32 is off by its sum's roundings, which a row of small variance divides by a small number: what is
// left of it in the centred values is summed with their squares and taken off too.
template <int W, int PER>
__device__ __forceinline__ float normalise(Cols<PER>& v, int64_t C, int layer, float eps, float (*lds)[W][2], int& turn)
{
    const float n = (float)C;
    float rest = 0.f, var;
    auto for_each = [&](auto f) {
#pragma unroll
        for (int j = 0; j < PER; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) f(j, i, v.v[j][i]);
    };
    if (layer) {
        float t[1] = {0.f};
        for_each([&](int, int, float x) { t[0] += x; });
        unit_sums<W, 1>(t, lds, turn);
        const float mean = t[0] / n;
        for_each([&](int j, int i, float& x) { x = inside<W>(j, i, C) ? x - mean : 0.f; });
        float s[2] = {0.f, 0.f};
        for_each([&](int, int, float x) { s[0] = fmaf(x, x, s[0]), s[1] += x; });
        unit_sums<W, 2>(s, lds, turn);
        rest = s[1] / n;
        var = fmaf(-rest, rest, s[0] / n);
        var = var < 0.f ? 0.f : var;  // (a NaN stays one)
    } else {
        float q[1] = {0.f};
        for_each([&](int, int, float x) { q[0] = fmaf(x, x, q[0]); });
        unit_sums<W, 1>(q, lds, turn);
        var = q[0] / n;
    }
    const float r = 1.f / sqrtf(var + eps);
    for_each([&](int j, int i, float& x) { x = (x - rest) * r; });
    return r;
}
// dn, the gradient of n(v) -> that of v:  r (dn - n mean(dn n) [- mean(dn)])
template <int W, int PER>
__device__ __forceinline__ void normalise_back(Cols<PER>& dn, const Cols<PER>& n, float r, int64_t C, int layer, float (*lds)[W][2], int& turn)
{
    const float inv = 1.f / (float)C;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[0] = fmaf(dn.v[j][i], n.v[j][i], s[0]);
            s[1] += dn.v[j][i];
        }
    unit_sums<W, 2>(s, lds, turn);
    const float a = s[0] * inv, b = layer ? s[1] * inv : 0.f;
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) dn.v[j][i] = r * (dn.v[j][i] - fmaf(n.v[j][i], a, b));
}

// POST: y = scale x + gate (n(h) weight + bias); without it y is x.  PRE: u = n(y) next_weight + next_bias.
template <class T, bool POST, bool PRE, int W, int PER>
__global__ __launch_bounds__(Unit<W>::kThreads) void k_norm(NormArgs a)
{
    __shared__ float lds[2][W][2];
    int turn = 0;
    const int64_t first = Unit<W>::index() * a.rows, end = first + a.rows < a.M ? first + a.rows : a.M;
    if (first >= end) return;
    Cols<PER> w, b, gate, nw, nb;
    if constexpr (POST) load_cols<W>(w, a.weight, a.C, 1.f), load_cols<W>(b, a.bias, a.C, 0.f);
    if constexpr (PRE) load_cols<W>(nw, a.next_weight, a.C, 1.f), load_cols<W>(nb, a.next_bias, a.C, 0.f);
    int64_t owner = -1;
    for (int64_t m = first; m < end; ++m) {
        Row<W, PER> x, h;
        x.load(a.x, a.ldx, m, a.C);
        Cols<PER> v;
        if constexpr (POST) {
            h.load(a.h, a.ldh, m, a.C);
            if (m / a.run != owner) {
                owner = m / a.run;
                load_cols<W>(gate, a.gate ? a.gate + owner * a.C : nullptr, a.C, 1.f);
            }
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) v.v[j][i] = h.template get<T>(j, i);
            normalise<W, PER>(v, a.C, a.layer, a.eps, lds, turn);
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) v.v[j][i] = fmaf(gate.v[j][i], fmaf(v.v[j][i], w.v[j][i], b.v[j][i]), a.scale * x.template get<T>(j, i));
            store_row<T, W, PER>(a.y, a.ldy, m, a.C, v);
        } else {
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) v.v[j][i] = x.template get<T>(j, i);
        }
        if constexpr (PRE) {
            if constexpr (POST) {  // (past the end of the row)
#pragma unroll
                for (int j = 0; j < PER; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v.v[j][i] = inside<W>(j, i, a.C) ? v.v[j][i] : 0.f;
            }
            normalise<W, PER>(v, a.C, a.layer, a.eps, lds, turn);
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) v.v[j][i] = fmaf(v.v[j][i], nw.v[j][i], nb.v[j][i]);
            store_row<T, W, PER>(a.u, a.ldu, m, a.C, v);
        }
    }
}

// With d the gradient of y, du's part among it:
//   dx = scale d,  dh = n'(h) (d gate weight),  and per unit, for k_norm_sums: sum d n(h), sum d, sum du n(y), sum du
// A unit's rows share a row of the gate.
template <class T, bool POST, bool PRE, int W, int PER>
__global__ __launch_bounds__(Unit<W>::kThreads) void k_norm_back(NormBackArgs a)
{
    __shared__ float lds[2][W][2];
    int turn = 0;
    const int64_t unit = Unit<W>::index();
    if (unit >= a.owners * a.parts) return;
    const int64_t owner = unit / a.parts, from = (unit - owner * a.parts) * a.rows;
    const int64_t run_end = (owner + 1) * a.run < a.M ? (owner + 1) * a.run : a.M;
    const int64_t first = owner * a.run + from, end = first + a.rows < run_end ? first + a.rows : run_end;
    Cols<PER> gw, nw, sums[4];
    if constexpr (POST) {
        Cols<PER> gate;
        load_cols<W>(gw, a.weight, a.C, 1.f);
        load_cols<W>(gate, a.gate ? a.gate + owner * a.C : nullptr, a.C, 1.f);
#pragma unroll
        for (int j = 0; j < PER; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) gw.v[j][i] *= gate.v[j][i];
    }
    if constexpr (PRE) load_cols<W>(nw, a.next_weight, a.C, 1.f);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < PER; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[k].v[j][i] = 0.f;
    for (int64_t m = first; m < end; ++m) {
        Row<W, PER> dy, du, h, y;
        if (a.dy) dy.load(a.dy, a.lddy, m, a.C);
        if constexpr (PRE) du.load(a.du, a.lddu, m, a.C), y.load(a.y, a.ldy, m, a.C);
        if constexpr (POST) h.load(a.h, a.ldh, m, a.C);
        Cols<PER> d;
#pragma unroll
        for (int j = 0; j < PER; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) d.v[j][i] = a.dy ? dy.template get<T>(j, i) : 0.f;
        if constexpr (PRE) {
            Cols<PER> n, t;
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) n.v[j][i] = y.template get<T>(j, i);
            const float r = normalise<W, PER>(n, a.C, a.layer, a.eps, lds, turn);
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float g = du.template get<T>(j, i);
                    sums[2].v[j][i] = fmaf(g, n.v[j][i], sums[2].v[j][i]);
                    sums[3].v[j][i] += g;
                    t.v[j][i] = g * nw.v[j][i];
                }
            normalise_back<W, PER>(t, n, r, a.C, a.layer, lds, turn);
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) d.v[j][i] += t.v[j][i];
        }
        if (a.dx) {
            Cols<PER> v;
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) v.v[j][i] = a.scale * d.v[j][i];
            store_row<T, W, PER>(a.dx, a.lddx, m, a.C, v);
        }
        if constexpr (POST) {
            Cols<PER> n;
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) n.v[j][i] = h.template get<T>(j, i);
            const float r = normalise<W, PER>(n, a.C, a.layer, a.eps, lds, turn);
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sums[0].v[j][i] = fmaf(d.v[j][i], n.v[j][i], sums[0].v[j][i]);
                    sums[1].v[j][i] += d.v[j][i];
                    d.v[j][i] = inside<W>(j, i, a.C) ? d.v[j][i] * gw.v[j][i] : 0.f;
                }
            if (a.dh) {
                normalise_back<W, PER>(d, n, r, a.C, a.layer, lds, turn);
                store_row<T, W, PER>(a.dh, a.lddh, m, a.C, d);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (a.part[k])
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (inside<W>(j, i, a.C)) a.part[k][unit * a.C + (int64_t)(j * W * 64 + Unit<W>::lane()) * 8 + i] = sums[k].v[j][i];
}

// The units' sums into the gradients of the vectors, in one order: 64 columns a block, its 16 waves share the units of one owner (a row of the
// gate), and blockIdx.y owners out of a.owners.  With S, T the first two sums over an owner's units:
//   dgate = S weight + T bias,  dweight += gate S,  dbias += gate T
// Several blocks of owners leave partial sums for a second launch.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(1024) void k_norm_sums(NormSumArgs a)
{
    __shared__ float lds[kSumWaves][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane, per = (a.owners + gridDim.y - 1) / gridDim.y;
    const int64_t o0 = blockIdx.y * per, o1 = o0 + per < a.owners ? o0 + per : a.owners;
    const bool in = c < a.C;
    float total[4] = {0.f, 0.f, 0.f, 0.f};
    const float w = in && a.weight ? a.weight[c] : 1.f, b = in && a.bias ? a.bias[c] : 0.f;
    for (int64_t o = o0; o < o1; ++o) {
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        if (in)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (a.part[k])
                    for (int64_t u = wave; u < a.parts; u += kSumWaves) s[k] += a.part[k][(o * a.parts + u) * a.C + c];
#pragma unroll
        for (int k = 0; k < 4; ++k) lds[wave][k][lane] = s[k];
        __syncthreads();
        if (wave == 0 && in) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                s[k] = 0.f;
                for (int v = 0; v < kSumWaves; ++v) s[k] += lds[v][k][lane];
            }
            const float g = a.gate ? a.gate[o * a.C + c] : 1.f;
            if (a.dgate) a.dgate[o * a.C + c] = fmaf(s[0], w, s[1] * b);
            total[0] = fmaf(g, s[0], total[0]), total[1] = fmaf(g, s[1], total[1]);
            total[2] += s[2], total[3] += s[3];
        }
        __syncthreads();
    }
    if (wave == 0 && in) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (a.out[k]) a.out[k][(int64_t)blockIdx.y * a.C + c] = total[k];
    }
}

// W waves of PER pieces for rows of C columns
template <class F>
hipError_t with_shape(int64_t C, F&& f)
{
    if (C <= 512) return f(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{});
    if (C <= 2048) return f(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
    if (C <= 4096) return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
    if (C <= 8192) return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 2>{});
    return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 4>{});
}

template <class T>
hipError_t forward(NormArgs a, hipStream_t st)
{
    return with_shape(a.C, [&](auto wi, auto pi) {
        constexpr int W = decltype(wi)::value, PER = decltype(pi)::value;
        a.rows = (a.M + 2047) / 2048;
        const int64_t units = (a.M + a.rows - 1) / a.rows;
        const unsigned grid = (unsigned)((units + Unit<W>::kRows - 1) / Unit<W>::kRows);
        if (a.h && a.u)
            k_norm<T, true, true, W, PER><<<grid, Unit<W>::kThreads, 0, st>>>(a);
        else if (a.h)
            k_norm<T, true, false, W, PER><<<grid, Unit<W>::kThreads, 0, st>>>(a);
        else
            k_norm<T, false, true, W, PER><<<grid, Unit<W>::kThreads, 0, st>>>(a);
        return hipGetLastError();
    });
}

// Units of an owner's rows: 512 in all if there are as many rows
int64_t norm_parts(int64_t M, int64_t run)
{
    const int64_t owners = (M + run - 1) / run, want = (512 + owners - 1) / owners;
    const int64_t rows = (run + want - 1) / want;
    return (run + rows - 1) / rows;
}
constexpr int64_t kOwnerBlocks = 64;

template <class T>
hipError_t backward(NormBackArgs a, hipStream_t st)
{
    return with_shape(a.C, [&](auto wi, auto pi) {
        constexpr int W = decltype(wi)::value, PER = decltype(pi)::value;
        const int64_t units = a.owners * a.parts, blocks = (units + Unit<W>::kRows - 1) / Unit<W>::kRows;
        if (blocks > 0x7fffffff) return hipErrorInvalidValue;
        const unsigned grid = (unsigned)blocks;
        if (a.h && a.du)
            k_norm_back<T, true, true, W, PER><<<grid, Unit<W>::kThreads, 0, st>>>(a);
        else if (a.h)
            k_norm_back<T, true, false, W, PER><<<grid, Unit<W>::kThreads, 0, st>>>(a);
        else
            k_norm_back<T, false, true, W, PER><<<grid, Unit<W>::kThreads, 0, st>>>(a);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t st) { return a.f16 ? forward<F16>(a, st) : forward<BF16>(a, st); }

// four sums of each unit, then those of each block of owners
size_t norm_backward_workspace(int64_t M, int64_t C, int64_t run)
{
    if (M == 0) return 0;
    run = run < M ? run : M;
    const int64_t owners = (M + run - 1) / run;
    return (size_t)(4 * (owners * norm_parts(M, run) + (owners < kOwnerBlocks ? owners : kOwnerBlocks)) * C * 4);
}

hipError_t launch_norm_backward(NormBackArgs a, const NormGrads& g, float* workspace, hipStream_t st)
{
    NormSumArgs s = {};
    s.C = a.C, s.weight = a.weight, s.bias = g.bias, s.gate = a.gate, s.dgate = g.dgate;
    a.run = a.run < a.M ? a.run : a.M;
    a.owners = s.owners = a.M ? (a.M + a.run - 1) / a.run : 0;
    a.parts = s.parts = a.M ? norm_parts(a.M, a.run) : 0;
    a.rows = a.M ? (a.run + a.parts - 1) / a.parts : 0;
    const int64_t units = a.owners * a.parts;
    float* const out[4] = {g.dweight, g.dbias, g.dnext_weight, g.dnext_bias};
    const bool want[4] = {g.dweight || g.dgate, g.dbias || (g.dgate && g.bias), g.dnext_weight != nullptr, g.dnext_bias != nullptr};
    bool any = false;
    for (int k = 0; k < 4; ++k) {
        any |= want[k];
        a.part[k] = want[k] && a.M ? workspace + k * units * a.C : nullptr;
        s.part[k] = a.part[k];
    }
    hipError_t e = hipSuccess;
    if (a.M && (e = a.f16 ? backward<F16>(a, st) : backward<BF16>(a, st)) != hipSuccess) return e;
    if (!any) return hipSuccess;
    const int64_t blocks = s.owners < kOwnerBlocks ? s.owners : kOwnerBlocks;
    const dim3 grid((unsigned)((a.C + 63) / 64), (unsigned)(blocks > 1 ? blocks : 1));
    float* second = workspace + 4 * units * a.C;
    for (int k = 0; k < 4; ++k) s.out[k] = !out[k] ? nullptr : blocks > 1 ? second + k * blocks * a.C : out[k];
    k_norm_sums<<<grid, 1024, 0, st>>>(s);
    if ((e = hipGetLastError()) != hipSuccess || blocks <= 1) return e;
    NormSumArgs t = {};
    t.C = a.C, t.owners = 1, t.parts = blocks;
    for (int k = 0; k < 4; ++k) t.part[k] = s.out[k], t.out[k] = out[k];
    k_norm_sums<<<dim3(grid.x, 1), 1024, 0, st>>>(t);
    return hipGetLastError();
}

}  // namespace rtn
