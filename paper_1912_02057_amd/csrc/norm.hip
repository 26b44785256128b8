// Norms before and after a block of a language model, with the block's gate and residual scale, and their gradients:
//   y = scale x + gate (n(h) weight + bias)      u = n(y) next_weight + next_bias
// either line alone or both in one pass.  n is x / sqrt(mean x^2 + eps) or (x - mean) / sqrt(var + eps) of a row.
//
// All of them are one pass over memory: a row stays with the lanes of W waves (PER pieces of 8 columns a lane) from its load to its
// stores, and statistics are sums over those lanes, the variance of the centred values, in fp32.  A unit (W waves) walks
// consecutive rows, so that the vectors of the columns are read once.  Up to 8192 columns (PER 1) all of that is in registers, but for 10 of them
// in the gradients of both lines of a float16 layer norm in 16 waves.  Beyond (PER 2), where 16 waves leave a lane 128 registers, scratch holds 41
// (RMS) or 50 of the forward pass of both lines and 6 to 208 of most gradients.
#include "mx4_math.h"
#include "rtn_kernels.h"

namespace rtn {

namespace {

template <int W>
struct Unit {
    static constexpr int kRows = W == 1 ? 4 : 1, kThreads = W == 1 ? 256 : W * 64;  // units of a block
    static __device__ __forceinline__ int64_t index() { return W == 1 ? (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : (int64_t)blockIdx.x; }
    static __device__ __forceinline__ int lane() { return W == 1 ? threadIdx.x & 63 : threadIdx.x; }
};

// Sum over a wave, in a scalar register: within rows of 16 lanes, then across them, all in the vector unit.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float v)
{
    v = dpp_add<0x111>(v);  // row_shr 1, 2, 4, 8: lane 15 of a row has its sum
    v = dpp_add<0x112>(v);
    v = dpp_add<0x114>(v);
    v = dpp_add<0x118>(v);
    v = dpp_add<0x142>(v);  // row_bcast 15, 31: lane 63 has the wave's
    v = dpp_add<0x143>(v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
// Sums over a unit, in all its lanes: each wave's, then those over lanes that hold one wave's each.  `turn` alternates between two sets of LDS
// words, so that one barrier a sum is enough.
template <int W, int N>
__device__ __forceinline__ void unit_sums(float (&v)[N], float (*lds)[2][W], int& turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (W > 1) {
        static_assert(W == 4 || W == 8 || W == 16, "the waves' sums fill a part of a row of lanes");
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) lds[turn][i][wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float t = lds[turn][i][threadIdx.x & (W - 1)];
            t = dpp_add<0x111>(t);
            t = dpp_add<0x112>(t);
            if constexpr (W > 4) t = dpp_add<0x114>(t);
            if constexpr (W > 8) t = dpp_add<0x118>(t);
            v[i] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(t), W - 1));
        }
        turn ^= 1;
    }
}

template <int PER>
struct Cols {
    float v[PER][8];
};
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));  // of a vector that starts anywhere
template <int W>
__device__ __forceinline__ int64_t column(int j) { return (int64_t)(j * W * 64 + Unit<W>::lane()) * 8; }
// A lane's part of a row.  Loaded without a branch, so that the loads of several rows are in flight together: pieces that the row does not fill
// come from its last 16 bytes and are put right when they are used (settle).
template <int W, int PER>
struct Row {
    u32x4 q[PER];
    __device__ __forceinline__ void load(const void* base, int64_t ld, int64_t m, int64_t C)
    {
        const unsigned short* row = (const unsigned short*)base + m * ld;
        if (C < 8) {
#pragma unroll
            for (int j = 0; j < PER; ++j) q[j] = load_row8(row, column<W>(j), C);
            return;
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int64_t k = column<W>(j);
            q[j] = load16(row + (k < C - 8 ? k : C - 8));
        }
    }
    __device__ __forceinline__ void settle(int64_t C)
    {
        if (C < 8) return;
        if (C % 8 == 0) {
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (column<W>(j) >= C) q[j] = u32x4{0, 0, 0, 0};
            return;
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int64_t over = column<W>(j) + 8 - C;  // elements that are not there
            const int n = over <= 0 ? 0 : over < 8 ? (int)over * 16 : 128;
            const uint64_t lo = q[j][0] | (uint64_t)q[j][1] << 32, hi = q[j][2] | (uint64_t)q[j][3] << 32;
            const uint64_t l = n >= 64 ? hi >> (n & 63) : n ? lo >> n | hi << (64 - n) : lo, u = n >= 64 ? 0 : hi >> n;
            q[j] = n == 128 ? u32x4{0, 0, 0, 0} : u32x4{(unsigned)l, (unsigned)(l >> 32), (unsigned)u, (unsigned)(u >> 32)};
        }
    }
    template <class T>
    __device__ __forceinline__ float get(int j, int i) const
    {
        return half_of<T>(q[j][i >> 1], i & 1);
    }
};
// A vector of the columns, or `otherwise` where it is NULL.  Past the end are others of its entries, which reach no sum and no output.
template <int W, int PER>
__device__ __forceinline__ void load_cols(Cols<PER>& c, const float* p, int64_t C, float otherwise)
{
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int64_t k = column<W>(j);
        if (!p) {
#pragma unroll
            for (int i = 0; i < 8; ++i) c.v[j][i] = otherwise;
        } else if (C < 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) c.v[j][i] = p[k + i < C ? k + i : C - 1];
        } else {
            const f32x4_any* q = (const f32x4_any*)(p + (k < C - 8 ? k : C - 8));
            const f32x4_any a = q[0], b = q[1];
            const int over = k < C && k > C - 8 ? (int)(k - (C - 8)) : 0;  // of the lane that has the row's end
            const bool by4 = over & 4, by2 = over & 2, by1 = over & 1;
            const f32x4_any a4 = by4 ? b : a, b4 = b;
            const f32x4_any a2 = by2 ? f32x4_any{a4[2], a4[3], b4[0], b4[1]} : a4, b2 = by2 ? f32x4_any{b4[2], b4[3], b4[2], b4[3]} : b4;
            const f32x4_any a1 = by1 ? f32x4_any{a2[1], a2[2], a2[3], b2[0]} : a2, b1 = by1 ? f32x4_any{b2[1], b2[2], b2[3], b2[3]} : b2;
#pragma unroll
            for (int i = 0; i < 4; ++i) c.v[j][i] = a1[i], c.v[j][4 + i] = b1[i];
        }
    }
}
// (rounded and returned as rounded)
template <class T, int W, int PER>
__device__ __forceinline__ void store_row(void* base, int64_t ld, int64_t m, int64_t C, Cols<PER>& v)
{
    unsigned short* row = (unsigned short*)base + m * ld;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int64_t k = column<W>(j);
        const u32x4 q = {pack2<T>(v.v[j][0], v.v[j][1]), pack2<T>(v.v[j][2], v.v[j][3]), pack2<T>(v.v[j][4], v.v[j][5]), pack2<T>(v.v[j][6], v.v[j][7])};
#pragma unroll
        for (int i = 0; i < 8; ++i) v.v[j][i] = half_of<T>(q[i >> 1], i & 1);
        if (k + 8 <= C) {
            store16(row + k, q);
        } else if (C % 8) {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (k + i < C) row[k + i] = (unsigned short)(i & 1 ? q[i >> 1] >> 16 : q[i >> 1] & 0xffffu);
        }
    }
}
template <int W>
__device__ __forceinline__ bool inside(int j, int i, int64_t C) { return column<W>(j) + i < C; }

// Elementwise over a lane's part of a row: f(j, i)
template <int PER, class F>
__device__ __forceinline__ void each(F f)
{
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) f(j, i);
}

// 1 / sqrt(v) within an ulp, also of numbers that the instruction takes as 0
__device__ __forceinline__ float inverse_root(float v)
{
    const bool small = v < 0x1p-96f;
    return __builtin_amdgcn_rsqf(small ? v * 0x1p96f : v) * (small ? 0x1p48f : 1.f);
}
// K rows v -> n(v), and 1 / sqrt(..) of each.  A mean in fp32 is off by its sum's roundings, which a row of small variance divides by a small
// number: what is left of it in the centred values is summed with their squares and taken off too.
template <bool LAYER, int W, int PER, int K>
__device__ __forceinline__ void normalise(Cols<PER> (&v)[K], float (&r)[K], int64_t C, float eps, float (*lds)[2][W], int& turn)
{
    const float inv = 1.f / (float)C;
    float s[K] = {}, rest[K] = {};
    if constexpr (LAYER) {
#pragma unroll
        for (int k = 0; k < K; ++k) each<PER>([&](int j, int i) { s[k] += v[k].v[j][i]; });
        unit_sums<W, K>(s, lds, turn);
        float q[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float mean = s[k] * inv;
            each<PER>([&](int j, int i) { v[k].v[j][i] = inside<W>(j, i, C) ? v[k].v[j][i] - mean : 0.f; });
            q[0] = q[1] = 0.f;
            each<PER>([&](int j, int i) { q[0] = fmaf(v[k].v[j][i], v[k].v[j][i], q[0]), q[1] += v[k].v[j][i]; });
            unit_sums<W, 2>(q, lds, turn);
            rest[k] = q[1] * inv;
            s[k] = fmaf(-rest[k], q[1], q[0]);
            s[k] = s[k] < 0.f ? 0.f : s[k];  // (a NaN stays one)
        }
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) each<PER>([&](int j, int i) { s[k] = fmaf(v[k].v[j][i], v[k].v[j][i], s[k]); });
        unit_sums<W, K>(s, lds, turn);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        r[k] = inverse_root(fmaf(s[k], inv, eps));
        each<PER>([&](int j, int i) { v[k].v[j][i] = LAYER ? (v[k].v[j][i] - rest[k]) * r[k] : v[k].v[j][i] * r[k]; });
    }
}
// dn, the gradient of n(v) -> that of v:  r (dn - n mean(dn n) [- mean(dn)])
template <bool LAYER, int W, int PER>
__device__ __forceinline__ void normalise_back(Cols<PER>& dn, const Cols<PER>& n, float r, int64_t C, float (*lds)[2][W], int& turn)
{
    float s[LAYER ? 2 : 1] = {};
    each<PER>([&](int j, int i) {
        s[0] = fmaf(dn.v[j][i], n.v[j][i], s[0]);
        if constexpr (LAYER) s[1] += dn.v[j][i];
    });
    unit_sums<W, LAYER ? 2 : 1>(s, lds, turn);
    const float inv = 1.f / (float)C, a = s[0] * inv * r;
    if constexpr (LAYER) {
        const float b = s[1] * inv * r;
        each<PER>([&](int j, int i) { dn.v[j][i] = fmaf(dn.v[j][i], r, -fmaf(n.v[j][i], a, b)); });
    } else {
        each<PER>([&](int j, int i) { dn.v[j][i] = fmaf(dn.v[j][i], r, -n.v[j][i] * a); });
    }
}

// POST: y = scale x + gate (n(h) weight + bias); without it y is x.  PRE: u = n(y) next_weight + next_bias.
// The next row is fetched while this one is worked on: a block of 16 waves has its CU to itself, and a row's sums and barriers take as long as
// its bytes (16384 x 8192, both lines: 260 us without, 200 with: 5.4 TB/s, the rate of a large copy; the first line alone 168 to 185, 4.4 to 4.8
// TB/s, the second alone 86 to 89, 6.1).  4096 x 16384: the second line alone 48 us, 5.6 TB/s, both 144 to 153, 3.6, with the registers of
// PER 2 in scratch.
template <class T, bool LAYER, bool POST, bool PRE, int W, int PER>
__global__ __launch_bounds__(Unit<W>::kThreads) void k_norm(NormArgs a)
{
    __shared__ __attribute__((aligned(16))) float lds[2][2][W];
    int turn = 0;
    const int64_t first = Unit<W>::index() * a.rows, end = first + a.rows < a.M ? first + a.rows : a.M;
    if (first >= end) return;
    Row<W, PER> x, h, x_next, h_next;
    x.load(a.x, a.ldx, first, a.C);
    if constexpr (POST) h.load(a.h, a.ldh, first, a.C);
    Cols<PER> w, b, gate, nw, nb;
    if constexpr (POST) load_cols<W>(w, a.weight, a.C, 1.f), load_cols<W>(b, a.bias, a.C, 0.f);
    if constexpr (PRE) load_cols<W>(nw, a.next_weight, a.C, 1.f), load_cols<W>(nb, a.next_bias, a.C, 0.f);
    int64_t owner = -1, owner_end = first;
    for (int64_t m = first; m < end; ++m) {
        if (m + 1 < end) {
            x_next.load(a.x, a.ldx, m + 1, a.C);
            if constexpr (POST) h_next.load(a.h, a.ldh, m + 1, a.C);
        }
        Cols<PER> rows[1], &v = rows[0];
        float r[1];
        x.settle(a.C);
        if constexpr (POST) h.settle(a.C);
        if constexpr (POST) {
            if (m >= owner_end) {
                owner = m / a.run, owner_end = (owner + 1) * a.run;
                load_cols<W>(gate, a.gate ? a.gate + owner * a.C : nullptr, a.C, 1.f);
            }
            each<PER>([&](int j, int i) { v.v[j][i] = h.template get<T>(j, i); });
            normalise<LAYER, W, PER, 1>(rows, r, a.C, a.eps, lds, turn);
            each<PER>([&](int j, int i) { v.v[j][i] = fmaf(gate.v[j][i], fmaf(v.v[j][i], w.v[j][i], b.v[j][i]), a.scale * x.template get<T>(j, i)); });
            store_row<T, W, PER>(a.y, a.ldy, m, a.C, v);
        } else {
            each<PER>([&](int j, int i) { v.v[j][i] = x.template get<T>(j, i); });
        }
        if constexpr (PRE) {
            if constexpr (POST) each<PER>([&](int j, int i) { v.v[j][i] = inside<W>(j, i, a.C) ? v.v[j][i] : 0.f; });
            normalise<LAYER, W, PER, 1>(rows, r, a.C, a.eps, lds, turn);
            each<PER>([&](int j, int i) { v.v[j][i] = fmaf(v.v[j][i], nw.v[j][i], nb.v[j][i]); });
            store_row<T, W, PER>(a.u, a.ldu, m, a.C, v);
        }
        x = x_next;
        if constexpr (POST) h = h_next;
    }
}

// With d the gradient of y, du's part among it:
//   dx = scale d,  dh = n'(h) (d gate weight),  and per unit, for k_norm_sums: sum d n(h), sum d, sum du n(y), sum du
// A unit's rows share a row of the gate.  BIASES: the second and fourth sum are wanted.  Rows are fetched ahead as above (16384 x 8192: 411 us
// with loads that wait for each other, 320 in flight together: 5.0 TB/s); with PER of 2 there are no registers for that, and the vectors of
// the columns are read again for every row (4096 x 16384: 415 to 427 us, 1.9 TB/s, as a layer norm 705; the second line alone 116 to 120, 4.5 TB/s).
template <class T, bool LAYER, bool POST, bool PRE, bool BIASES, int W, int PER>
__global__ __launch_bounds__(Unit<W>::kThreads) void k_norm_back(NormBackArgs a)
{
    constexpr bool KEEP = PER == 1;
    __shared__ __attribute__((aligned(16))) float lds[2][2][W];
    int turn = 0;
    const int64_t unit = Unit<W>::index();
    if (unit >= a.owners * a.parts) return;
    const int64_t owner = unit / a.parts, from = (unit - owner * a.parts) * a.rows;
    const int64_t run_end = (owner + 1) * a.run < a.M ? (owner + 1) * a.run : a.M;
    const int64_t first = owner * a.run + from, end = first + a.rows < run_end ? first + a.rows : run_end;
    struct Rows {
        Row<W, PER> dy, du, h, y;
    } now, next;
    auto load = [&](Rows& r, int64_t m) {
        if (a.dy) r.dy.load(a.dy, a.lddy, m, a.C);
        if constexpr (PRE) r.du.load(a.du, a.lddu, m, a.C), r.y.load(a.y, a.ldy, m, a.C);
        if constexpr (POST) r.h.load(a.h, a.ldh, m, a.C);
    };
    if (KEEP && first < end) load(now, first);
    Cols<PER> gw, nw, sums[4];
    auto post_vectors = [&] {
        Cols<PER> gate;
        load_cols<W>(gw, a.weight, a.C, 1.f);
        load_cols<W>(gate, a.gate ? a.gate + owner * a.C : nullptr, a.C, 1.f);
        each<PER>([&](int j, int i) { gw.v[j][i] *= gate.v[j][i]; });
    };
    if constexpr (KEEP && POST) post_vectors();
    if constexpr (KEEP && PRE) load_cols<W>(nw, a.next_weight, a.C, 1.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) each<PER>([&](int j, int i) { sums[k].v[j][i] = 0.f; });
    for (int64_t m = first; m < end; ++m) {
        if (!KEEP) {
            load(now, m);
        } else if (m + 1 < end) {
            load(next, m + 1);
        }
        if (a.dy) now.dy.settle(a.C);
        if constexpr (PRE) now.du.settle(a.C), now.y.settle(a.C);
        if constexpr (POST) now.h.settle(a.C);
        constexpr int K = (POST ? 1 : 0) + (PRE ? 1 : 0);
        Cols<PER> d, n[K];  // n(h) first, n(y) last
        float r[K];
        if constexpr (POST) each<PER>([&](int j, int i) { n[0].v[j][i] = now.h.template get<T>(j, i); });
        if constexpr (PRE) each<PER>([&](int j, int i) { n[K - 1].v[j][i] = now.y.template get<T>(j, i); });
        normalise<LAYER, W, PER, K>(n, r, a.C, a.eps, lds, turn);
        if constexpr (PRE) {
            if (!KEEP) load_cols<W>(nw, a.next_weight, a.C, 1.f);
            each<PER>([&](int j, int i) {
                const float g = now.du.template get<T>(j, i);
                sums[2].v[j][i] = fmaf(g, n[K - 1].v[j][i], sums[2].v[j][i]);
                if (BIASES) sums[3].v[j][i] += g;
                d.v[j][i] = g * nw.v[j][i];
            });
            normalise_back<LAYER, W, PER>(d, n[K - 1], r[K - 1], a.C, lds, turn);
            if (a.dy) each<PER>([&](int j, int i) { d.v[j][i] += now.dy.template get<T>(j, i); });
        } else {
            each<PER>([&](int j, int i) { d.v[j][i] = now.dy.template get<T>(j, i); });
        }
        if (a.dx) {
            Cols<PER> v;
            each<PER>([&](int j, int i) { v.v[j][i] = a.scale * d.v[j][i]; });
            store_row<T, W, PER>(a.dx, a.lddx, m, a.C, v);
        }
        if constexpr (POST) {
            if (!KEEP) post_vectors();
            each<PER>([&](int j, int i) {
                sums[0].v[j][i] = fmaf(d.v[j][i], n[0].v[j][i], sums[0].v[j][i]);
                if (BIASES) sums[1].v[j][i] += d.v[j][i];
                // (past the end d is 0 without a mean)
                d.v[j][i] = !LAYER || inside<W>(j, i, a.C) ? d.v[j][i] * gw.v[j][i] : 0.f;
            });
            if (a.dh) {
                normalise_back<LAYER, W, PER>(d, n[0], r[0], a.C, lds, turn);
                store_row<T, W, PER>(a.dh, a.lddh, m, a.C, d);
            }
        }
        if (KEEP) now = next;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (a.part[k]) {
            float* out = a.part[k] + unit * a.C;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int64_t c = column<W>(j);
                if (c + 8 <= a.C) {
                    const float* v = sums[k].v[j];
                    ((f32x4_any*)(out + c))[0] = f32x4_any{v[0], v[1], v[2], v[3]};
                    ((f32x4_any*)(out + c))[1] = f32x4_any{v[4], v[5], v[6], v[7]};
                } else {
#pragma unroll
                    for (int i = 0; i < 7; ++i)
                        if (c + i < a.C) out[c + i] = sums[k].v[j][i];
                }
            }
        }
}

// The units' sums into the gradients of the vectors, in one order: 16 columns a block, its SLICES groups of 16 lanes share the units of one owner (a
// row of the gate), and blockIdx.y owners out of a.owners.  With S, T the first two sums over an owner's units:
//   dgate = S weight + T bias,  dweight += gate S,  dbias += gate T
// Several blocks of owners leave partial sums for a second launch.  Made for few owners with many units each: with a gate for every token, where
// an owner has one, a single slice loads, and a block passes from owner to owner (16384 x 8192, RMS: 7.5 ms, beside 0.7 of k_norm_back).
constexpr int kSumCols = 16;
template <int SLICES>
__global__ __launch_bounds__(SLICES * 16) void k_norm_sums(NormSumArgs a)
{
    __shared__ float lds[4][SLICES][kSumCols + 1];
    const int col = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const int64_t c = (int64_t)blockIdx.x * kSumCols + col, per = (a.owners + gridDim.y - 1) / gridDim.y;
    const int64_t o0 = blockIdx.y * per, o1 = o0 + per < a.owners ? o0 + per : a.owners;
    const bool in = c < a.C;
    float total[4] = {0.f, 0.f, 0.f, 0.f};
    const float w = in && a.weight ? a.weight[c] : 1.f, b = in && a.bias ? a.bias[c] : 0.f;
    for (int64_t o = o0; o < o1; ++o) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float s = 0.f;
            if (in && a.part[k]) {
                const float* p = a.part[k] + o * a.parts * a.C + c;
#pragma unroll 8
                for (int64_t u = slice; u < a.parts; u += SLICES) s += p[u * a.C];
            }
            lds[k][slice][col] = s;
        }
        __syncthreads();
        if (slice < 4) {  // slice k of 16 lanes adds up the k-th sum
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < SLICES; ++v) s += lds[slice][v][col];
            lds[slice][0][col] = s;  // (each lane's own column)
        }
        __syncthreads();
        if (slice == 0 && in) {
            float s[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k] = lds[k][0][col];
            const float g = a.gate ? a.gate[o * a.C + c] : 1.f;
            if (a.dgate) a.dgate[o * a.C + c] = fmaf(s[0], w, s[1] * b);
            total[0] = fmaf(g, s[0], total[0]), total[1] = fmaf(g, s[1], total[1]);
            total[2] += s[2], total[3] += s[3];
        }
        __syncthreads();
    }
    if (slice == 0 && in) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (a.out[k]) a.out[k][(int64_t)blockIdx.y * a.C + c] = total[k];
    }
}

// W waves of PER pieces for rows of C columns
inline int norm_waves(int64_t C) { return C <= 512 ? 1 : C <= 2048 ? 4 : C <= 4096 ? 8 : 16; }
template <class F>
hipError_t with_shape(int64_t C, F&& f)
{
    const std::integral_constant<int, 1> one{};
    switch (norm_waves(C)) {
        case 1: return f(one, one);
        case 4: return f(std::integral_constant<int, 4>{}, one);
        case 8: return f(std::integral_constant<int, 8>{}, one);
        default: return C <= 8192 ? f(std::integral_constant<int, 16>{}, one) : f(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
    }
}
// Units that the chip holds at once: 16 waves to a CU
inline int64_t norm_units(int64_t C) { return 256 * 16 / norm_waves(C); }

template <class T, bool LAYER>
hipError_t forward(NormArgs a, hipStream_t st)
{
    return with_shape(a.C, [&](auto wi, auto pi) {
        constexpr int W = decltype(wi)::value, PER = decltype(pi)::value;
        a.rows = (a.M + 2 * norm_units(a.C) - 1) / (2 * norm_units(a.C));  // (twice what the registers of the largest form allow)
        const int64_t units = (a.M + a.rows - 1) / a.rows;
        const unsigned grid = (unsigned)((units + Unit<W>::kRows - 1) / Unit<W>::kRows);
        if (a.h && a.u)
            k_norm<T, LAYER, true, true, W, PER><<<grid, Unit<W>::kThreads, 0, st>>>(a);
        else if (a.h)
            k_norm<T, LAYER, true, false, W, PER><<<grid, Unit<W>::kThreads, 0, st>>>(a);
        else
            k_norm<T, LAYER, false, true, W, PER><<<grid, Unit<W>::kThreads, 0, st>>>(a);
        return hipGetLastError();
    });
}

// Units of an owner's rows: as many in all as the chip holds for many rows, down to one a CU for a few, since each leaves its sums (1000 x 2187:
// 500 units 17.5 us and 9.3 for their sums, 250 units 15.6 and 5.7; with
// both, 128 / 256 / 512 / 1024 / 2048 units: 2000 x 8192 40 31 36 45, 8192 x 4096 88 53 42 46 52, 16384 x 512 108 59 35 24 21).
// No more in all than the chip holds, since what is beyond is a second round of as many rows each (three gates, 16384 x 8192: 3 x 86 units 469 us,
// 3 x 85 335); but where a unit an owner would leave more than a third of the chip idle, three of them in two rounds (300 gates,
// 16384 x 2187, 512 at once: 1 each 222, 2 196, 3 176).
int64_t norm_parts(int64_t M, int64_t C, int64_t run)
{
    const int64_t all = norm_units(C), few = M / 8 < 256 ? 256 : M / 8, units = few < all ? few : all;
    const int64_t owners = (M + run - 1) / run, wish = (units + owners - 1) / owners, fit = all / owners;
    const int64_t want = wish <= fit ? wish : fit > 1 ? fit : wish > 1 && 3 * owners < 2 * all ? 3 : 1, rows = (run + want - 1) / want;
    return (run + rows - 1) / rows;
}
constexpr int64_t kOwnerBlocks = 64;

template <class T, bool LAYER, bool BIASES>
hipError_t backward(const NormBackArgs& a, hipStream_t st)
{
    return with_shape(a.C, [&](auto wi, auto pi) {
        constexpr int W = decltype(wi)::value, PER = decltype(pi)::value;
        const int64_t units = a.owners * a.parts, blocks = (units + Unit<W>::kRows - 1) / Unit<W>::kRows;
        if (blocks > 0x7fffffff) return hipErrorInvalidValue;
        const unsigned grid = (unsigned)blocks;
        if (a.h && a.du)
            k_norm_back<T, LAYER, true, true, BIASES, W, PER><<<grid, Unit<W>::kThreads, 0, st>>>(a);
        else if (a.h)
            k_norm_back<T, LAYER, true, false, BIASES, W, PER><<<grid, Unit<W>::kThreads, 0, st>>>(a);
        else
            k_norm_back<T, LAYER, false, true, BIASES, W, PER><<<grid, Unit<W>::kThreads, 0, st>>>(a);
        return hipGetLastError();
    });
}

hipError_t run_sums(const NormSumArgs& a, dim3 grid, hipStream_t st)
{
    if (a.parts > 64)
        k_norm_sums<64><<<grid, 1024, 0, st>>>(a);
    else
        k_norm_sums<16><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t st)
{
    if (a.layer) return a.f16 ? forward<F16, true>(a, st) : forward<BF16, true>(a, st);
    return a.f16 ? forward<F16, false>(a, st) : forward<BF16, false>(a, st);
}

// four sums of each unit, then those of each block of owners
size_t norm_backward_workspace(int64_t M, int64_t C, int64_t run)
{
    if (M == 0) return 0;
    run = run < M ? run : M;
    const int64_t owners = (M + run - 1) / run;
    return (size_t)(4 * (owners * norm_parts(M, C, run) + (owners < kOwnerBlocks ? owners : kOwnerBlocks)) * C * 4);
}

hipError_t launch_norm_backward(NormBackArgs a, const NormGrads& g, float* workspace, hipStream_t st)
{
    NormSumArgs s = {};
    s.C = a.C, s.weight = a.weight, s.bias = g.bias, s.gate = a.gate, s.dgate = g.dgate;
    a.run = a.run < a.M ? a.run : a.M;
    a.owners = s.owners = a.M ? (a.M + a.run - 1) / a.run : 0;
    a.parts = s.parts = a.M ? norm_parts(a.M, a.C, a.run) : 0;
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
    const bool biases = want[1] || want[3];
    if (a.M && a.layer)  // (biases there or not: a layer norm without them pays for two sums)
        e = a.f16 ? backward<F16, true, true>(a, st) : backward<BF16, true, true>(a, st);
    else if (a.M && biases)
        e = a.f16 ? backward<F16, false, true>(a, st) : backward<BF16, false, true>(a, st);
    else if (a.M)
        e = a.f16 ? backward<F16, false, false>(a, st) : backward<BF16, false, false>(a, st);
    if (e != hipSuccess) return e;
    if (!any) return hipSuccess;
    const int64_t blocks = s.owners < kOwnerBlocks ? s.owners : kOwnerBlocks;
    const dim3 grid((unsigned)((a.C + kSumCols - 1) / kSumCols), (unsigned)(blocks > 1 ? blocks : 1));
    float* second = workspace + 4 * units * a.C;
    for (int k = 0; k < 4; ++k) s.out[k] = !out[k] ? nullptr : blocks > 1 ? second + k * blocks * a.C : out[k];
    if ((e = run_sums(s, grid, st)) != hipSuccess || blocks <= 1) return e;
    NormSumArgs t = {};
    t.C = a.C, t.owners = 1, t.parts = blocks;
    for (int k = 0; k < 4; ++k) t.part[k] = s.out[k], t.out[k] = out[k];
    return run_sums(t, dim3(grid.x, 1), st);
}

}  // namespace rtn
