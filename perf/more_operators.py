"""Performance cases of the microscaled 4-bit operators of language models and of the norms around their blocks.

Each case is one pass of something a program built on this library does.  With `own` the pass goes
through the binding (mx4_pack, mx4_unpack, mx4_linear, mx4_linear_backward, norm, norm_backward,
block_norm, block_norm_backward); without it the same operators run in elementary torch operations
in 32 bits.

Microscaled 4-bit values: 32 consecutive columns of a row share a power of two 2^e (8 bits), a value
is q 2^e with q one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign.  With a = max |v| of the group:
  to nearest   e = floor(log2 a) - 2 (at least -127), q the nearest of v / 2^e, ties to the even
               code, 6 beyond 6
  stochastic   e is one more where a / 2^e > 6; q is the upper neighbour of |v| / 2^e in the place of
               the lower one where k < 65536 * (their distance in units of the gap), k 16 bits of
               Philox4x32-10 (Salmon et al. 2011): key = the seed's two words, counter = (the
               group's index row * groups + group: low, high word; j = 0 .. 3; 0, or 1 for the
               transposed packing).  Element i takes bits 16 (i & 1) .. of word (i / 2) & 3 of j = i / 8.
Q(v) is what such a packing of v stands for, Qt(v) = Q(v^T), grouped along v's rows.

The operators, for M tokens, K input and N output features:
  pack         Q(v), and Qt(v) where both directions are wanted
  linear       y = act(Q(x) Q(w)^T + bias) + residual, weights packed once by a model that answers
  train        a layer's step from this step's fp32 weights: y as above; then with dz = dy act'(z)
               (z kept in 16 bits) and stochastic packings of dz
               dx = Q(dz) Qt(w)^T,  dw = Qt(dz) Qt(x)^T,  dbias = sum_m dz
  norm         u = n(x) weight + bias, n(x) = x / sqrt(mean x^2 + eps) or (x - mean) / sqrt(var + eps);
               with the gradients of x (on top of the residual path's), weight and bias in training
  block        the end of a block and the start of the next one in one pass:
               y = scale x + gate (n(h) weight + bias),  u = n(y) next_weight + next_bias
               with gate [G][C], one row for a run of tokens; in training the gradients of everything

Sizes are those of the repository's GEMM configurations (4096^3, 16384 x 8192 x 8192, 1000 x 1003 x
2187) or generic powers of two, with odd ones drawn.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


def listed():
    return [
        # the activation of a short sequence into 4 bits and back: latency
        dict(name="pack_small", kind="pack", dtype="fp16", M=77, K=1024, both=False, stochastic=False),
        # a large training batch's gradient for both of its products, rounded stochastically
        dict(name="pack_large", kind="pack", dtype="bf16", M=16384, K=8192, both=True, stochastic=True),
        # one token through a square projection with its residual: a decoding step's layer
        dict(name="linear_one_token", kind="linear", dtype="bf16", M=1, N=4096, K=4096, act="none", residual=True),
        # a batch of sequences decoding together
        dict(name="linear_24_tokens", kind="linear", dtype="fp16", M=24, N=8192, K=8192, act="silu", residual=False),
        # a prompt of odd length through a layer of odd sizes
        dict(name="linear_ragged", kind="linear", dtype="fp16", M=1000, N=1003, K=2187, act="gelu", residual=True),
        # the largest point of the benchmark's GEMM sweep as a layer
        dict(name="linear_16384x8192", kind="linear", dtype="bf16", M=16384, N=8192, K=8192, act="none", residual=True),
        # fine-tuning on a short sequence: launches and latency count
        dict(name="train_small", kind="train", dtype="bf16", M=256, N=1024, K=1024, act="relu", residual=True),
        # a training step of the GEMM configuration
        dict(name="train_4096", kind="train", dtype="bf16", M=4096, N=4096, K=4096, act="none", residual=False),
        # the norm before a decoding step's block
        dict(name="norm_one_token", kind="norm", dtype="bf16", M=1, C=4096, layer=False, bias=False, train=False),
        # odd sizes, layer norm with biases, a training step
        dict(name="norm_ragged", kind="norm", dtype="fp16", M=1000, C=2187, layer=True, bias=True, train=True),
        # between two blocks of a decoding step of several sequences
        dict(name="block_24_tokens", kind="block", dtype="bf16", M=24, C=8192, layer=False, bias=False, G=1, train=False),
        # between two blocks of a training step, a gate for each of 8 sequences
        dict(name="block_train", kind="block", dtype="bf16", M=16384, C=8192, layer=False, bias=False, G=8, train=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A number of features: mostly a multiple of 64, as layers have, now and then any number."""
    v = _log_int(rng, lo, hi)
    return v if rng.random() < 0.3 else max(64, v // 64 * 64)


def draw(rng):
    kind = rng.choice(["pack"] * 2 + ["linear"] * 4 + ["train"] * 2 + ["norm"] * 2 + ["block"] * 2)
    c = dict(kind=kind, dtype=rng.choice(["bf16", "fp16"]))
    if kind == "pack":
        if rng.random() < 0.25:
            c["dtype"] = "fp32"
        c.update(M=_log_int(rng, 1, 16384), K=_width(rng, 64, 8192), both=rng.random() < 0.5, stochastic=rng.random() < 0.5)
    elif kind in ("linear", "train"):
        most = 16384 * 8192 * 8192 if kind == "linear" else 4096 ** 3
        while True:
            # half of the layers that answer do it for a few tokens
            M = _log_int(rng, 1, 64) if kind == "linear" and rng.random() < 0.5 else _log_int(rng, 16, 16384)
            N, K = _width(rng, 64, 16384), _width(rng, 64, 16384)
            if M * N * K <= most:
                break
        acts = ["none", "relu", "gelu", "silu"] if kind == "linear" else ["none", "relu"]
        c.update(M=M, N=N, K=K, act=rng.choice(acts), residual=rng.random() < 0.5)
    else:
        while True:
            M, C = _log_int(rng, 1, 16384), _width(rng, 64, 16384)
            if M * C <= 16384 * 8192:
                break
        layer = rng.random() < 0.5
        c.update(M=M, C=C, layer=layer, bias=layer and rng.random() < 0.7, train=rng.random() < 0.6)
        if kind == "block":
            c["G"] = rng.choice([1, min(M, 3), min(M, 16)])
    return c


# ------------------------------------------------------------------ inputs

def _activations(M, C, dtype, g):
    """Normal values whose channels differ in scale, a few of them by much, as those of a language model do."""
    scale = torch.exp(0.5 * torch.randn(C, generator=g, device=DEV))
    scale *= torch.where(torch.rand(C, generator=g, device=DEV) < 0.005, 20.0, 1.0)
    return torch.randn((M, C), generator=g, device=DEV).mul_(scale).to(dtype)


def _run(c):
    """Tokens that share a row of the gate: the last run may be shorter."""
    return -(-c["M"] // c["G"])


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & 0x7FFFFFFF)
    dtype, M = DTYPES[c["dtype"]], c["M"]
    normal = lambda *shape: torch.randn(shape, generator=g, device=DEV)
    s = dict(case=c)
    if c["kind"] in ("norm", "block"):
        C = c["C"]
        s["x"] = _activations(M, C, dtype, g)
        s["weight"] = 1 + 0.2 * normal(C)
        s["bias"] = 0.1 * normal(C) if c["bias"] else None
        if c["kind"] == "block":
            s["h"] = _activations(M, C, dtype, g)
            s["gate"] = 0.5 + 0.3 * normal(-(-M // _run(c)), C)
            s["scale"] = 0.75
            s["next_weight"] = 1 + 0.2 * normal(C)
            s["next_bias"] = 0.1 * normal(C) if c["bias"] else None
        if c["train"]:
            s["du"] = normal(M, C).to(dtype)
            s["dy"] = normal(M, C).to(dtype)
        return s
    K = c["K"]
    s["x"] = _activations(M, K, dtype, g)
    # the seed of the stochastic rounding: on the device, so that a captured graph takes a new one every step
    s["seed"] = torch.randint(-2 ** 62, 2 ** 62, (1,), generator=g, device=DEV)
    if c["kind"] == "pack":
        return s
    N = c["N"]
    w = normal(N, K) / math.sqrt(K)
    s["bias"] = (0.1 * normal(N)).to(dtype)
    s["residual"] = normal(M, N).to(dtype) if c["residual"] else None
    if c["kind"] == "train":
        s["w"] = w
        s["dy"] = normal(M, N).to(dtype)
    elif own:  # a model that answers packs its weights once ...
        from paper_1912_02057_amd import binding as B
        s["weights"] = B.mx4_pack(w)
    else:  # ... here to the matrix that the product takes
        s["weights"] = _four(w)
    return s


# ------------------------------------------------------------------ the plain forms, in 32 bits

def _philox(c0, c1, c2, c3, k0, k1):
    """Four 32-bit words of every counter, as int64 tensors."""
    low = 0xFFFFFFFF
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # mod 2^64
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _bits16(first, groups, seed, transposed):
    """The 16-bit numbers of groups first .. first + groups - 1: [groups][32]."""
    index = torch.arange(first, first + groups, device=DEV)[:, None].expand(groups, 4)
    j = torch.arange(4, device=DEV).expand(groups, 4)
    zero = torch.zeros_like(j)
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    words = torch.stack(_philox(index & 0xFFFFFFFF, zero + (index >> 32), j + 0, zero + int(transposed), k0, k1), dim=-1)
    return torch.stack([words & 0xFFFF, words >> 16], dim=-1).view(groups, 32)


def _four(v, seed=None, transposed=False):
    """What the 4-bit packing of v's rows stands for, in 32 bits."""
    R, C = v.shape
    n = -(-C // 32)
    v = torch.nn.functional.pad(v.float(), (0, 32 * n - C)).reshape(R * n, 32)
    out = torch.empty_like(v)
    for i in range(0, R * n, 1 << 20):  # some groups at a time: the random words take 8 bytes each
        p = v[i:i + (1 << 20)]
        a = p.abs().amax(dim=1, keepdim=True)
        e = torch.clamp(torch.frexp(a)[1] - 3, min=-127)
        if seed is not None:
            e = e + (torch.ldexp(a, -e) > 6).int()
        r = torch.ldexp(p.abs(), -e)
        gap = torch.where(r < 2, 0.5, torch.where(r < 4, 1.0, 2.0))
        if seed is None:
            q = torch.clamp(torch.round(r / gap) * gap, max=6)
        else:
            low = torch.floor(r / gap)
            q = (low + (_bits16(i, p.shape[0], seed, transposed) < (r / gap - low) * 65536).float()) * gap
        out[i:i + (1 << 20)] = torch.copysign(torch.ldexp(q, e), p)
    return out.view(R, 32 * n)[:, :C]


def _act(z, act):
    if act == "relu":
        return torch.clamp_min(z, 0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _normalise(x, layer):
    """(n(x), the factor of each row)"""
    if layer:
        x = x - x.mean(dim=1, keepdim=True)
    r = 1 / torch.sqrt((x * x).mean(dim=1, keepdim=True) + EPS)
    return x * r, r


def _normalise_back(dn, n, r, layer):
    d = dn - n * (dn * n).mean(dim=1, keepdim=True)
    if layer:
        d = d - dn.mean(dim=1, keepdim=True)
    return d * r


def _plain_norm(s):
    c = s["case"]
    x, layer, dtype = s["x"].float(), c["layer"], s["x"].dtype
    b = 0 if s["bias"] is None else s["bias"]
    if c["kind"] == "norm":
        n, r = _normalise(x, layer)
        out = dict(u=(n * s["weight"] + b).to(dtype))
        if c["train"]:
            du = s["du"].float()
            out["dx"] = (s["dy"].float() + _normalise_back(du * s["weight"], n, r, layer)).to(dtype)
            out["dweight"] = (du * n).sum(0)
            out["dbias"] = du.sum(0) if c["bias"] else None
        return out
    run, G = _run(c), s["gate"].shape[0]
    gate = s["gate"].repeat_interleave(run, dim=0)[:c["M"]]
    n, r = _normalise(s["h"].float(), layer)
    post = n * s["weight"] + b
    y = (s["scale"] * x + gate * post).to(dtype)
    nn, rn = _normalise(y.float(), layer)
    nb = 0 if s["next_bias"] is None else s["next_bias"]
    out = dict(y=y, u=(nn * s["next_weight"] + nb).to(dtype))
    if c["train"]:
        du = s["du"].float()
        d = s["dy"].float() + _normalise_back(du * s["next_weight"], nn, rn, layer)
        out["dx"] = (s["scale"] * d).to(dtype)
        out["dh"] = _normalise_back(d * gate * s["weight"], n, r, layer).to(dtype)
        out["dweight"] = (d * gate * n).sum(0)
        out["dbias"] = (d * gate).sum(0) if c["bias"] else None
        dg = torch.nn.functional.pad(d * post, (0, 0, 0, G * run - c["M"]))
        out["dgate"] = dg.view(G, run, c["C"]).sum(1)
        out["dnext_weight"] = (du * nn).sum(0)
        out["dnext_bias"] = du.sum(0) if c["bias"] else None
    return out


def _plain(s):
    c = s["case"]
    if c["kind"] in ("norm", "block"):
        return _plain_norm(s)
    x, dtype = s["x"], s["x"].dtype
    if c["kind"] == "pack":
        seed = s["seed"] if c["stochastic"] else None
        out = [_four(x, seed).to(dtype)]
        if c["both"]:
            out.append(_four(x.t(), seed, True).to(dtype))
        return out
    w = s["weights"] if c["kind"] == "linear" else _four(s["w"])
    z = _four(x) @ w.t() + s["bias"].float()
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    y = y.to(dtype)
    if c["kind"] == "linear":
        return y
    dz = s["dy"].float()
    if c["act"] == "relu":
        dz = torch.where(z.to(dtype) > 0, dz, 0.0)
    dx = _four(dz, s["seed"]) @ _four(s["w"].t()).t()
    dw = _four(dz.t(), s["seed"], True) @ _four(x.t()).t()
    return dict(y=y, dx=dx.to(dtype), dw=dw, dbias=dz.sum(0).to(dtype))


# ------------------------------------------------------------------ the library's operators

def _own_norm(s, B):
    c = s["case"]
    kind = B.RTN_NORM_LAYER if c["layer"] else B.RTN_NORM_RMS
    if c["kind"] == "norm":
        out = dict(u=B.norm(s["x"], s["weight"], bias=s["bias"], kind=kind, eps=EPS))
        if c["train"]:
            out["dx"], out["dweight"], out["dbias"] = B.norm_backward(s["du"], s["x"], s["weight"], kind=kind, eps=EPS,
                                                                      dx_add=s["dy"], want_dbias=c["bias"])
        return out
    y, u = B.block_norm(s["h"], s["x"], s["weight"], bias=s["bias"], gate=s["gate"], gate_run=_run(c), scale=s["scale"],
                        next_weight=s["next_weight"], next_bias=s["next_bias"], kind=kind, eps=EPS)
    out = dict(y=y, u=u)
    if c["train"]:
        names = ("dh", "dx", "dweight", "dbias", "dgate", "dnext_weight", "dnext_bias")
        out.update(zip(names, B.block_norm_backward(s["dy"], s["h"], s["weight"], bias=s["bias"], gate=s["gate"], gate_run=_run(c),
                                                    scale=s["scale"], du=s["du"], y=y, next_weight=s["next_weight"], kind=kind,
                                                    eps=EPS, want_dbias=c["bias"], want_dnext_bias=c["bias"])))
    return out


def _own(s):
    from paper_1912_02057_amd import binding as B
    c = s["case"]
    if c["kind"] in ("norm", "block"):
        return _own_norm(s, B)
    x, M, K = s["x"], c["M"], c["K"]
    if c["kind"] == "pack":
        seed = s["seed"] if c["stochastic"] else None
        if not c["both"]:
            return [B.mx4_unpack(B.mx4_pack(x, seed=seed), M, K, x.dtype)]
        p, pt = B.mx4_pack(x, seed=seed, transposed=True)
        return [B.mx4_unpack(p, M, K, x.dtype), B.mx4_unpack(pt, K, M, x.dtype)]
    N, act = c["N"], {"none": B.RTN_ACT_NONE, "relu": B.RTN_ACT_RELU, "gelu": B.RTN_ACT_GELU, "silu": B.RTN_ACT_SILU}[c["act"]]
    if c["kind"] == "linear":
        return B.mx4_linear(x, s["weights"], N, bias=s["bias"], act=act, residual=s["residual"])
    w, wt = B.mx4_pack(s["w"], transposed=True)
    x4, xt = B.mx4_pack(x, transposed=True)
    z = torch.empty((M, N), dtype=x.dtype, device=x.device) if c["act"] != "none" else None
    y = B.mx4_linear(x, w, N, bias=s["bias"], act=act, residual=s["residual"], x_packed=x4, z_out=z)
    dx, dw, dbias = B.mx4_linear_backward(s["dy"], wt, K, xt, act=act, z=z, seed=s["seed"], dw_dtype=torch.float32)
    return dict(y=y, dx=dx, dw=dw, dbias=dbias)


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    c = case
    M = c["M"]
    if c["kind"] in ("norm", "block"):
        C = c["C"]
        tensors = {("norm", False): 2, ("norm", True): 5, ("block", False): 4, ("block", True): 8}[c["kind"], c["train"]]
        vectors = {("norm", False): 1, ("norm", True): 2, ("block", False): 2 + c.get("G", 0), ("block", True): 4 + 2 * c.get("G", 0)}
        return {"bytes": 2 * tensors * M * C + 4 * vectors[c["kind"], c["train"]] * C * (2 if c["bias"] else 1), "flops": 0}
    K = c["K"]
    if c["kind"] == "pack":  # read, kept in 4.25 bits, read again, given back
        size, ways = (4 if c["dtype"] == "fp32" else 2), (2 if c["both"] else 1)
        return {"bytes": M * K * (size + ways * (17 / 16 + size)), "flops": 0}
    N = c["N"]
    bytes_ = 2 * M * K + 2 * M * N * (2 if c["residual"] else 1) + 2 * N
    if c["kind"] == "linear":  # 4.25 bits of a weight
        return {"bytes": bytes_ + N * K * 17 / 32, "flops": 2 * M * N * K}
    return {"bytes": bytes_ + 4 * N * K + 2 * M * N + 2 * M * K + 4 * N * K + 2 * N, "flops": 6 * M * N * K}


# ------------------------------------------------------------------ the definition, in 64 bits

_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _product_words(a, b):
    """(high, low) 32-bit words of a * b, b a number below 2^32, from 16-bit limbs."""
    a0, a1, b0, b1 = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
    mid = a1 * b0 + ((a0 * b0) >> 16)
    mid2 = a0 * b1 + (mid & 0xFFFF)
    return a1 * b1 + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | ((a0 * b0) & 0xFFFF)


def _random16(rows, groups, seed, transposed):
    """[rows * groups, 32] random numbers of a packing; the seed as a Python number."""
    keys = [seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32]
    n = torch.arange(rows * groups, device=DEV)
    out = torch.empty((rows * groups, 32), dtype=torch.int32, device=DEV)
    for j in range(4):
        x = [n % 2 ** 32, n // 2 ** 32, torch.full_like(n, j), torch.full_like(n, 1 if transposed else 0)]
        for turn in range(10):
            k = [(keys[0] + turn * 0x9E3779B9) % 2 ** 32, (keys[1] + turn * 0xBB67AE85) % 2 ** 32]
            h0, l0 = _product_words(x[0], 0xD2511F53)
            h2, l2 = _product_words(x[2], 0xCD9E8D57)
            x = [h2 ^ x[1] ^ k[0], l2, h0 ^ x[3] ^ k[1], l0]
        for w in range(4):
            out[:, 8 * j + 2 * w] = (x[w] % 65536).int()
            out[:, 8 * j + 2 * w + 1] = (x[w] // 65536).int()
    return out


def _exact_four(v, seed=None, transposed=False):
    """Q(v) of a 64-bit matrix."""
    rows, cols = v.shape
    groups = -(-cols // 32)
    full = torch.zeros((rows, 32 * groups), dtype=torch.float64, device=DEV)
    full[:, :cols] = v
    full = full.reshape(-1, 32)
    rnd = None if seed is None else _random16(rows, groups, seed, transposed)
    for i in range(0, full.shape[0], 1 << 20):
        p = full[i:i + (1 << 20)]
        a = p.abs().max(dim=1, keepdim=True).values
        e = torch.where(a > 0, torch.floor(torch.log2(torch.where(a > 0, a, 1.0))), torch.full_like(a, -200.0))
        e = torch.where((a > 0) & (torch.exp2(e) > a), e - 1, e)
        e = torch.where(torch.exp2(e + 1) <= a, e + 1, e)
        e = (e - 2).clamp(min=-127)
        if seed is not None:
            e = torch.where(a > 6 * torch.exp2(e), e + 1, e)
        unit = torch.exp2(e)
        r = p.abs() / unit
        q = torch.zeros_like(r)
        for n in range(1, 8):
            lo, hi = _GRID[n - 1], _GRID[n]
            if seed is None:  # past the middle, or on it where the upper code is the even one
                up = (r > (lo + hi) / 2) | ((r == (lo + hi) / 2) & (n % 2 == 0))
            else:
                up = (r >= hi) | ((r > lo) & (rnd[i:i + (1 << 20)] < (r - lo) / (hi - lo) * 65536))
            q = torch.where(up, hi, q)
        full[i:i + (1 << 20)] = q * unit * torch.sign(p)
    return full.view(rows, -1)[:, :cols]


def _exact_norm(s):
    c = s["case"]
    layer = c["layer"]

    def forward(v, w, b):
        if layer:
            v = v - v.mean(1, keepdim=True)
        r = (v.pow(2).mean(1, keepdim=True) + EPS).rsqrt()
        return v * r, r, v * r * w + (0 if b is None else b)

    def backward(du, w, n, r):
        d = du * w
        inner = d - n * (d * n).mean(1, keepdim=True)
        return r * (inner - d.mean(1, keepdim=True) if layer else inner)

    d64 = {k: v.double() for k, v in s.items() if torch.is_tensor(v)}
    x, w, b = d64["x"], d64["weight"], d64.get("bias")
    if c["kind"] == "norm":
        n, r, u = forward(x, w, b)
        out = dict(u=u)
        if c["train"]:
            out["dx"] = d64["dy"] + backward(d64["du"], w, n, r)
            out["dweight"] = (d64["du"] * n).sum(0)
            out["dbias"] = d64["du"].sum(0) if c["bias"] else None
        return out
    owner = torch.arange(c["M"], device=DEV) // _run(c)
    gate = d64["gate"][owner]
    n, r, post = forward(d64["h"], w, b)
    y = s["scale"] * x + gate * post
    kept = y.to(s["x"].dtype).double()  # what the next norm reads
    nn, rn, u = forward(kept, d64["next_weight"], d64.get("next_bias"))
    out = dict(y=y, u=u)
    if c["train"]:
        du = d64["du"]
        d = d64["dy"] + backward(du, d64["next_weight"], nn, rn)
        out["dx"] = s["scale"] * d
        out["dh"] = backward(d * gate, w, n, r)
        out["dweight"] = (d * gate * n).sum(0)
        out["dbias"] = (d * gate).sum(0) if c["bias"] else None
        out["dgate"] = torch.zeros_like(d64["gate"]).index_add_(0, owner, d * post)
        out["dnext_weight"] = (du * nn).sum(0)
        out["dnext_bias"] = du.sum(0) if c["bias"] else None
    return out


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] in ("norm", "block"):
        return _exact_norm(s)
    x, key = s["x"].double(), int(s["seed"])
    if c["kind"] == "pack":
        key = key if c["stochastic"] else None
        out = [_exact_four(x, key)]
        if c["both"]:
            out.append(_exact_four(x.t().contiguous(), key, True))
        return out
    if c["kind"] == "train":
        w = s["w"].double()
    else:  # the weights before their packing, made again from the seed
        g = torch.Generator(device=DEV)
        g.manual_seed(int(seed) & 0x7FFFFFFF)
        _activations(c["M"], c["K"], DTYPES[c["dtype"]], g)
        torch.randint(-2 ** 62, 2 ** 62, (1,), generator=g, device=DEV)
        w = (torch.randn((c["N"], c["K"]), generator=g, device=DEV) / math.sqrt(c["K"])).double()
    act = c["act"]
    z = torch.addmm(s["bias"].double(), _exact_four(x), _exact_four(w).t())
    cdf = torch.special.ndtr if act == "gelu" else torch.sigmoid
    y = {"none": lambda: z.clone(), "relu": lambda: z.relu(), "gelu": lambda: z * cdf(z), "silu": lambda: z * cdf(z)}[act]()
    if s["residual"] is not None:
        y += s["residual"].double()
    if c["kind"] == "linear":
        return y
    dz = s["dy"].double()
    if act == "relu":
        dz[z.to(s["x"].dtype) <= 0] = 0
    dx = _exact_four(dz, key) @ _exact_four(w.t().contiguous()).t().contiguous()
    dw = _exact_four(dz.t().contiguous(), key, True) @ _exact_four(x.t().contiguous()).t().contiguous()
    return dict(y=y, dx=dx, dw=dw, dbias=dz.sum(0))
