"""The operators of a residual block trained and served in 8-bit floating point, each through the public entry points:

  gemm     the product of two tensors of 8-bit floating-point codes (e4m3 or e5m2) with a power-of-two scale for each
           block of 128 along the reduction, each operand either way round: 128 to 8192 in each direction, the outer
           extent of an operand also odd
  serve    a linear layer with its weights kept as codes (one scale for each 128 x 128 block): the activation is
           quantised (one scale for each row's 128 columns) and multiplied; 1 to 8192 rows, 128 to 8192 features
  train    forward and backward of that layer: the fp32 weights, the activation and the gradient quantised (the last two
           along their rows and along their columns), then y = x w^T, dx = g w and dw = g^T x; 16 to 8192 rows
  norm     the join between two blocks: r = alpha x + gate * dropout(norm(b) w_post), h = norm(r) w_pre, forward alone or
           with its backward; a gate per channel or per group of rows, with and without dropout; 1 to 32768 rows, 64 to 8192 columns
  dropout  y = x / (1 - p) where the element's draw keeps it, else 0, on its own: 1 K to 128 M elements

Values: activations ~N(0,1) with a few channels ten times as large, as a residual stream has them; weights
Kaiming-uniform; gradients ~N(0, 1e-2)."""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

E4M3, E5M2 = "e4m3", "e5m2"
_MAX = {E4M3: 448.0, E5M2: 57344.0}
_BITS = {E4M3: (3, -6), E5M2: (2, -14)}                 # mantissa bits, exponent of the smallest normal value
_F8 = {E4M3: torch.float8_e4m3fn, E5M2: torch.float8_e5m2}
_T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def listed():
    return [
        # one token of a generated text through a square projection: the weights' bytes and latency
        dict(name="serve_token", kind="serve", m=1, n=4096, k=4096, type="bf16"),
        # a few requests through the odd classifier of the linear benchmark
        dict(name="serve_batch_odd", kind="serve", m=77, n=1008, k=2048, type="f32"),
        # a long prompt of ragged length through a widening projection
        dict(name="serve_prompt", kind="serve", m=5001, n=8192, k=4096, type="bf16"),
        # the product alone, at the largest size of the dense sweep
        dict(name="gemm_8192", kind="gemm", m=8192, n=8192, k=8192, ta=False, tb=True, fa=E4M3, fb=E4M3, type="f32"),
        # a training step of a wide layer over a full minibatch of tokens
        dict(name="train_8192", kind="train", m=8192, n=4096, k=4096, type="bf16", fg=E4M3),
        # a training step of a small layer: ragged rows, odd features, gradients in the wider format
        dict(name="train_odd", kind="train", m=1111, n=1520, k=1024, type="f32", fg=E5M2),
        # the join at one token: latency
        dict(name="norm_token", kind="norm", rows=1, c=4096, stream="bf16", type="bf16", gate_rows=0, p=0.0, alpha=1.0, back=False),
        # the join in training, fp32 residual stream between bf16 blocks
        dict(name="norm_train", kind="norm", rows=16384, c=4096, stream="f32", type="bf16", gate_rows=0, p=0.1, alpha=1.0, back=True),
        # a gate per sequence, odd rows and columns
        dict(name="norm_groups_odd", kind="norm", rows=6 * 333, c=1000, stream="f32", type="f32", gate_rows=333, p=0.0, alpha=0.5, back=True),
        # dropout of the smallest layer's output: launch and latency
        dict(name="dropout_small", kind="dropout", count=64 * 256, type="f32", p=0.5),
        # of an odd number of half-precision elements
        dict(name="dropout_odd", kind="dropout", count=12345677, type="f16", p=0.25),
        # of a full minibatch of hidden activations
        dict(name="dropout_large", kind="dropout", count=16384 * 8192, type="bf16", p=0.1),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _mult(rng, lo, hi, step):
    return int(min(hi, max(lo, step * round(_log(rng, lo, hi) / step))))


_MOST_FLOPS = 2.0 * 8192 ** 3


def draw(rng):
    kind = rng.choice(("gemm", "serve", "serve", "train", "train", "norm", "norm", "dropout"))
    if kind == "gemm":
        ta, tb = rng.random() < 0.5, rng.random() < 0.5
        m, n, k = (_mult(rng, 128, 8192, 16) for _ in range(3))
        # an extent that is no operand's innermost one may be odd
        m = m if ta else min(8192, m + rng.randrange(16))
        n = min(8192, n + rng.randrange(16)) if tb else n
        k = min(8192, k + rng.randrange(16)) if ta and not tb else k
        return dict(kind=kind, m=m, n=n, k=k, ta=ta, tb=tb, fa=rng.choice((E4M3, E5M2)), fb=E4M3, type=rng.choice(("f32", "bf16", "f16")))
    if kind == "serve":
        m = int(_log(rng, 1, 64.9)) if rng.random() < 0.5 else int(_log(rng, 65, 8192.9))
        return dict(kind=kind, m=m, n=_mult(rng, 128, 8192, 16), k=_mult(rng, 128, 8192, 16), type=rng.choice(("f32", "bf16", "bf16", "f16")))
    if kind == "train":
        while True:
            m, n, k = int(_log(rng, 16, 8192.9)), _mult(rng, 128, 8192, 16), _mult(rng, 128, 8192, 16)
            if 6.0 * m * n * k <= _MOST_FLOPS:
                return dict(kind=kind, m=m, n=n, k=k, type=rng.choice(("f32", "bf16")), fg=rng.choice((E4M3, E5M2)))
    if kind == "norm":
        while True:
            rows, c = int(_log(rng, 1, 32768.9)), int(_log(rng, 64, 8192.9))
            c = c if rng.random() < 0.3 else max(64, c // 64 * 64)
            if rows * c <= 16384 * 4096:
                break
        back = rng.random() < 0.7
        groups = rng.choice((0, 0, 1, 3, 8))
        gate_rows = 0 if groups == 0 else max(1, rows // groups)
        return dict(kind=kind, rows=rows, c=c, stream=rng.choice(("f32", "bf16")), type=rng.choice(("f32", "bf16", "bf16", "f16")),
                    gate_rows=gate_rows, p=rng.choice((0.0, 0.1, 0.3)), alpha=rng.choice((1.0, 0.5)), back=back)
    return dict(kind=kind, count=int(_log(rng, 1024, 16384 * 8192)), type=rng.choice(("f32", "bf16", "f16")), p=rng.choice((0.1, 0.25, 0.5)))


# ------------------------------------------------------------------------- inputs
def _normal(g, shape, std, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _activation(g, rows, c, dtype):
    x = torch.randn((rows, c), generator=g, device="cuda")
    x[:, torch.randint(0, c, (max(1, c // 256),), generator=g, device="cuda")] *= 10.0
    return x.to(dtype)


def _weight(g, n, k):
    b = math.sqrt(6.0 / k)
    return torch.rand((n, k), generator=g, device="cuda") * (2.0 * b) - b


def _pack(exps, rows, kb):
    """Exponents [rows, kb] of a tensor's blocks as the products take them: a byte (exponent + 127) for each row and block, in
    512-byte pieces of 128 rows x 4 blocks, the bytes of rows r, r + 32, r + 64, r + 96 side by side."""
    rt, kg = (rows + 127) // 128, (kb + 3) // 4
    full = torch.full((rt * 128, kg * 4), 127, dtype=torch.uint8, device=exps.device)
    full[:rows, :kb] = (exps + 127).to(torch.uint8)
    return full.view(rt, 4, 32, kg, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _codes_in_hand(x, fmt, along, square=False):
    """A tensor as it lies in a user's memory after an earlier call: codes (as x), exponents of the blocks along dimension
    `along` (their rows first), and the packed scales."""
    e = _exponents(x.float(), fmt, along, square)
    rows = x.shape[1 - along]
    spread = e.repeat_interleave(128, 1)[:, : x.shape[along]]
    v = torch.ldexp(x.float(), -(spread if along else spread.t()))
    return v.to(_F8[fmt]).view(torch.uint8), e, _pack(e, rows, e.shape[1])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    kind = case["kind"]
    if kind == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        a = _activation(g, *((k, m) if case["ta"] else (m, k)), torch.float32)
        b = _weight(g, n, k) if case["tb"] else _weight(g, k, n)
        s["a"], s["ea"], s["sa"] = _codes_in_hand(a, case["fa"], 0 if case["ta"] else 1)
        s["b"], s["eb"], s["sb"] = _codes_in_hand(b, case["fb"], 1 if case["tb"] else 0)
    elif kind == "serve":
        s["x"] = _activation(g, case["m"], case["k"], _T[case["type"]])
        s["w"], s["ew"], s["sw"] = _codes_in_hand(_weight(g, case["n"], case["k"]), E4M3, 1, square=True)
    elif kind == "train":
        s["x"] = _activation(g, case["m"], case["k"], _T[case["type"]])
        s["w"] = _weight(g, case["n"], case["k"])
        s["g"] = _normal(g, (case["m"], case["n"]), 1e-2, _T[case["type"]])
    elif kind == "norm":
        rows, c = case["rows"], case["c"]
        s["x"] = _activation(g, rows, c, _T[case["stream"]])
        s["b"] = _normal(g, (rows, c), 0.5, _T[case["type"]])
        s["w_post"], s["w_pre"] = (1.0 + _normal(g, (c,), 0.1) for _ in range(2))
        s["gate"] = 0.5 + _normal(g, (1 if not case["gate_rows"] else -(-rows // case["gate_rows"]), c), 0.1)
        s["seed"] = seed * 2654435761 % (1 << 62)
        if case["back"]:
            s["dr"] = _normal(g, (rows, c), 1e-2, _T[case["stream"]])
            s["dh"] = _normal(g, (rows, c), 1e-2, _T[case["type"]])
    else:
        s["x"] = _normal(g, (case["count"],), 1.0, _T[case["type"]])
        s["seed"] = seed * 2654435761 % (1 << 62)
    return s


# ------------------------------------------------------------------- plain forms
def _amax(x, along, square):
    """Largest magnitude of each block of 128 along `along`, [other extent, blocks]; the same over 128 x 128 blocks if square."""
    a = (x if along else x.t()).abs()
    rows, k = a.shape
    a = torch.nn.functional.pad(a, (0, -k % 128)).view(rows, -1, 128).amax(2)
    if square:
        b = torch.nn.functional.pad(a, (0, 0, 0, -rows % 128)).view(-1, 128, a.shape[1]).amax(1)
        a = b.repeat_interleave(128, 0)[:rows]
    return a


def _exponents(x, fmt, along, square=False):
    """The smallest e with amax <= max * 2^e (0 for a block of zeros, at least -127)."""
    a = _amax(x, along, square)
    mant, e = torch.frexp(a)                                        # a = mant * 2^e, mant in [0.5, 1)
    top = 8 if fmt == E4M3 else 15                                  # both formats end at 1.75 * 2^top
    e = e - 1 - top + (mant > 0.875).int()
    return torch.where(a == 0, torch.zeros_like(e), e).clamp(min=-127)


def _rounded(v, fmt):
    """v to the nearest value of the format, ties to even."""
    bits, low = _BITS[fmt]
    _, e = torch.frexp(v)
    step = (e - 1).clamp(min=low) - bits
    return torch.ldexp(torch.round(torch.ldexp(v, -step)), step).clamp(-_MAX[fmt], _MAX[fmt])


def _values(x, fmt, along, square=False):
    """What the codes of x stand for."""
    x = x.float()
    e = _exponents(x, fmt, along, square).repeat_interleave(128, 1)[:, : x.shape[along]]
    e = e if along else e.t()
    return torch.ldexp(_rounded(torch.ldexp(x, -e), fmt), e)


def _decoded(q, e, fmt, along):
    v = q.view(_F8[fmt]).float()
    e = e.repeat_interleave(128, 1)[:, : q.shape[along]]
    return torch.ldexp(v, e if along else e.t())


def _mul_hi_lo(a, b):
    """High and low words of the product of a 32-bit constant and 32-bit words held in int64."""
    a0, a1 = a & 0xFFFF, a >> 16
    low = b * a0                                                    # < 2^48
    high = b * a1 + (low >> 16)                                     # < 2^49
    return high >> 16, ((high & 0xFFFF) << 16) | (low & 0xFFFF)


def _draws(count, seed, tensor_id):
    """The 16-bit draws of elements 0 .. count - 1: eight from each Philox4x32-10 block."""
    i = torch.arange((count + 7) // 8, device="cuda", dtype=torch.int64)
    c = [i & 0xFFFFFFFF, i >> 32, torch.full_like(i, tensor_id), torch.full_like(i, 0xFFFFFFFF)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for r in range(10):
        h0, l0 = _mul_hi_lo(0xD2511F53, c[0])
        h1, l1 = _mul_hi_lo(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ ((k0 + r * 0x9E3779B9) & 0xFFFFFFFF), l1, h0 ^ c[3] ^ ((k1 + r * 0xBB67AE85) & 0xFFFFFFFF), l0]
    w = torch.stack(c, 1)
    return torch.stack((w & 0xFFFF, w >> 16), 2).view(-1)[:count]


def _threshold(p):
    return int(math.floor(p * 65536.0 + 0.5))


def _keep(shape, p, seed, tensor_id):
    """Factors of a dropout: 1 / (1 - p) (p in steps of 2^-16) where kept, else 0."""
    t = _threshold(p)
    d = _draws(math.prod(shape), seed, tensor_id).view(shape)
    return torch.where(d >= t, 65536.0 / (65536 - t), 0.0)


def _spread(gate, s):
    """The gate of each row."""
    if not s["gate_rows"]:
        return gate
    return gate.repeat_interleave(s["gate_rows"], 0)[: s["rows"]]


def _norm_plain(s):
    x, b, w1, w2 = s["x"].float(), s["b"].float(), s["w_post"], s["w_pre"]
    gate = _spread(s["gate"], s)
    keep = _keep(b.shape, s["p"], s["seed"], 3) if s["p"] else 1.0
    rstd1 = torch.rsqrt((b * b).mean(1, keepdim=True) + EPS)
    bh = b * rstd1
    d = bh * w1 * keep
    r = (s["alpha"] * x + gate * d).to(s["x"].dtype)
    rf = r.float()
    rstd2 = torch.rsqrt((rf * rf).mean(1, keepdim=True) + EPS)
    rh = rf * rstd2
    out = dict(r=r, h=(rh * w2).to(s["b"].dtype), rstd_post=rstd1.view(-1), rstd_pre=rstd2.view(-1))
    if not s["back"]:
        return out
    dh = s["dh"].float()
    t = dh * w2
    dR = s["dr"].float() + rstd2 * (t - rh * (t * rh).mean(1, keepdim=True))
    dn = dR * gate * keep
    t1 = dn * w1
    db = rstd1 * (t1 - bh * (t1 * bh).mean(1, keepdim=True))
    dgate = dR * d
    n = s["gate"].shape[0]
    if s["gate_rows"]:
        pad = n * s["gate_rows"] - s["rows"]
        dgate = torch.nn.functional.pad(dgate, (0, 0, 0, pad)).view(n, s["gate_rows"], -1)
    else:
        dgate = dgate[None]
    out.update(dx=(s["alpha"] * dR).to(s["x"].dtype), db=db.to(s["b"].dtype), dw_post=(dn * bh).sum(0), dgate=dgate.sum(1), dw_pre=(dh * rh).sum(0))
    return out


def _plain(s):
    kind = s["kind"]
    if kind == "gemm":
        a = _decoded(s["a"], s["ea"], s["fa"], 0 if s["ta"] else 1)
        b = _decoded(s["b"], s["eb"], s["fb"], 1 if s["tb"] else 0)
        return ((a.t() if s["ta"] else a) @ (b.t() if s["tb"] else b)).to(_T[s["type"]])
    if kind == "serve":
        return (_values(s["x"], E4M3, 1) @ _decoded(s["w"], s["ew"], E4M3, 1).t()).to(_T[s["type"]])
    if kind == "train":
        w = _values(s["w"], E4M3, 1, square=True)
        y = _values(s["x"], E4M3, 1) @ w.t()
        dx = _values(s["g"], s["fg"], 1) @ w
        dw = _values(s["g"], s["fg"], 0).t() @ _values(s["x"], E4M3, 0)
        return dict(y=y.to(s["x"].dtype), dx=dx.to(s["x"].dtype), dw=dw)
    if kind == "norm":
        return _norm_plain(s)
    x = s["x"].float()
    return (x * _keep(x.shape, s["p"], s["seed"], 3)).to(s["x"].dtype)


# ---------------------------------------------------------- the framework's calls
def _kernels(s):
    from paper_1805_11046_b200 import binding as B

    fmt = {E4M3: B.QBP_E4M3, E5M2: B.QBP_E5M2}
    kind = s["kind"]
    if kind == "gemm":
        return B.qbp_gemm_f8(s["a"], s["sa"], s["b"], s["sb"], transA=s["ta"], transB=s["tb"], formatA=fmt[s["fa"]], formatB=fmt[s["fb"]],
                             out_dtype=_T[s["type"]])
    if kind == "serve":
        return B.qbp_linear_f8(s["x"], s["w"], s["sw"])
    if kind == "train":
        f = fmt[s["fg"]]
        wq, sw, swt = B.qbp_quantize_f8_square(s["w"])
        xq, sx, xqt, sxt = B.qbp_quantize_f8(s["x"], cols=True)
        y = B.qbp_gemm_f8(xq, sx, wq, sw, transB=True, out_dtype=s["x"].dtype)
        gq, sg, gqt, sgt = B.qbp_quantize_f8(s["g"], format=f, cols=True)
        dx = B.qbp_gemm_f8(gq, sg, wq, swt, formatA=f, out_dtype=s["x"].dtype)
        dw = B.qbp_gemm_f8(gqt, sgt, xqt, sxt, transA=True, formatA=f)
        return dict(y=y, dx=dx, dw=dw)
    if kind == "norm":
        d = B.resnorm_desc(s["x"], s["b"], alpha=s["alpha"], eps=EPS, gate_rows=s["gate_rows"], p=s["p"], seed=s["seed"], tensor_id=3)
        r, h, rstd1, rstd2 = B.qbp_resnorm_fwd(d, s["x"], s["b"], s["w_post"], s["gate"], s["w_pre"])
        out = dict(r=r, h=h, rstd_post=rstd1, rstd_pre=rstd2)
        if s["back"]:
            dx, db, dw1, dgate, dw2 = B.qbp_resnorm_bwd(d, s["dr"], s["dh"], s["b"], r, rstd1, rstd2, s["w_post"], s["gate"], s["w_pre"])
            out.update(dx=dx, db=db, dw_post=dw1, dgate=dgate, dw_pre=dw2)
        return out
    return B.qbp_dropout(s["x"], s["p"], s["seed"], tensor_id=3)


def run(state):
    if own:
        return _kernels(state)
    return _plain(state)


# ------------------------------------------------------------------------ in 64 bits
def _exact_values(x, fmt, along, square=False):
    """What the codes stand for, by the definition: per block, the power of two that just brings the largest value into range."""
    x = (x if along else x.t()).double()
    rows, k = x.shape
    high = 128 if square else 1
    full = torch.zeros((-(-rows // high) * high, -(-k // 128) * 128), dtype=torch.float64, device=x.device)
    full[:rows, :k] = x
    blocks = full.view(-1, high, full.shape[1] // 128, 128)
    largest = blocks.abs().amax((1, 3), keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(largest / _MAX[fmt])))
    scale = torch.where(largest * 1.0 > _MAX[fmt] * scale, scale * 2, torch.where(largest <= _MAX[fmt] * scale / 2, scale / 2, scale))
    scale = torch.where(largest == 0, torch.ones_like(scale), scale.clamp(min=2.0 ** -127))
    v = ((blocks / scale).float().to(_F8[fmt]).double() * scale).reshape(full.shape)[:rows, :k]
    return v if along else v.t()


def _exact_keep(shape, p, seed):
    """The dropout's factors, its generator in unsigned 64-bit words on the host."""
    count = math.prod(shape)
    t = _threshold(p)
    n = (count + 7) // 8
    out = np.empty((n, 8), dtype=bool)
    low32 = np.uint64(0xFFFFFFFF)
    for at in range(0, n, 1 << 20):
        i = np.arange(at, min(n, at + (1 << 20)), dtype=np.uint64)
        x0, x1, x2, x3 = i & low32, i >> np.uint64(32), np.full_like(i, 3), np.full_like(i, 0xFFFFFFFF)
        key0, key1 = seed & 0xFFFFFFFF, seed >> 32
        for _ in range(10):
            p0, p1 = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
            x0, x1, x2, x3 = (p1 >> np.uint64(32)) ^ x1 ^ np.uint64(key0), p1 & low32, (p0 >> np.uint64(32)) ^ x3 ^ np.uint64(key1), p0 & low32
            key0, key1 = (key0 + 0x9E3779B9) & 0xFFFFFFFF, (key1 + 0xBB67AE85) & 0xFFFFFFFF
        words = np.stack((x0, x1, x2, x3), 1).astype(np.uint32)
        out[at: at + len(i)] = words.view(np.uint16) >= t
    keep = torch.from_numpy(out.reshape(-1)[:count]).cuda().view(shape)
    return keep.double() * (65536.0 / (65536 - t))


def _exact_norm(s):
    """The join and its gradients by the chain rule, row by row in 64 bits; r is what is stored of it."""
    rows, c = s["rows"], s["c"]
    x, b = s["x"].double(), s["b"].double()
    w1, w2 = s["w_post"].double(), s["w_pre"].double()
    group = torch.arange(rows, device="cuda") // (s["gate_rows"] or rows)
    g = s["gate"].double()[group]
    m = _exact_keep((rows, c), s["p"], s["seed"]) if s["p"] else torch.ones_like(b)
    q1 = 1.0 / torch.sqrt(torch.einsum("rc,rc->r", b, b) / c + EPS)
    d = m * w1 * b * q1[:, None]
    r = s["alpha"] * x + g * d
    y = r.to(s["x"].dtype).double()
    q2 = 1.0 / torch.sqrt(torch.einsum("rc,rc->r", y, y) / c + EPS)
    out = dict(r=r, h=w2 * y * q2[:, None], rstd_post=q1, rstd_pre=q2)
    if s["back"]:
        dh = s["dh"].double()
        u = dh * w2
        total = s["dr"].double() + u * q2[:, None] - y * (q2 ** 3 * torch.einsum("rc,rc->r", u, y) / c)[:, None]
        v = total * g * m
        z = v * w1
        out["dx"] = s["alpha"] * total
        out["db"] = z * q1[:, None] - b * (q1 ** 3 * torch.einsum("rc,rc->r", z, b) / c)[:, None]
        out["dw_post"] = torch.einsum("rc,rc,r->c", v, b, q1)
        out["dgate"] = torch.zeros_like(s["gate"], dtype=torch.float64).index_add_(0, group, total * d)
        out["dw_pre"] = torch.einsum("rc,rc,r->c", dh, y, q2)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "gemm":
        def value(q, e, fmt, along):
            scale = torch.exp2(e.double()).repeat_interleave(128, 1)[:, : q.shape[along]]
            return q.view(_F8[fmt]).double() * (scale if along else scale.t())
        a, b = value(s["a"], s["ea"], s["fa"], 0 if s["ta"] else 1), value(s["b"], s["eb"], s["fb"], 1 if s["tb"] else 0)
        return torch.matmul(a.t() if s["ta"] else a, b.t() if s["tb"] else b)
    if kind == "serve":
        w = s["w"].view(_F8[E4M3]).double() * torch.exp2(s["ew"].double()).repeat_interleave(128, 1)[:, : case["k"]]
        return torch.matmul(_exact_values(s["x"], E4M3, 1), w.t())
    if kind == "train":
        w = _exact_values(s["w"], E4M3, 1, square=True)
        return dict(y=torch.matmul(_exact_values(s["x"], E4M3, 1), w.t()), dx=torch.matmul(_exact_values(s["g"], s["fg"], 1), w),
                    dw=torch.matmul(_exact_values(s["g"], s["fg"], 0).t(), _exact_values(s["x"], E4M3, 0)))
    if kind == "norm":
        return _exact_norm(s)
    return s["x"].double() * _exact_keep((case["count"],), case["p"], s["seed"])


def work(case):
    kind = case["kind"]
    if kind == "dropout":
        return {"bytes": 2.0 * _SIZE[case["type"]] * case["count"], "flops": float(case["count"])}
    if kind == "norm":
        n, st, bl = float(case["rows"] * case["c"]), _SIZE[case["stream"]], _SIZE[case["type"]]
        small = 4.0 * case["c"] * (2 + (1 if not case["gate_rows"] else -(-case["rows"] // case["gate_rows"]))) + 8.0 * case["rows"]
        fwd = 2 * n * (st + bl) + small
        # the backward reads both gradients, b and r, and writes both gradients
        return {"bytes": fwd + (n * (3 * st + 3 * bl) + 2 * small if case["back"] else 0.0), "flops": n * (34 if case["back"] else 12)}
    m, n, k = case["m"], case["n"], case["k"]
    e = _SIZE[case["type"]]
    if kind == "gemm":
        return {"bytes": (1 + 1 / 128) * (m * k + n * k) + float(e) * m * n, "flops": 2.0 * m * n * k}
    if kind == "serve":
        return {"bytes": float(e) * (m * k + m * n) + (1 + 1 / 16384) * n * k, "flops": 2.0 * m * n * k}
    # x, w, g in; y, dx, dw out
    return {"bytes": e * (2.0 * m * k + 2.0 * m * n) + 8.0 * n * k, "flops": 6.0 * m * n * k}
