"""The operators of a decoder block on 4-bit weights with group scales, as a program that answers with such a model, or that
sends gradients through it, calls them.

  quantise     4-bit codes and group scales of a float32 weight matrix
  matmul       y = x W^T, one token to a long prompt, activations in bfloat16 or in e4m3 with one scale a token
  matmul_dx    dx = dy W, the gradient to the input
  glu          silu(x Wg^T) * (x Wu^T), both projections, activation and product
  glu_back     its backward pass: gradients to the input and to both projections' results (the weights are frozen)
  norm         residual's addition, root-mean-square norm, output in e4m3 with one scale a token
  norm_back    gradients to the input and to the norm's weight

Format of the weights.  A group is `group` neighbouring columns of a row.  Its scale s is the least number of 5 significant bits
that is not below max |w| / 7 (at least 2^-126; 0 for a group of zeros), its codes are w / s rounded to whole numbers, ties to even.
Codes are kept in blocks of 16 rows x 128 columns, 64 x 4 words: word k of place (c, r) holds row r, columns 32 k + 8 c + 0..7; in it,
for b = 0..3, the size of column b's code is in bits 8 b.. 8 b + 2 and its sign in bit 8 b + 7, that of column 4 + b in bits
8 b + 4 .. 8 b + 6 and in bit 8 ((b + 1) % 4) + 3.  Scales: [groups][rows].  Rows and columns that fill the last block are 0.

Inputs stand in for what such programs hold: weights = a narrow normal core with 0.5 % wide outliers, activations = normal
values with 1 % of the columns 20 times larger, gradients = normal values, small.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

EPS = 1e-5
_CTX = None


def _ctx():
    """The process's context: a program keeps one for all its layers."""
    global _CTX
    if _CTX is None:
        import paper_2412_04180_amd as skim

        _CTX = skim.Context(0)
    return _CTX


def listed():
    return [
        # a small layer: launches and latency count
        dict(name="quantise_512x512_g32", kind="quantise", n=512, m=512, group=32),
        # a gate or up projection
        dict(name="quantise_11008x4096_g128", kind="quantise", n=11008, m=4096, group=128),
        # the down projection while answering: one token
        dict(name="matmul_1x4096x11008", kind="matmul", tokens=1, n=4096, m=11008, group=128, x="bf16", y="bf16"),
        # several requests together on a layer whose sizes no tile divides; results in float32
        dict(name="matmul_17x1021x2999_e4m3", kind="matmul", tokens=17, n=1021, m=2999, group=64, x="e4m3", y="f32"),
        # the down projection of a prompt
        dict(name="matmul_2048x4096x11008", kind="matmul", tokens=2048, n=4096, m=11008, group=128, x="bf16", y="bf16"),
        # gradients through the down projection
        dict(name="matmul_dx_1024x4096x11008", kind="matmul_dx", tokens=1024, n=4096, m=11008, group=128, y="bf16"),
        # gate and up projections while answering: one token, then a prompt, from the norm's 8-bit output
        dict(name="glu_1x11008x4096_e4m3", kind="glu", tokens=1, n=11008, m=4096, group=128, x="e4m3"),
        dict(name="glu_512x11008x4096_e4m3", kind="glu", tokens=512, n=11008, m=4096, group=128, x="e4m3"),
        # gradients through the gated block, its input kept in 8 bits
        dict(name="glu_back_1024x11008x4096_e4m3", kind="glu_back", tokens=1024, n=11008, m=4096, group=128, x="e4m3"),
        # the norm while answering, and of a batch of prompts
        dict(name="norm_1x4096", kind="norm", tokens=1, m=4096, x="bf16"),
        dict(name="norm_8192x4096", kind="norm", tokens=8192, m=4096, x="bf16"),
        # gradients through the norm
        dict(name="norm_back_4096x4096", kind="norm_back", tokens=4096, m=4096, x="bf16"),
    ]


def _size(rng, lo, hi):
    """A size spread evenly over its logarithm; half of them multiples of 128, the others as they fall."""
    v = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
    if rng.random() < 0.5 and v >= 128:
        v = v // 128 * 128
    return min(hi, max(lo, v))


def draw(rng):
    kind = rng.choice(["quantise", "matmul", "matmul", "matmul_dx", "glu", "glu", "glu_back", "norm", "norm_back"])
    if kind == "norm":
        return dict(kind=kind, tokens=_size(rng, 1, 8192), m=_size(rng, 64, 8192), x=rng.choice(["bf16", "bf16", "f32"]))
    if kind == "norm_back":
        return dict(kind=kind, tokens=_size(rng, 1, 4096), m=_size(rng, 64, 8192), x=rng.choice(["bf16", "bf16", "f32"]))
    c = dict(kind=kind, n=_size(rng, 256, 11008), m=_size(rng, 256, 11008), group=rng.choice([32, 64, 128, 128]))
    while c["n"] * c["m"] > 11008 * 4096:
        c["n"], c["m"] = (c["n"] + 1) // 2, (c["m"] + 1) // 2
    if kind == "quantise":
        return c
    c["tokens"] = _size(rng, 1, 1024 if kind == "glu_back" else 2048)
    if kind in ("matmul", "glu", "glu_back"):
        c["x"] = rng.choice(["bf16", "e4m3"])
    if kind in ("matmul", "matmul_dx"):
        c["y"] = rng.choice(["bf16", "bf16", "f32"])
    return c


# ---- the format, in elementary operations -----------------------------------------------------------------------

def _scale5(top):
    """The least number of 5 significant bits >= top / 7, at least 2^-126; 0 for 0.  float64 in and out."""
    t = top / torch.full_like(top, 7.0)                          # (by a tensor: divided, not multiplied by the reciprocal)
    kept = (t.view(torch.int64) + ((1 << 48) - 1)) >> 48 << 48   # sign, exponent and 4 bits, rounded up
    return torch.where(top > 0, kept.view(torch.float64).clamp_min(2.0 ** -126), torch.zeros_like(t))


def _blocks(v, n16, m128):
    """[n, m] filled up with zeros to whole blocks."""
    return torch.nn.functional.pad(v, (0, m128 - v.shape[1], 0, n16 - v.shape[0]))


def _quantise(W, group):
    """Codes in the layout above (int32 words) and scales (bfloat16) of a float32 matrix."""
    n, m = W.shape
    n16, m128 = -(-n // 16) * 16, -(-m // 128) * 128
    Wp = _blocks(W, n16, m128)
    top = Wp.view(n16, m128 // group, group).abs().amax(2)
    s = _scale5(top.double())
    q = torch.round(Wp.view(n16, m128 // group, group).double() / torch.where(s > 0, s, torch.ones_like(s))[:, :, None])
    q = q.to(torch.int32).view(n16, m128)
    f = q.abs() | ((q < 0).to(torch.int32) << 3)                 # sign and size in four bits
    # row block, row, column block, word, c, half, b  ->  row block, column block, c, row, word, half, b
    f = f.view(n16 // 16, 16, m128 // 128, 4, 4, 2, 4).permute(0, 2, 4, 1, 3, 5, 6)
    b = torch.arange(4, device=W.device, dtype=torch.int32)
    size, sign = f & 7, f >> 3
    words = ((size[..., 0, :] << (8 * b)) | (sign[..., 0, :] << (8 * b + 7))
             | (size[..., 1, :] << (8 * b + 4)) | (sign[..., 1, :] << (8 * ((b + 1) % 4) + 3)))
    words = words[..., 0] | words[..., 1] | words[..., 2] | words[..., 3]
    return words.reshape(-1).contiguous(), s.t().contiguous().to(torch.bfloat16)


def _weights(w):
    """The float32 matrix that a packed one stands for."""
    n, m, group = w["n"], w["m"], w["group"]
    nb, mb = -(-n // 16), -(-m // 128)
    words = w["codes"].view(nb, mb, 4, 16, 4, 1)
    b = torch.arange(4, device=words.device, dtype=torch.int32)
    first = ((words >> (8 * b)) & 7) * (1 - 2 * ((words >> (8 * b + 7)) & 1))
    second = ((words >> (8 * b + 4)) & 7) * (1 - 2 * ((words >> (8 * ((b + 1) % 4) + 3)) & 1))
    q = torch.stack((first, second), 5)                          # row block, column block, c, row, word, half, b
    q = q.permute(0, 3, 1, 4, 2, 5, 6).reshape(nb * 16, mb * 128 // group, group)
    return (q.float() * w["scales"].float().t()[:, :, None]).view(nb * 16, mb * 128)[:n, :m]


def _e4m3(v):
    """float64 numbers of at most 448 in size, rounded to e4m3 (ties to even); float64."""
    e = ((v.view(torch.int64) >> 52) & 2047).clamp_min(1023 - 6) - 3          # of the last place that is kept
    step = (e << 52).view(torch.float64)
    return torch.round(v / step) * step


def _token_scales(y):
    """One scale a row: max |y| / 448 in float32, 1 for a row of zeros."""
    top = y.abs().amax(1)
    s = (top / 448.0).float().clamp_min(2.0 ** -126)
    return torch.where(top > 0, s, torch.ones_like(s))


# ---- inputs -----------------------------------------------------------------------------------------------------

def _dense(gen, n, m):
    W = torch.randn((n, m), device="cuda", generator=gen) * 0.02
    wide = torch.rand((n, m), device="cuda", generator=gen) < 0.005
    return torch.where(wide, W * 10.0, W)


def _packed(gen, case):
    n, m, group = case["n"], case["m"], case["group"]
    codes, scales = _quantise(_dense(gen, n, m), group)
    return dict(codes=codes, scales=scales, n=n, m=m, group=group)


def _columns(gen, m):
    scale = torch.ones(m, device="cuda")
    scale[torch.randperm(m, device="cuda", generator=gen)[: max(1, m // 100)]] = 20.0
    return scale


def _activations(gen, tokens, m, kind):
    """(x, scales): bfloat16 or float32 and None, or e4m3 and one scale a token."""
    x = torch.randn((tokens, m), device="cuda", generator=gen) * _columns(gen, m)
    if kind == "f32":
        return x, None
    if kind == "bf16":
        return x.to(torch.bfloat16), None
    s = _token_scales(x.double())
    return _e4m3(x.double() / s.double()[:, None]).float().to(torch.float8_e4m3fn), s


def _gradient(gen, tokens, n, kind="bf16"):
    g = torch.randn((tokens, n), device="cuda", generator=gen) * 1e-3
    return g.to(torch.bfloat16) if kind == "bf16" else g


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    kind = case["kind"]
    st = dict(case=case)
    if kind == "quantise":
        st["W"] = _dense(gen, case["n"], case["m"])
        return st
    T, m = case["tokens"], case["m"]
    if kind in ("norm", "norm_back"):
        st["weight"] = 1.0 + 0.1 * torch.randn(m, device="cuda", generator=gen)
        st["x"], _ = _activations(gen, T, m, case["x"])
        st["residual"], _ = _activations(gen, T, m, case["x"])
        if kind == "norm_back":
            st["dy"], st["dh"] = _gradient(gen, T, m, case["x"]), _gradient(gen, T, m, case["x"])
            st["rstd"] = torch.rsqrt(st["x"].double().square().mean(1) + EPS).float()
        return st
    st["w"] = _packed(gen, case)
    if kind == "matmul_dx":
        st["dy"] = _gradient(gen, T, case["n"])
        return st
    if kind != "matmul":
        st["up"] = _packed(gen, case)
    st["x"], st["x_scales"] = _activations(gen, T, m, case["x"])
    if kind == "glu_back":
        st["da"] = _gradient(gen, T, case["n"])
    return st


# ---- one pass ---------------------------------------------------------------------------------------------------

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def run(st):
    c = st["case"]
    kind = c["kind"]
    if own:
        ctx = _ctx()
        if kind == "quantise":
            w = ctx.group_quantize(st["W"], group=c["group"])
            return dict(codes=w["codes"], scales=w["scales"])
        if kind == "matmul":
            return ctx.group_matmul(st["w"], st["x"], x_scales=st["x_scales"], out_dtype=_TYPES[c["y"]])
        if kind == "matmul_dx":
            return ctx.group_matmul_dx(st["w"], st["dy"], out_dtype=_TYPES[c["y"]])
        if kind == "glu":
            return ctx.group_glu(st["w"], st["up"], st["x"], x_scales=st["x_scales"])
        if kind == "glu_back":
            return ctx.group_glu_backward(st["w"], st["up"], st["x"], st["da"], x_scales=st["x_scales"])
        if kind == "norm":
            o = ctx.rms_norm(st["x"], st["weight"], residual=st["residual"], eps=EPS)
            return dict(h=o["h"], q=o["q"], scales=o["scales"], rstd=o["rstd"])
        return ctx.rms_norm_backward(st["dy"], st["x"], st["rstd"], st["weight"], dh=st["dh"])
    if kind == "quantise":
        codes, scales = _quantise(st["W"], c["group"])
        return dict(codes=codes, scales=scales)
    if kind == "norm":
        h = (st["x"].float() + st["residual"].float()).to(st["x"].dtype)
        hd = h.double()
        rstd = torch.rsqrt(hd.square().mean(1) + torch.tensor(EPS, dtype=torch.float32).double().item())
        y = hd * st["weight"].double() * rstd[:, None]
        s = _token_scales(y)
        q = _e4m3((y / s.double()[:, None]).clamp(-448.0, 448.0))
        return dict(h=h, q=q.float().to(torch.float8_e4m3fn), scales=s, rstd=rstd.float())
    if kind == "norm_back":
        dy, hat = st["dy"].float(), st["x"].float() * st["rstd"][:, None]
        g = dy * st["weight"]
        dx = st["rstd"][:, None] * (g - hat * (g * hat).mean(1, keepdim=True)) + st["dh"].float()
        return dict(dx=dx.to(st["dy"].dtype), dweight=(dy * hat).sum(0))
    if kind == "matmul_dx":
        return (st["dy"].float() @ _weights(st["w"])).to(_TYPES[c["y"]])
    x = st["x"].float()
    if st["x_scales"] is not None:
        x = x * st["x_scales"][:, None]
    if kind == "matmul":
        return (x @ _weights(st["w"]).t()).to(_TYPES[c["y"]])
    Wg, Wu = _weights(st["w"]), _weights(st["up"])
    g, u = x @ Wg.t(), x @ Wu.t()
    sig = 1.0 / (1.0 + torch.exp(-g))
    if kind == "glu":
        return (g * sig * u).to(torch.bfloat16)
    da = st["da"].float()
    dg, du = da * u * sig * (1.0 + g * (1.0 - sig)), da * g * sig
    return dict(dx=(dg @ Wg + du @ Wu).to(torch.bfloat16), dgate=dg.to(torch.bfloat16), dup=du.to(torch.bfloat16))


def work(case):
    kind, m = case["kind"], case["m"]
    if kind in ("norm", "norm_back"):
        b, tm = 2 if case["x"] == "bf16" else 4, case["tokens"] * m
        if kind == "norm":
            return dict(bytes=tm * (3 * b + 1) + 8 * case["tokens"] + 4 * m, flops=8 * tm)
        return dict(bytes=tm * 4 * b + 4 * case["tokens"] + 8 * m, flops=12 * tm)
    n = case["n"]
    w = n * m / 2 + 2 * n * m / case["group"]
    if kind == "quantise":
        return dict(bytes=4 * n * m + w, flops=4 * n * m)
    T = case["tokens"]
    xb = T * m * (1 if case.get("x") == "e4m3" else 2) + (4 * T if case.get("x") == "e4m3" else 0)
    yb = 2 if case.get("y", "bf16") == "bf16" else 4
    if kind == "matmul":
        return dict(bytes=w + xb + T * n * yb, flops=2 * T * n * m)
    if kind == "matmul_dx":
        return dict(bytes=w + T * n * 2 + T * m * yb, flops=2 * T * n * m)
    if kind == "glu":
        return dict(bytes=2 * w + xb + T * n * 2, flops=4 * T * n * m)
    return dict(bytes=2 * w + xb + 3 * T * n * 2 + T * m * 2, flops=8 * T * n * m)


# ---- the definition in 64 bits ----------------------------------------------------------------------------------

def _dense64(w):
    """W from the words, code by code: float64 [n, m]."""
    n, m = w["n"], w["m"]
    mb = -(-m // 128)
    i = torch.arange(n, device="cuda")[:, None]
    j = torch.arange(m, device="cuda")[None, :]
    k = j % 128
    word = (((i // 16) * mb + j // 128) * 64 + (k % 32) // 8 * 16 + i % 16) * 4 + k // 32
    bits = w["codes"].long()[word]
    b, high = k % 4, (k % 8) // 4
    size = (bits >> (8 * b + 4 * high)) & 7
    sign = (bits >> torch.where(high > 0, 8 * ((b + 1) % 4) + 3, 8 * b + 7)) & 1
    return torch.where(sign > 0, -size, size).double() * w["scales"].double()[j // w["group"], i]


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantise":
        n, m, G = case["n"], case["m"], case["group"]
        n16, groups = (n + 15) // 16 * 16, (m + 127) // 128 * 128 // G
        least = np.zeros((groups, n16))
        for g in range((m + G - 1) // G):
            f, e = np.frexp(st["W"][:, g * G:(g + 1) * G].abs().max(1).values.cpu().numpy().astype(np.float64) / 7)
            least[g, :n] = np.ldexp(np.ceil(f * 32), e - 5)
        return dict(codes=None, scales=torch.from_numpy(least).cuda())
    if kind == "norm":
        h = (st["x"].double() + st["residual"].double()).to(st["x"].dtype).double()
        rms = torch.sqrt((h * h).sum(1) / case["m"] + EPS)
        return dict(h=h, q=None, scales=(h * st["weight"].double()).abs().max(1).values / rms / 448, rstd=1 / rms)
    if kind == "norm_back":
        dy, h, r = st["dy"].double(), st["x"].double(), st["rstd"].double()[:, None]
        a = dy * st["weight"].double()
        inner = (a * h).sum(1, keepdim=True) / case["m"]
        return dict(dx=r * a - r ** 3 * h * inner + st["dh"].double(), dweight=(dy * h * r).sum(0))
    W = _dense64(st["w"])
    if kind == "matmul_dx":
        return torch.matmul(st["dy"].double(), W)
    x = st["x"].double()
    if st["x_scales"] is not None:
        x = st["x_scales"].double()[:, None] * x
    g = torch.matmul(x, W.t())
    if kind == "matmul":
        return g
    U = _dense64(st["up"])
    u = torch.matmul(x, U.t())
    p = torch.sigmoid(g)
    if kind == "glu":
        return u * g * p
    da = st["da"].double()
    dg, du = da * u * (p + g * p * (1 - p)), da * g * p
    return dict(dx=torch.matmul(dg, W) + torch.matmul(du, U), dgate=dg, dup=du)
