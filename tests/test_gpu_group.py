"""4-bit weights with group scales, the products with them, and the norm that makes their 8-bit input, against plain
implementations in float64 on the CPU.

Tolerances.  u = half a step of the result's type, relative: 2^-8 for bfloat16, 2^-24 for float32.  The products' operands are exact, so a
result differs from the formula's by one rounding (u |y|) and by what the float32 sums lose: each addition is off by at most 2^-24 of
a partial sum, partial sums are at most A = sum |x_j w_j|, and no order of k additions loses more than k 2^-24 A.  Additions do not all
fall one after the other (32 columns enter a matrix instruction at once, the sums of wavefronts are added at the end): LOSS below, 2^-24 (m / 8 + 64), stays
ahead of that by a factor of two and more, and the scale's product and the sum's add two roundings a group, counted by the same bound.
An 8-bit input adds one product with the token's scale: 2 roundings more.
"""
import ctypes as C

import numpy as np
import pytest
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


# ---- the format and the formulas, plainly ---------------------------------------------------------------------------

def quantise(W, group):
    """(codes int [n, m], scales float64 [n, groups]) of a float32 matrix, entry by entry of the definition."""
    n, m = W.shape
    groups = -(-m // group)
    q, s = np.zeros((n, m), np.int64), np.zeros((n, groups))
    for g in range(groups):
        w = W[:, g * group:(g + 1) * group].astype(np.float64)
        f, e = np.frexp(np.abs(w).max(1) / 7.0)
        s[:, g] = np.where(f > 0, np.maximum(np.ldexp(np.ceil(f * 32), e - 5), 2.0 ** -126), 0.0)
        q[:, g * group:(g + 1) * group] = np.rint(w / np.where(s[:, g] > 0, s[:, g], 1.0)[:, None])
    return q, s


def dense(q, s, group):
    return q * np.repeat(s, group, axis=1)[:, :q.shape[1]]


def pack(q, s, group):
    """Words and scales in the documented layout, code by code."""
    n, m = q.shape
    rb, cb = -(-n // 16), -(-m // 128)
    words = np.zeros(rb * cb * 256, np.uint32)
    i, j = np.meshgrid(np.arange(n), np.arange(m), indexing="ij")
    k = j % 128
    at = ((i // 16) * cb + j // 128) * 256 + 4 * (16 * ((k % 32) // 8) + i % 16) + k // 32
    b, high = k % 4, (k % 8) // 4
    size, sign = np.abs(q).astype(np.uint32), (q < 0).astype(np.uint32)
    bits = np.where(high, size << (8 * b + 4) | sign << (8 * ((b + 1) % 4) + 3), size << (8 * b) | sign << (8 * b + 7)).astype(np.uint32)
    np.bitwise_or.at(words, at.ravel(), bits.ravel())
    sc = np.zeros((cb * 128 // group, rb * 16), np.float32)
    sc[:s.shape[1], :n] = s.T
    return torch.from_numpy(words.view(np.int32)), torch.from_numpy(sc).to(torch.bfloat16)


def e4m3(v):
    """float64 rounded to e4m3, ties to even."""
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e, -5) - 4)
    return np.rint(v / step) * step


def silu(g):
    return g / (1.0 + np.exp(-g))


def dsilu(g):
    p = 1.0 / (1.0 + np.exp(-g))
    return p * (1.0 + g * (1.0 - p))


def weights(rng, n, m):
    W = rng.standard_normal((n, m)) * 0.02
    return np.where(rng.random((n, m)) < 0.005, W * 10, W).astype(np.float32)


def matrix(rng, n, m, group):
    """(what the calls take, on the GPU; the dense float64 matrix)."""
    q, s = quantise(weights(rng, n, m), group)
    codes, scales = pack(q, s, group)
    return dict(codes=codes.cuda(), scales=scales.cuda(), n=n, m=m, group=group), dense(q, s, group)


def inputs(rng, T, m, kind, ld=None, offset=0):
    """(x on the GPU, its scales, what they stand for in float64): rows of `ld` values, the tensor `offset` values into its memory.  Whatever
    lies between the rows is NaN."""
    ld = m if ld is None else ld
    x = rng.standard_normal((T, m)) * np.where(rng.random(m) < 0.01, 20.0, 1.0)
    if kind == "bf16":
        v, s = torch.from_numpy(x).to(torch.bfloat16), None
        value = v.double().numpy()
    else:
        s = np.maximum(np.abs(x).max(1), 1e-3).astype(np.float32) / np.float32(448)
        v = torch.from_numpy(np.clip(e4m3(x / s[:, None].astype(np.float64)), -448, 448)).float().to(torch.float8_e4m3fn)
        value = v.double().numpy() * s[:, None].astype(np.float64)
        s = torch.from_numpy(s).cuda()
    size = v.element_size()
    mem = torch.full(((T * ld + offset + 16) * size,), 0x7F, dtype=torch.uint8)        # (0x7F: a NaN of e4m3)
    if kind == "bf16":
        mem.view(torch.int16).fill_(0x7FC0)
    mem = mem.cuda().view(v.dtype)
    out = mem.as_strided((T, m), (ld, 1), offset)
    out.view(torch.int16 if size == 2 else torch.uint8).copy_(v.view(torch.int16 if size == 2 else torch.uint8).cuda())
    return out, s, value


def gradient(rng, T, n):
    g = torch.from_numpy(rng.standard_normal((T, n)) * 1e-2).to(torch.bfloat16)
    return g.cuda(), g.double().numpy()


def loss(k):
    return 2.0 ** -24 * (k / 8 + 64)


def close(got, want, allowed, what):
    got = got.detach().cpu().double().numpy()
    assert got.shape == want.shape, what
    over = np.abs(got - want) - allowed
    assert np.all(np.isfinite(got)) and np.all(over <= 0), f"{what}: {np.nanmax(over)} over at {np.unravel_index(np.nanargmax(over), over.shape)}"


# ---- CPU: sizes and refusals ------------------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def lib():
    import os

    import paper_2412_04180_amd as skim

    if not os.path.exists(skim.LIB_PATH):
        from paper_2412_04180_amd import _build

        _build.build()
    return skim.load_library()


def test_sizes_of_the_format(lib):
    for n, m in ((1, 1), (16, 128), (17, 129), (4096, 11008), (1021, 2999)):
        rb, cb = -(-n // 16), -(-m // 128)
        assert lib.skim_group_code_words(n, m) == rb * cb * 256
        for group in (32, 64, 128):
            assert lib.skim_group_scale_entries(n, m, group) == rb * 16 * cb * (128 // group)
    for n, m in ((0, 4), (4, 0), (-1, 4), ((1 << 24) + 1, 4), (4, (1 << 24) + 1)):
        assert lib.skim_group_code_words(n, m) == -1
        assert lib.skim_group_scale_entries(n, m, 128) == -1
    for group in (0, 16, 48, 256, -32):
        assert lib.skim_group_scale_entries(64, 64, group) == -1


def test_sizes_past_the_reach_of_a_copy_are_refused(lib):
    most = 1 << 23                                       # a tile's last row begins 127 rows of 2 bytes a value behind its first: below 2^31
    assert lib.skim_group_code_words(most, 1) == most // 16 * 256 and lib.skim_group_scale_entries(1, most, 64) == 16 * most // 64
    for n, m in ((most + 1, 4), (4, most + 1), (1 << 24, 4), (4, 1 << 24)):
        assert lib.skim_group_code_words(n, m) == -1 and lib.skim_group_scale_entries(n, m, 32) == -1


def test_calls_without_a_context_are_refused(lib):
    assert lib.skim_group_quantize(None, None, 1, 1, 1, 128, None, None) == -1
    assert lib.skim_group_unpack(None, None, None, 1, 1, 128, None) == -1
    assert lib.skim_group_matmul(None, None, None, 1, 1, 128, None, 1, 1, None, 1, None, 1, None, 0) == -1
    assert lib.skim_group_matmul_dx(None, None, None, 1, 1, 128, None, 1, 1, None, 1, None, 0) == -1
    assert lib.skim_group_glu(None, None, None, None, None, 1, 1, 128, None, 1, 1, None, 1, None, 1, None, 0) == -1
    assert lib.skim_group_glu_backward(None, None, None, None, None, 1, 1, 128, None, 1, 1, None, 1, None, 1, None, None, None, 1, None, 0) == -1
    assert lib.skim_rms_norm(None, None, 1, None, 0, 1, None, 1e-6, 1, 1, None, None, None, None, None) == -1
    assert lib.skim_rms_norm_backward(None, None, 1, None, 1, None, 0, 1, None, None, 1, 1, None, None, None, 0) == -1
    assert lib.skim_rms_norm_scratch_bytes(None, 4, 4) == 0


@pytest.mark.parametrize("group", [32, 64, 128])
def test_the_definition_keeps_its_promises(group):
    """Of the format itself: no code above 7, errors of half a step, products of code and scale exact in bfloat16, words that take
    apart into the codes."""
    rng = np.random.default_rng(group)
    W = weights(rng, 37, 333)
    W[3] = 0
    W[5, :40] = np.float32(1e-42)
    W[6] *= np.float32(2.0) ** 100
    q, s = quantise(W, group)
    D = dense(q, s, group)
    assert np.abs(q).max() == 7 and not q[3].any()
    step = np.repeat(s, group, axis=1)[:, :333]
    assert np.all(np.abs(W.astype(np.float64) - D) <= step / 2)
    assert np.array_equal(torch.from_numpy(D).to(torch.bfloat16).double().numpy(), D)
    words, scales = pack(q, s, group)
    w = words.numpy().view(np.uint32)
    byte = np.concatenate([np.frombuffer((w & 0x87878787).astype("<u4").tobytes(), np.uint8).reshape(-1, 4),
                           np.frombuffer((((w >> 4) | (w << 28)) & 0x87878787).astype("<u4").tobytes(), np.uint8).reshape(-1, 4)], axis=1)
    assert byte.shape == (w.size, 8) and np.all((byte & 7) <= 7)
    value = torch.from_numpy(byte.copy()).view(torch.float8_e4m3fn).double().numpy() * 512
    i, j = np.meshgrid(np.arange(37), np.arange(333), indexing="ij")
    k = j % 128
    at = ((i // 16) * 3 + j // 128) * 256 + 4 * (16 * ((k % 32) // 8) + i % 16) + k // 32
    assert np.array_equal(value[at, k % 8], q)


# ---- GPU ----------------------------------------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def ctx(gpu_lib):
    c = gpu_lib.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


SHAPES = [(1, 1, 32), (16, 128, 128), (17, 129, 64), (5, 31, 32), (48, 96, 32), (100, 1000, 128), (257, 513, 64), (1021, 2999, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("n,m,group", SHAPES)
@pytest.mark.parametrize("pad", [0, 3])
def test_quantize_and_unpack(ctx, n, m, group, pad):
    rng = np.random.default_rng(n * 1000 + m + pad)
    W = weights(rng, n, m)
    if n > 4:
        W[1] = 0                                               # no scale
        W[2] = np.float32(1e-44)                               # below the least scale
        W[3] = rng.integers(-7, 8, m) * np.float32(0.5)        # whole steps
        W[4] = (rng.integers(-13, 14, m) + np.float32(0.5)) * np.float32(0.25)     # ties
    store = torch.full((n, m + pad), float("nan"), device="cuda")
    store[:, :m] = torch.from_numpy(W).cuda()
    gq = ctx.group_quantize(store[:, :m], group=group)
    q, s = quantise(W, group)
    codes, scales = pack(q, s, group)
    assert torch.equal(gq["codes"].cpu(), codes)
    assert torch.equal(gq["scales"].cpu().view(torch.int16), scales.view(torch.int16))
    Wq = ctx.group_unpack(gq)
    assert np.array_equal(Wq.cpu().double().numpy(), dense(q, s, group))


@pytest.mark.gpu
def test_quantize_of_large_and_small_weights(ctx):
    rng = np.random.default_rng(8)
    W = (rng.standard_normal((64, 256)) * np.exp2(rng.integers(-140, 120, (64, 1)))).astype(np.float32)
    gq = ctx.group_quantize(torch.from_numpy(W).cuda(), group=64)
    q, s = quantise(W, 64)
    assert torch.equal(gq["codes"].cpu(), pack(q, s, 64)[0])
    assert np.array_equal(ctx.group_unpack(gq).cpu().double().numpy(), dense(q, s, 64))


PRODUCTS = [(1, 1, 1, 32), (1, 16, 128, 128), (1, 300, 1000, 64), (2, 17, 129, 32), (15, 33, 96, 32), (16, 64, 512, 128), (17, 50, 513, 64),
            (33, 129, 640, 128), (64, 256, 256, 32), (65, 100, 384, 64), (130, 272, 1100, 128), (300, 513, 520, 128), (129, 130, 5000, 64), (70, 2100, 300, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,n,m,group", PRODUCTS)
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_matmul(ctx, T, n, m, group, kind):
    rng = np.random.default_rng(T * 7 + n * 3 + m)
    gq, W = matrix(rng, n, m, group)
    for ld, offset in ((m, 0), (m + 5, 3)):
        x, s, value = inputs(rng, T, m, kind, ld, offset)
        want, size = value @ W.T, np.abs(value) @ np.abs(W).T
        for dtype in (torch.float32, torch.bfloat16):
            y = ctx.group_matmul(gq, x, x_scales=s, out_dtype=dtype)
            close(y, want, U[dtype] * np.abs(want) * 1.01 + loss(m) * size, f"{dtype} ld={ld}")


@pytest.mark.gpu
@pytest.mark.parametrize("T,n,m,group", PRODUCTS)
def test_matmul_dx(ctx, T, n, m, group):
    rng = np.random.default_rng(T * 5 + n * 3 + m)
    gq, W = matrix(rng, n, m, group)
    for ld, offset in ((n, 0), (n + 5, 3)):
        dy, _, value = inputs(rng, T, n, "bf16", ld, offset)
        want, size = value @ W, np.abs(value) @ np.abs(W)
        for dtype in (torch.float32, torch.bfloat16):
            dx = ctx.group_matmul_dx(gq, dy, out_dtype=dtype)
            close(dx, want, U[dtype] * np.abs(want) * 1.01 + loss(n) * size, f"{dtype} ld={ld}")


def glu_errors(value, Wg, Wu, m):
    """g, u and how far the float32 ones may be off."""
    g, u = value @ Wg.T, value @ Wu.T
    return g, u, loss(m) * (np.abs(value) @ np.abs(Wg).T), loss(m) * (np.abs(value) @ np.abs(Wu).T)


@pytest.mark.gpu
@pytest.mark.parametrize("T,n,m,group", PRODUCTS)
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_glu(ctx, T, n, m, group, kind):
    """The result's error: |silu'| <= 1.1 times g's, times |u|; |silu| times u's; a rounding of the type; and 8 roundings of float32 for the
    activation (the exponential's argument loses at most |g| 2^-24 of itself, below 100 of them counted)."""
    rng = np.random.default_rng(T * 11 + n * 3 + m)
    (gate, Wg), (up, Wu) = matrix(rng, n, m, group), matrix(rng, n, m, group)
    x, s, value = inputs(rng, T, m, kind, m + 8, 0)
    g, u, eg, eu = glu_errors(value, Wg, Wu, m)
    want = silu(g) * u
    for dtype in (torch.float32, torch.bfloat16):
        a = ctx.group_glu(gate, up, x, x_scales=s, out_dtype=dtype)
        allowed = 1.1 * eg * np.abs(u) + np.abs(silu(g)) * eu + 1.1 * eg * eu + (U[dtype] * 1.01 + (8 + np.minimum(np.abs(g), 100)) * 2.0 ** -24) * np.abs(want)
        close(a, want, allowed, str(dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("T,n,m,group", PRODUCTS)
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_glu_backward(ctx, T, n, m, group, kind):
    """dgate: |silu''| <= 0.5 times g's error.  dx: up to 64 tokens of two bfloat16 pieces of dgate and dup, 2^-16 of them off; of more tokens it is made
    of them as stored, and against those has the error of a product."""
    rng = np.random.default_rng(T * 13 + n * 3 + m)
    (gate, Wg), (up, Wu) = matrix(rng, n, m, group), matrix(rng, n, m, group)
    x, s, value = inputs(rng, T, m, kind)
    da, dav = gradient(rng, T, n)
    o = ctx.group_glu_backward(gate, up, x, da, x_scales=s)
    g, u, eg, eu = glu_errors(value, Wg, Wu, m)
    few = U[torch.bfloat16] * 1.01 + (8 + np.minimum(np.abs(g), 100)) * 2.0 ** -24
    dg, du = dav * u * dsilu(g), dav * silu(g)
    # (dsilu is a sum that cancels near its zero: its own roundings count against 1 + |g|)
    edg = np.abs(dav) * (1.1 * eu + 0.5 * eg * (np.abs(u) + eu) + 16 * 2.0 ** -24 * (1 + np.abs(g)) * np.abs(u))
    edu = np.abs(dav) * 1.1 * eg
    close(o["dgate"], dg, edg + few * np.abs(dg), "dgate")
    close(o["dup"], du, edu + few * np.abs(du), "dup")
    if T <= 64:
        fine = few - U[torch.bfloat16] * 1.01 + 2.0 ** -16
        off = (edg + fine * np.abs(dg)) @ np.abs(Wg) + (edu + fine * np.abs(du)) @ np.abs(Wu)
    else:
        dg, du, off = o["dgate"].cpu().double().numpy(), o["dup"].cpu().double().numpy(), 0.0
    want = dg @ Wg + du @ Wu
    size = np.abs(dg) @ np.abs(Wg) + np.abs(du) @ np.abs(Wu)
    close(o["dx"], want, U[torch.bfloat16] * 1.01 * (np.abs(want) + off) + off + loss(4 * n) * 1.01 * size, "dx")


@pytest.mark.gpu
def test_glu_backward_agrees_with_differences(ctx):
    """d sum(a da) along a direction, from float32 results either side of x (bfloat16 steps are exact there)."""
    rng = np.random.default_rng(5)
    T, n, m = 3, 96, 256
    (gate, Wg), (up, Wu) = matrix(rng, n, m, 64), matrix(rng, n, m, 64)
    x = torch.from_numpy(rng.integers(-8, 9, (T, m)) / 8.0).to(torch.bfloat16).cuda()
    v = torch.from_numpy(rng.integers(-1, 2, (T, m)) / 64.0).to(torch.bfloat16).cuda()
    da = torch.from_numpy(rng.standard_normal((T, n))).to(torch.bfloat16).cuda()
    o = ctx.group_glu_backward(gate, up, x, da)
    ahead = ctx.group_glu(gate, up, (x.float() + v.float()).to(torch.bfloat16), out_dtype=torch.float32).double()
    behind = ctx.group_glu(gate, up, (x.float() - v.float()).to(torch.bfloat16), out_dtype=torch.float32).double()
    change = ((ahead - behind) / 2 * da.double()).sum(1)
    slope = (o["dx"].double() * v.double()).sum(1)
    # third derivatives: |a'''| of a step below 0.1 in g and u; bfloat16 of dgate, dup and dx: 3 roundings of the terms' sizes
    size = (o["dx"].double().abs() * v.double().abs()).sum(1) + (da.double().abs() * (ahead - behind).abs()).sum(1)
    assert torch.all((change - slope).abs() <= 3 * 2.0 ** -8 * size + 1e-3), (change, slope, size)


@pytest.mark.gpu
def test_products_repeat_bit_for_bit_and_vectors_are_single_tokens(ctx):
    rng = np.random.default_rng(3)
    gq, W = matrix(rng, 200, 700, 64)
    x, _, _ = inputs(rng, 70, 700, "bf16")
    y = ctx.group_matmul(gq, x)
    assert torch.equal(y, ctx.group_matmul(gq, x))
    assert torch.equal(ctx.group_matmul(gq, x[3]), ctx.group_matmul(gq, x[3:4])[0])
    dy, _ = gradient(rng, 70, 200)
    assert torch.equal(ctx.group_matmul_dx(gq, dy), ctx.group_matmul_dx(gq, dy))


@pytest.mark.gpu
def test_no_tokens_and_rows_behind_the_last(ctx):
    rng = np.random.default_rng(4)
    gq, _ = matrix(rng, 40, 200, 128)
    x, _, _ = inputs(rng, 5, 200, "bf16")
    assert ctx.group_matmul(gq, x[:0]).shape == (0, 40)
    assert ctx.group_glu(gq, gq, x[:0]).shape == (0, 40)
    assert ctx.group_matmul_dx(gq, torch.zeros((0, 40), dtype=torch.bfloat16, device="cuda")).shape == (0, 200)
    assert ctx.rms_norm(x[:0])["q"].shape == (0, 200)
    back = ctx.rms_norm_backward(x[:0], x[:0], torch.zeros(0, device="cuda"))
    assert back["dx"].shape == (0, 200) and not back["dweight"].any()
    whole = torch.full((8, 40), 3.0, dtype=torch.bfloat16, device="cuda")
    ctx.group_matmul(gq, x, out=whole[:5])
    assert torch.all(whole[5:] == 3.0) and not torch.any(whole[:5] == 3.0)
    wide = torch.full((8, 200), 3.0, dtype=torch.bfloat16, device="cuda")
    ctx.group_matmul_dx(gq, gradient(rng, 5, 40)[0], out=wide[:5])
    assert torch.all(wide[5:] == 3.0) and not torch.any(wide[:5] == 3.0)


# ---- norm ---------------------------------------------------------------------------------------------------------------

NORMS = [(1, 1), (1, 7), (3, 64), (5, 129), (2, 1000), (9, 4096), (4, 8200), (2, 11008), (2, 22016), (1, 32768), (600, 72), (600, 1000), (1100, 5000)]


def rows(rng, T, m, dtype, ld=None):
    """[T, m] of dtype on the GPU with row stride ld (NaN between the rows), and its values."""
    ld = m if ld is None else ld
    v = torch.from_numpy(rng.standard_normal((T, m)) * np.where(rng.random(m) < 0.01, 20.0, 1.0)).to(dtype)
    mem = torch.full((T, ld), float("nan"), dtype=dtype, device="cuda")
    mem[:, :m] = v.cuda()
    return mem[:, :m], v.double().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("T,m", NORMS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad", [0, 5])
def test_rms_norm(ctx, T, m, dtype, pad):
    """Everything is the rounding of the formula's value: h and q exactly (the float64 quotient is off by 4 2^-53 at most, and no value of these
    inputs comes that near a border), scales and rstd by a rounding."""
    rng = np.random.default_rng(T + m + pad)
    x, xv = rows(rng, T, m, dtype, m + pad)
    r, rv = rows(rng, T, m, dtype, m + 2 * pad)
    wv = (1 + 0.1 * rng.standard_normal(m)).astype(np.float32)
    eps = float(np.float32(1e-5))
    for residual, weight in ((r, torch.from_numpy(wv).cuda()), (None, None)):
        o = ctx.rms_norm(x, weight, residual=residual, eps=eps, want_y=True)
        h = xv
        if residual is not None:
            h = torch.from_numpy(xv + rv).to(torch.float32).to(dtype).double().numpy()
            assert np.array_equal(o["h"].cpu().double().numpy(), h)
        else:
            assert o["h"] is None
        rstd = 1 / np.sqrt((h * h).mean(1) + eps)
        y = h * (wv.astype(np.float64) if weight is not None else 1.0) * rstd[:, None]
        close(o["rstd"], rstd, 2.0 ** -24 * 1.01 * rstd, "rstd")
        close(o["y"], y, U[dtype] * 1.01 * np.abs(y), "y")
        top = np.abs(y).max(1) / 448
        close(o["scales"], top, 2.0 ** -24 * 1.01 * top, "scales")
        s = o["scales"].cpu().double().numpy()
        assert np.array_equal(o["q"].cpu().double().numpy(), e4m3(np.clip(y / s[:, None], -448, 448)))


@pytest.mark.gpu
def test_rms_norm_of_zeros_of_tiny_and_of_large_values_and_in_place(ctx):
    m = 256
    x = torch.zeros((4, m), device="cuda")
    x[1] = 1e-30
    x[2] = 1e18
    x[3, 5] = -3.0
    o = ctx.rms_norm(x, eps=1e-6, want_y=True)
    assert not o["q"][0].double().any() and o["scales"][0] == 1
    v = x.cpu().double().numpy()
    y = v / np.sqrt((v * v).mean(1, keepdims=True) + float(np.float32(1e-6)))
    close(o["y"], y, 2.0 ** -23 * np.abs(y), "y")
    s = o["scales"].cpu().double().numpy()[:, None]
    assert np.array_equal(o["q"].cpu().double().numpy(), e4m3(np.clip(y / s, -448, 448)))
    a, b = torch.randn((7, m), device="cuda"), torch.randn((7, m), device="cuda")
    ref = ctx.rms_norm(a, residual=b)
    got = ctx.rms_norm(a, residual=b, out=dict(h=b))
    assert got["h"] is b and torch.equal(b, ref["h"]) and torch.equal(got["q"].view(torch.uint8), ref["q"].view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("T,m", NORMS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad", [0, 5])
def test_rms_norm_backward(ctx, T, m, dtype, pad):
    """float32 arithmetic: g, n and their product 3 roundings, the mean m / 8 + 64 of the terms' sizes, dx another 6 and that of its type;
    dweight: T products of 2 roundings added in at most T additions."""
    rng = np.random.default_rng(T * 3 + m + pad)
    dy, dyv = rows(rng, T, m, dtype, m + pad)
    h, hv = rows(rng, T, m, dtype, m + 2 * pad)
    dh, dhv = rows(rng, T, m, dtype, m + pad)
    wv = (1 + 0.1 * rng.standard_normal(m)).astype(np.float32)
    r = (1 / np.sqrt((hv * hv).mean(1) + 1e-5)).astype(np.float32)
    rd, rt = r.astype(np.float64)[:, None], torch.from_numpy(r).cuda()
    f = 2.0 ** -24
    for weight, past in ((torch.from_numpy(wv).cuda(), dh), (None, None)):
        o = ctx.rms_norm_backward(dy, h, rt, weight, dh=past)
        g = dyv * (wv.astype(np.float64) if weight is not None else 1.0)
        n = hv * rd
        mean, size = (g * n).mean(1, keepdims=True), np.abs(g * n).mean(1, keepdims=True)
        dx = rd * (g - n * mean) + (dhv if past is not None else 0.0)
        terms = rd * (np.abs(g) + np.abs(n) * size) + (np.abs(dhv) if past is not None else 0.0)
        close(o["dx"], dx, U[dtype] * 1.01 * np.abs(dx) + 10 * f * terms + rd * np.abs(n) * f * (m / 8 + 64) * size, "dx")
        close(o["dweight"], (dyv * n).sum(0), f * (T + 4) * np.abs(dyv * n).sum(0), "dweight")
        again = ctx.rms_norm_backward(dy, h, rt, weight, dh=past)
        assert torch.equal(again["dx"], o["dx"]) and torch.equal(again["dweight"], o["dweight"])
        assert ctx.rms_norm_backward(dy, h, rt, weight, dh=past, want_dweight=False)["dweight"] is None


@pytest.mark.gpu
def test_rms_norm_backward_agrees_with_differences(ctx):
    rng = np.random.default_rng(12)
    m = 96
    x, w = rng.standard_normal((2, m)), 1 + 0.1 * rng.standard_normal(m).astype(np.float32)
    dy, v = rng.standard_normal((2, m)), rng.standard_normal((2, m))

    def value(h):
        return (h / np.sqrt((h * h).mean(1, keepdims=True) + 1e-5) * w * dy).sum(1)

    x, dy, v = (a.astype(np.float32).astype(np.float64) for a in (x, dy, v))
    slope = (value(x + 1e-5 * v) - value(x - 1e-5 * v)) / 2e-5
    t = [torch.from_numpy(a.astype(np.float32)).cuda() for a in (dy, x, w)]
    o = ctx.rms_norm_backward(t[0], t[1], ctx.rms_norm(t[1], t[2], eps=1e-5)["rstd"], t[2])
    got = (o["dx"].cpu().double().numpy() * v).sum(1)
    # differences: third derivatives 1e-10, roundings of float64 1e-16 / 1e-5; float32: 2^-24 (m / 8 + 80) of the terms
    assert np.all(np.abs(got - slope) <= 2.0 ** -24 * (m / 8 + 80) * (np.abs(dy * v).sum(1) + np.abs(v * x).sum(1) * np.abs(dy * x).mean(1)) + 1e-8)


# ---- together -----------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 37])
def test_a_feed_forward_block_and_its_gradients(ctx, T):
    """Norm with the residual -> gated projections -> down projection, and back to the block's input, as a model runs them.  Each step is
    checked against float64 on the values that the step before it left."""
    rng = np.random.default_rng(T)
    d, n = 384, 1000
    mats = [weights(rng, n, d), weights(rng, n, d), weights(rng, d, n)]
    gate, up, down = (ctx.group_quantize(torch.from_numpy(W).cuda(), group=64) for W in mats)
    Wg, Wu, Wd = (dense(*quantise(W, 64), 64) for W in mats)
    x, xv = rows(rng, T, d, torch.bfloat16)
    res, rv = rows(rng, T, d, torch.bfloat16)
    w = (1 + 0.1 * rng.standard_normal(d)).astype(np.float32)
    wt = torch.from_numpy(w).cuda()
    o = ctx.rms_norm(x, wt, residual=res, eps=1e-5)
    a = ctx.group_glu(gate, up, o["q"], x_scales=o["scales"])
    y = ctx.group_matmul(down, a)
    xq = o["q"].cpu().double().numpy() * o["scales"].cpu().double().numpy()[:, None]
    g, u, eg, eu = glu_errors(xq, Wg, Wu, d)
    close(a, silu(g) * u, 1.1 * eg * np.abs(u) + np.abs(silu(g)) * eu + eg * eu + 2.0 ** -8 * 1.02 * np.abs(silu(g) * u) + 1e-30, "a")
    av = a.cpu().double().numpy()
    close(y, av @ Wd.T, 2.0 ** -8 * 1.01 * np.abs(av @ Wd.T) + loss(n) * (np.abs(av) @ np.abs(Wd).T), "y")
    dy, dyv = gradient(rng, T, d)
    da = ctx.group_matmul_dx(down, dy)
    close(da, dyv @ Wd, 2.0 ** -8 * 1.01 * np.abs(dyv @ Wd) + loss(d) * (np.abs(dyv) @ np.abs(Wd)), "da")
    back = ctx.group_glu_backward(gate, up, o["q"], da, x_scales=o["scales"])
    grads = ctx.rms_norm_backward(back["dx"], o["h"], o["rstd"], wt, dh=dy)
    # the whole of it, with the roundings to bfloat16 on the way: 6 of them, each at most 2^-8 of sizes that do not cancel much in norm
    h = torch.from_numpy(xv + rv).float().to(torch.bfloat16).double().numpy()
    rstd = 1 / np.sqrt((h * h).mean(1, keepdims=True) + 1e-5)
    dav = dyv @ Wd
    dn = (dav * u * dsilu(g)) @ Wg + (dav * silu(g)) @ Wu
    hat, gg = h * rstd, dn * w
    dx = rstd * (gg - hat * (gg * hat).mean(1, keepdims=True)) + dyv
    got = grads["dx"].cpu().double().numpy()
    assert np.linalg.norm(got - dx) <= 6 * 2.0 ** -8 * np.linalg.norm(dx)
    assert np.linalg.norm(grads["dweight"].cpu().double().numpy() - (dn * hat).sum(0)) <= 6 * 2.0 ** -8 * np.linalg.norm((dn * hat).sum(0))


@pytest.mark.gpu
def test_calls_replay_from_captured_graphs(gpu_lib):
    """Every operator captured into one graph, replayed with eager work of the same context on other inputs in between."""
    stream = torch.cuda.Stream()
    ctx = gpu_lib.Context(0, stream=stream)
    try:
        gen = torch.Generator(device="cuda").manual_seed(9)

        def rand(*shape, dtype=torch.bfloat16):
            return torch.randn(shape, device="cuda", generator=gen).to(dtype)

        with torch.cuda.stream(stream):
            W, V = rand(300, 640, dtype=torch.float32), rand(640, 300, dtype=torch.float32)
            sets = [(rand(T, 640), rand(T, 640), rand(T, 640), torch.rand(640, device="cuda", generator=gen)) for T in (90, 90, 1, 1)]

            def block(x, res, dy, w):
                gq, down = ctx.group_quantize(W, group=64), ctx.group_quantize(V, group=32)
                o = ctx.rms_norm(x, w, residual=res, want_y=True)
                a = ctx.group_glu(gq, gq, o["q"], x_scales=o["scales"])
                y = ctx.group_matmul(down, a, out_dtype=torch.float32)
                da = ctx.group_matmul_dx(down, dy)
                b = ctx.group_glu_backward(gq, gq, o["q"], da, x_scales=o["scales"])
                r = ctx.rms_norm_backward(b["dx"], o["h"], o["rstd"], w, dh=dy)
                return [gq["codes"], gq["scales"], ctx.group_unpack(gq), o["h"], o["q"].view(torch.uint8), o["scales"], o["y"], a, y, da, *b.values(), *r.values()]

            eager = [[v.clone() for v in block(*s)] for s in sets]
        stream.synchronize()
        graphs = []
        for s in sets[::2]:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                out = block(*s)
            graphs.append((g, out))
        for rep in range(3):
            with torch.cuda.stream(stream):
                for g, out in graphs:
                    for v in out:
                        v.zero_()
                    other = block(*sets[1])
                    g.replay()
            stream.synchronize()
            for (g, out), ref in zip(graphs, eager[::2]):
                for i, (v, e) in enumerate(zip(out, ref)):
                    assert torch.equal(v, e), (rep, i)
            for i, (v, e) in enumerate(zip(other, eager[1])):
                assert torch.equal(v, e), (rep, i, "eager")
    finally:
        ctx.close()


@pytest.mark.gpu
def test_refusals(ctx, gpu_lib):
    rng = np.random.default_rng(1)
    gq, _ = matrix(rng, 32, 128, 128)
    x, _, _ = inputs(rng, 4, 128, "bf16")
    q, s, _ = inputs(rng, 4, 128, "e4m3")
    y = torch.empty((4, 32), dtype=torch.bfloat16, device="cuda")
    big = torch.empty((4, 128), dtype=torch.float32, device="cuda")
    cp, sp, xp, yp, qp, fp = (t.data_ptr() for t in (gq["codes"], gq["scales"], x, y, q, s))
    lib, h = ctx.lib, ctx.h
    ARG, SHAPE, WS = -1, -2, -4
    mm = lib.skim_group_matmul
    assert mm(h, None, sp, 32, 128, 128, xp, 1, 128, None, 4, yp, 1, None, 0) == ARG
    assert mm(h, cp + 4, sp, 32, 128, 128, xp, 1, 128, None, 4, yp, 1, None, 0) == ARG and b"aligned" in lib.skim_last_error(h)
    assert mm(h, cp, sp, 32, 128, 96, xp, 1, 128, None, 4, yp, 1, None, 0) == ARG
    assert mm(h, cp, sp, 0, 128, 128, xp, 1, 128, None, 4, yp, 1, None, 0) == SHAPE
    assert mm(h, cp, sp, 1 << 24, 1 << 24, 128, xp, 1, 1 << 24, None, 4, yp, 1, None, 0) == SHAPE
    assert mm(h, cp, sp, 32, 128, 128, xp, 0, 128, None, 4, yp, 1, None, 0) == ARG
    assert mm(h, cp, sp, 32, 128, 128, xp, 1, 127, None, 4, yp, 1, None, 0) == SHAPE
    assert mm(h, cp, sp, 32, 128, 128, xp, 1, 128, None, -1, yp, 1, None, 0) == SHAPE
    assert mm(h, cp, sp, 32, 128, 128, xp, 1, 128, fp, 4, yp, 1, None, 0) == ARG
    assert mm(h, cp, sp, 32, 128, 128, qp, 2, 128, None, 4, yp, 1, None, 0) == ARG
    assert mm(h, cp, sp, 32, 128, 128, xp, 1, 128, None, 4, yp, 2, None, 0) == ARG
    assert mm(h, cp, sp, 32, 128, 128, xp, 1, 128, None, 4, None, 1, None, 0) == ARG
    assert mm(h, cp, sp, 32, 128, 128, xp, 1, 128, None, 4, yp, 1, None, 64) == ARG
    assert mm(h, cp, sp, 32, 128, 128, xp, 1, 128, None, 4, yp, 1, xp + 8, 64) == ARG and b"scratch" in lib.skim_last_error(h)
    dx = lib.skim_group_matmul_dx
    assert dx(h, cp, sp, 32, 128, 128, None, 32, 4, xp, 1, None, 0) == ARG
    assert dx(h, cp, sp, 32, 128, 128, yp, 31, 4, xp, 1, None, 0) == SHAPE
    assert lib.skim_group_glu(h, cp, sp, cp, None, 32, 128, 128, xp, 1, 128, None, 4, yp, 1, None, 0) == ARG
    assert lib.skim_group_glu_backward(h, cp, sp, cp, sp, 32, 128, 128, xp, 1, 128, None, 4, yp, 32, None, yp, None, 1, None, 0) == ARG
    assert lib.skim_group_quantize(h, big.data_ptr(), 4, 128, 127, 128, cp, sp) == SHAPE
    assert lib.skim_group_quantize(h, None, 4, 128, 128, 128, cp, sp) == ARG
    assert lib.skim_group_unpack(h, cp, sp, 4, 128, 128, None) == ARG
    norm = lib.skim_rms_norm
    assert norm(h, xp, 128, None, 0, 2, None, 1e-6, 4, 128, None, xp, None, None, None) == ARG
    assert norm(h, xp, 128, None, 0, 1, None, 0.0, 4, 128, None, xp, None, None, None) == ARG
    assert norm(h, xp, 128, None, 0, 1, None, float("nan"), 4, 128, None, xp, None, None, None) == ARG
    assert norm(h, xp, 128, xp, 128, 1, None, 1e-6, 4, 128, None, xp, None, None, None) == ARG
    assert norm(h, xp, 128, None, 0, 1, None, 1e-6, 4, 128, None, None, qp, None, None) == ARG
    assert norm(h, xp, 128, None, 0, 1, None, 1e-6, 4, 128, None, None, None, None, None) == ARG
    assert norm(h, xp, 40000, None, 0, 1, None, 1e-6, 1, 32769, None, xp, None, None, None) == SHAPE
    assert norm(h, xp, 100, None, 0, 1, None, 1e-6, 4, 128, None, xp, None, None, None) == SHAPE
    back = lib.skim_rms_norm_backward
    assert back(h, xp, 128, xp, 128, None, 0, 1, fp, None, 4, 128, xp, fp, None, 0) == WS
    assert back(h, xp, 128, xp, 128, None, 0, 1, None, None, 4, 128, xp, None, None, 0) == ARG
    with pytest.raises(AssertionError):
        ctx.group_matmul(gq, x.float())
    with pytest.raises(AssertionError):
        ctx.group_matmul(gq, q)
    with pytest.raises(AssertionError):
        ctx.group_matmul(gq, x, x_scales=s)
    with pytest.raises(AssertionError):
        ctx.group_matmul(gq, x.t())
    with pytest.raises(AssertionError):
        ctx.group_matmul(dict(gq, n=33), x)
    with pytest.raises(AssertionError):
        ctx.group_matmul(gq, x, out=torch.empty((4, 31), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(AssertionError):
        ctx.group_glu(gq, matrix(rng, 32, 128, 64)[0], x)
    with pytest.raises(ValueError):
        ctx.group_quantize(big, group=100)
    with pytest.raises(gpu_lib.SkimError):
        ctx.rms_norm(big, eps=0.0)


# ---- how the work is shared out, memory far away, other streams -----------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("T,n,m", [(2048, 4352, 1030), (4096, 4352, 140), (512, 4096, 4096), (4096, 4130, 1100)])
def test_many_tiles(ctx, T, n, m):
    """272 tiles (256 whole ones, the rest in parts), 544 (four wavefronts a workgroup), 64 (all in parts), 544 again as 512 and 32 in parts."""
    rng = np.random.default_rng(T + m)
    gq, W = matrix(rng, n, m, 64)
    x, s, value = inputs(rng, T, m, "e4m3")
    want, size = value @ W.T, np.abs(value) @ np.abs(W).T
    close(ctx.group_matmul(gq, x, x_scales=s, out_dtype=torch.float32), want, 2.0 ** -24 * np.abs(want) + loss(m) * size, "y")
    if m < 1000:
        return
    tq, V = matrix(rng, m, n, 32)                              # (the other way round: a gradient with as many tiles)
    dy, _, value = inputs(rng, T, m, "bf16")
    want, size = value @ V, np.abs(value) @ np.abs(V)
    close(ctx.group_matmul_dx(tq, dy, out_dtype=torch.float32), want, 2.0 ** -24 * np.abs(want) + loss(m) * size, "dx")


@pytest.mark.gpu
def test_without_scratch(ctx):
    """Fewer workgroups share a tile then, with the same result to the last digits; what has to be converted first is refused."""
    rng = np.random.default_rng(21)
    T, n, m = 100, 300, 4096
    gq, W = matrix(rng, n, m, 128)
    x, _, value = inputs(rng, T, m, "bf16")
    q, s, _ = inputs(rng, T, m, "e4m3")
    lib, h = ctx.lib, ctx.h
    y = torch.empty((T, n), device="cuda")
    cp, sp = gq["codes"].data_ptr(), gq["scales"].data_ptr()
    assert lib.skim_group_scratch_bytes(h, n, m, T, 0) > 0 and lib.skim_group_scratch_bytes(h, n, m, 64, 0) == 0
    assert lib.skim_group_scratch_bytes(h, n, m, 0, 0) == lib.skim_group_scratch_bytes(h, n, m, T, 3) == 0
    assert lib.skim_group_matmul(h, cp, sp, n, m, 128, x.data_ptr(), 1, m, None, T, y.data_ptr(), 0, None, 0) == 0
    want, size = value @ W.T, np.abs(value) @ np.abs(W).T
    close(y, want, 2.0 ** -24 * np.abs(want) + loss(m) * size, "y")
    assert lib.skim_group_matmul(h, cp, sp, n, m, 128, q.data_ptr(), 2, m, s.data_ptr(), T, y.data_ptr(), 0, None, 0) == -4
    assert b"scratch" in lib.skim_last_error(h)
    dy, _, dvalue = inputs(rng, 5, n, "bf16")                 # rows of 300 values: not on 16-byte borders
    dx = torch.empty((5, m), device="cuda")
    assert lib.skim_group_matmul_dx(h, cp, sp, n, m, 128, dy.data_ptr(), n, 5, dx.data_ptr(), 0, None, 0) == -4
    need = lib.skim_group_scratch_bytes(h, n, m, 5, 1)
    scratch = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert lib.skim_group_matmul_dx(h, cp, sp, n, m, 128, dy.data_ptr(), n, 5, dx.data_ptr(), 0, scratch.data_ptr(), need) == 0
    close(dx, dvalue @ W, 2.0 ** -24 * np.abs(dvalue @ W) + loss(n) * (np.abs(dvalue) @ np.abs(W)), "dx")


@pytest.mark.gpu
@pytest.mark.parametrize("T", [40, 70])
def test_rows_of_x_that_lie_far_apart(ctx, T):
    """The last rows begin more than 2^31 values (4 GB) behind the first, further than a tile's copies reach."""
    rng = np.random.default_rng(31)
    n, m, ld = 64, 256, 1 << 26
    gq, W = matrix(rng, n, m, 64)
    v = torch.from_numpy(rng.standard_normal((T, m))).to(torch.bfloat16)
    mem = torch.empty((T - 1) * ld + m, dtype=torch.bfloat16, device="cuda")
    x = mem.as_strided((T, m), (ld, 1))
    x.copy_(v.cuda())
    want, size = v.double().numpy() @ W.T, np.abs(v.double().numpy()) @ np.abs(W).T
    close(ctx.group_matmul(gq, x, out_dtype=torch.float32), want, 2.0 ** -24 * np.abs(want) + loss(m) * size, "y")
    o = ctx.rms_norm(x, eps=1e-5, want_y=True)
    h = v.double().numpy()
    yv = h / np.sqrt((h * h).mean(1, keepdims=True) + float(np.float32(1e-5)))
    close(o["y"], yv, U[torch.bfloat16] * 1.01 * np.abs(yv), "norm")
    dy = mem.as_strided((T, n), (ld, 1))
    d = v[:, :n].double().numpy()
    close(ctx.group_matmul_dx(gq, dy, out_dtype=torch.float32), d @ W, 2.0 ** -24 * np.abs(d @ W) + loss(n) * (np.abs(d) @ np.abs(W)), "dx")
    del mem, x, dy
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_matrices_of_more_than_2_31_bytes(ctx):
    """The last 16 rows, 2.1 GB behind the first, against the same rows as a matrix of their own."""
    n, m, G = (1 << 17) + 16, (1 << 15) + 128, 128
    gen = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(-2 ** 31, 2 ** 31, ((n // 16) * (m // 128) * 256,), dtype=torch.int32, device="cuda", generator=gen)
    scales = (torch.randint(16, 32, (m // G, n), device="cuda", generator=gen).float() / 1024).to(torch.bfloat16)
    big = dict(codes=codes, scales=scales, n=n, m=m, group=G)
    last = dict(codes=codes[-(m // 128) * 256:].clone(), scales=scales[:, -16:].contiguous(), n=16, m=m, group=G)
    assert codes.numel() * 4 > 2 ** 31
    D = ctx.group_unpack(last).cpu().double().numpy()
    for T in (1, 40, 70):
        x = torch.randn((T, m), device="cuda", generator=gen).to(torch.bfloat16)
        v = x.cpu().double().numpy()
        want, size = v @ D.T, np.abs(v) @ np.abs(D).T
        y = ctx.group_matmul(big, x, out_dtype=torch.float32)
        close(y[:, -16:], want, 2.0 ** -24 * np.abs(want) + loss(m) * size, f"T={T}")
        del y
        dy = torch.zeros((T, n), dtype=torch.bfloat16, device="cuda")
        dy[:, -16:] = x[:, :16]
        d = v[:, :16]
        close(ctx.group_matmul_dx(big, dy, out_dtype=torch.float32), d @ D, 2.0 ** -24 * np.abs(d @ D) + loss(n) * (np.abs(d) @ np.abs(D)), f"dx T={T}")
    del big, last, codes, scales
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_a_context_on_a_stream_that_is_not_current(gpu_lib, ctx):
    """Its outputs and scratch belong to its stream, whatever is current where it is called."""
    rng = np.random.default_rng(17)
    gq, _ = matrix(rng, 300, 1000, 64)
    x, s, _ = inputs(rng, 90, 1000, "e4m3")
    ref = ctx.group_matmul(gq, x, x_scales=s)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    other = gpu_lib.Context(0, stream=stream)
    try:
        for _ in range(3):
            y = other.group_matmul(gq, x, x_scales=s)
            n = other.rms_norm(y, want_y=True)
        stream.synchronize()
        assert torch.equal(y, ref) and torch.equal(n["y"], ctx.rms_norm(ref, want_y=True)["y"])
    finally:
        other.close()


@pytest.mark.gpu
def test_infinities_and_nans_stay_in_their_token(ctx):
    rng = np.random.default_rng(19)
    for T in (3, 90):
        gq, W = matrix(rng, 100, 300, 64)
        x, _, value = inputs(rng, T, 300, "bf16")
        want, size = value @ W.T, np.abs(value) @ np.abs(W).T
        x[1, 7] = float("nan")
        x[2, 299] = float("inf")
        y = ctx.group_matmul(gq, x, out_dtype=torch.float32)
        keep = [t for t in range(T) if t not in (1, 2)]
        close(y[keep], want[keep], 2.0 ** -24 * np.abs(want[keep]) + loss(300) * size[keep], "others")
        assert torch.isnan(y[1]).all() and not torch.isfinite(y[2]).all()
        dy, _, dvalue = inputs(rng, T, 100, "bf16")
        dy[1, 99] = float("nan")
        dx = ctx.group_matmul_dx(gq, dy, out_dtype=torch.float32)
        rest = [t for t in range(T) if t != 1]
        close(dx[rest], (dvalue @ W)[rest], 2.0 ** -24 * np.abs(dvalue @ W)[rest] + loss(100) * (np.abs(dvalue) @ np.abs(W))[rest], "dx")
        assert torch.isnan(dx[1]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_sums_over_the_longest_rows(ctx, kind):
    """2^23 values a token: the last tokens of a tile begin 2.1 GB behind its first."""
    T, k, few, G = 128, 1 << 23, 16, 128
    gen = torch.Generator(device="cuda").manual_seed(3)
    at = torch.cat([torch.arange(0, 100), torch.arange(k // 2 - 50, k // 2 + 50), torch.arange(k - 300, k)]).cuda()
    x = torch.zeros((T, k), dtype=torch.bfloat16, device="cuda")
    x[:, at] = torch.randint(-8, 9, (T, at.numel()), device="cuda", generator=gen).to(torch.bfloat16)       # (e4m3 numbers)
    v = x[:, at].cpu().double().numpy()
    codes = torch.randint(-2 ** 31, 2 ** 31, (few * k // 8,), dtype=torch.int32, device="cuda", generator=gen)
    scale = lambda *shape: (torch.randint(16, 32, shape, device="cuda", generator=gen).float() / 1024).to(torch.bfloat16)
    wide = dict(codes=codes, scales=scale(k // G, few), n=few, m=k, group=G)
    D = ctx.group_unpack(wide)[:, at].cpu().double().numpy()
    allowed = lambda D: 2.0 ** -24 * np.abs(v @ D) + loss(at.numel() + 64) * (np.abs(v) @ np.abs(D))          # (zeros add without loss)
    if kind == "bf16":
        y = ctx.group_matmul(wide, x, out_dtype=torch.float32)
    else:
        y = ctx.group_matmul(wide, x.to(torch.float8_e4m3fn), x_scales=torch.ones(T, device="cuda"), out_dtype=torch.float32)
    close(y, v @ D.T, allowed(D.T), "y")
    if kind == "bf16":
        tall = dict(codes=torch.randint(-2 ** 31, 2 ** 31, (k * 16,), dtype=torch.int32, device="cuda", generator=gen), scales=scale(1, k), n=k, m=few, group=G)
        D = ctx.group_unpack(tall)[at].cpu().double().numpy()
        close(ctx.group_matmul_dx(tall, x, out_dtype=torch.float32), v @ D, allowed(D), "dx")
    del x, wide, codes
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m", [1, 100, 4096, 20000])
def test_rms_norm_of_rows_with_nans_and_infinities(ctx, dtype, m):
    x = torch.randn((6, m), device="cuda").to(dtype)
    good = ctx.rms_norm(x, want_y=True)
    bad = x.clone()
    bad[1, m // 2], bad[2, m - 1], bad[4] = float("nan"), float("-inf"), float("nan")
    o = ctx.rms_norm(bad, want_y=True)
    for t in range(6):
        if t in (1, 2, 4):
            assert torch.isnan(o["scales"][t]) and torch.isnan(o["q"][t].float()).all(), t
            assert torch.isnan(o["y"][t]).all() if t != 2 else torch.isnan(o["y"][t, -1]) and not o["y"][t, :-1].any()
        else:
            for key in ("scales", "q", "y", "rstd"):
                assert torch.equal(o[key][t].float(), good[key][t].float()), (t, key)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 17, 32, 33, 64])
@pytest.mark.parametrize("n", [48, 200, 1021])
def test_gradients_of_few_tokens_are_rounded_once(ctx, T, n):
    """In float32 dx comes as near as the sums let it: a rounding of dgate and dup to 8 bits on the way would be 2^-8 of their products off."""
    rng = np.random.default_rng(41 + T)
    m, group = 300, 64
    (gate, Wg), (up, Wu) = matrix(rng, n, m, group), matrix(rng, n, m, group)
    x, _, value = inputs(rng, T, m, "bf16")
    value[T - 1, 5] = np.nan
    x[T - 1, 5] = float("nan")                                # (a token that must not reach the others)
    da, dav = gradient(rng, T, n)
    dgate, dup = (torch.empty((T, n), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dx = torch.empty((T, m), device="cuda")
    need = ctx.lib.skim_group_scratch_bytes(ctx.h, n, m, T, 2)
    scratch = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")      # (NaN wherever it is not written)
    mats = [gate["codes"].data_ptr(), gate["scales"].data_ptr(), up["codes"].data_ptr(), up["scales"].data_ptr(), n, m, group]

    def call(room):
        assert ctx.lib.skim_group_glu_backward(ctx.h, *mats, x.data_ptr(), 1, x.stride(0), None, T, da.data_ptr(), n, dgate.data_ptr(), dup.data_ptr(),
                                               dx.data_ptr(), 0, scratch.data_ptr(), room) == 0
        return dx.cpu().double().numpy()

    got = call(need)
    assert (scratch[need:] == 0xFF).all()
    g, u = value @ Wg.T, value @ Wu.T
    dg, du = dav * u * dsilu(g), dav * silu(g)
    want, size = dg @ Wg + du @ Wu, np.abs(dg) @ np.abs(Wg) + np.abs(du) @ np.abs(Wu)
    sums = np.abs(value) @ (np.abs(Wg) + np.abs(Wu)).T * loss(m)                     # of g and u, then as in test_glu_backward
    e = np.abs(dav) * (1.1 * sums * (1 + np.abs(u)) + 16 * 2.0 ** -24 * (1 + np.abs(g)) * np.abs(u)) + (2.0 ** -16 + (8 + np.minimum(np.abs(g), 100)) * 2.0 ** -24) * (np.abs(dg) + np.abs(du))
    allowed = e @ (np.abs(Wg) + np.abs(Wu)) + loss(4 * n) * 1.01 * size
    over = np.abs(got - want) - allowed
    assert np.all(over[: T - 1] <= 0) and np.isnan(got[T - 1]).all()
    if n % 8 == 0:                                            # without room for the pieces: of dgate and dup as stored
        got = call(0)
        sg, su = dgate.cpu().double().numpy(), dup.cpu().double().numpy()
        over = np.abs(got - (sg @ Wg + su @ Wu)) - loss(2 * n) * (np.abs(sg) @ np.abs(Wg) + np.abs(su) @ np.abs(Wu))
        assert np.all(over[: T - 1] <= 0) and np.isnan(got[T - 1]).all()
