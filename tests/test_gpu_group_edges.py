"""Products with 4-bit weights and the norm at the borders of what they are documented for: gradients in 16 bits, strides of every input, scratch of just
the size that a call needs, values at the ends of the types' ranges.  Plain float64 on the CPU; U and loss() are derived in test_gpu_group.py."""

import numpy as np
import pytest
import torch

from test_gpu_group import U, ctx, close, dense, dsilu, glu_errors, gradient, inputs, lib, loss, matrix, pack, quantise, silu, weights  # noqa: F401

BF16 = torch.bfloat16


# ---- CPU ----------------------------------------------------------------------------------------------------------------

def test_size_of_the_scratch_without_a_context(lib):
    assert lib.skim_group_scratch_bytes_for(None, 128, 128, 100, 0, None, 1, 128, 1) == 0


# ---- gradients of the gated block -----------------------------------------------------------------------------------------

def gated_gradients(value, dav, Wg, Wu, m):
    """dgate and dup by the formula, and how far float32 ones may be off (as in test_glu_backward; before any rounding to bfloat16)."""
    g, u, eg, eu = glu_errors(value, Wg, Wu, m)
    dg, du = dav * u * dsilu(g), dav * silu(g)
    f = (8 + np.minimum(np.abs(g), 100)) * 2.0 ** -24
    eg, eu = (np.abs(dav) * (1.1 * eu + 0.5 * eg * (np.abs(u) + eu) + 16 * 2.0 ** -24 * (1 + np.abs(g)) * np.abs(u)) + f * np.abs(dg),
              np.abs(dav) * 1.1 * eg + f * np.abs(du))
    return dg, du, eg, eu


GATED = [(65, 48, 300, 64), (100, 200, 300, 32), (128, 1021, 500, 128), (130, 272, 1100, 128), (300, 513, 520, 64), (1000, 330, 260, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,n,m,group", GATED)
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_float32_gradients_of_many_tokens_are_rounded_once(ctx, T, n, m, group, kind):
    """dx in float32 is made of two bfloat16 pieces of dgate and dup, 2^-16 of them off; dgate and dup stay what they are without it."""
    rng = np.random.default_rng(T + n)
    (gate, Wg), (up, Wu) = matrix(rng, n, m, group), matrix(rng, n, m, group)
    x, s, value = inputs(rng, T, m, kind)
    da, dav = gradient(rng, T, n)
    o = ctx.group_glu_backward(gate, up, x, da, x_scales=s, out_dtype=torch.float32)
    dg, du, eg, eu = gated_gradients(value, dav, Wg, Wu, m)
    want, size = dg @ Wg + du @ Wu, np.abs(dg) @ np.abs(Wg) + np.abs(du) @ np.abs(Wu)
    off = (eg + 2.0 ** -16 * np.abs(dg)) @ np.abs(Wg) + (eu + 2.0 ** -16 * np.abs(du)) @ np.abs(Wu)
    assert o["dx"].dtype == torch.float32
    close(o["dx"], want, 1.01 * off + loss(4 * n) * 1.01 * size + 2.0 ** -24 * np.abs(want), "dx")
    plain = ctx.group_glu_backward(gate, up, x, da, x_scales=s)
    assert plain["dx"].dtype == BF16 and torch.equal(plain["dgate"], o["dgate"]) and torch.equal(plain["dup"], o["dup"])
    into = torch.empty_like(o["dx"])                          # a given result says its type
    assert ctx.group_glu_backward(gate, up, x, da, x_scales=s, out=dict(dx=into))["dx"] is into and torch.equal(into, o["dx"])


@pytest.mark.gpu
@pytest.mark.parametrize("T,n,m,group", GATED)
def test_gradients_of_many_tokens_against_the_formula(ctx, T, n, m, group):
    """dx in bfloat16 is made of dgate and dup as they are returned: two roundings of at most U, each of at most U / sqrt(3) in the root of the mean square; the errors
    of the first are independent of one another and of the second, so that over the T m results they add up in squares (5 % more allowed for their number)."""
    rng = np.random.default_rng(T * 3 + n)
    (gate, Wg), (up, Wu) = matrix(rng, n, m, group), matrix(rng, n, m, group)
    x, s, value = inputs(rng, T, m, "bf16")
    da, dav = gradient(rng, T, n)
    got = ctx.group_glu_backward(gate, up, x, da)["dx"].cpu().double().numpy()
    dg, du, eg, eu = gated_gradients(value, dav, Wg, Wu, m)
    want, size = dg @ Wg + du @ Wu, np.abs(dg) @ np.abs(Wg) + np.abs(du) @ np.abs(Wu)
    u = U[BF16] * 1.01
    off = (eg + u * np.abs(dg)) @ np.abs(Wg) + (eu + u * np.abs(du)) @ np.abs(Wu) + loss(4 * n) * 1.01 * size
    assert np.all(np.abs(got - want) <= off + u * (np.abs(want) + off))
    assert np.linalg.norm(got - want) <= 1.05 * np.sqrt(2 / 3) * U[BF16] * np.linalg.norm(want)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [64, 65, 130])
@pytest.mark.parametrize("kind,ld,offset", [("bf16", 320, 0), ("bf16", 305, 3), ("e4m3", 304, 0)])
def test_scratch_of_float32_gradients_is_what_the_size_query_says(ctx, T, kind, ld, offset):
    """Nothing behind it is written; with less, dx is made of dgate and dup as they are stored; a token with a NaN does not reach the others."""
    rng = np.random.default_rng(T + ld)
    n, m, group = 208, 300, 64
    (gate, Wg), (up, Wu) = matrix(rng, n, m, group), matrix(rng, n, m, group)
    x, s, value = inputs(rng, T, m, kind, ld, offset)
    value[T - 1, 5] = np.nan
    x.view(torch.int16 if kind == "bf16" else torch.uint8)[T - 1, 5] = 0x7FC0 if kind == "bf16" else 0x7F
    da, dav = gradient(rng, T, n)
    dgate, dup = (torch.empty((T, n), dtype=BF16, device="cuda") for _ in range(2))
    dx = torch.empty((T, m), device="cuda")
    xt, sp = (1, None) if kind == "bf16" else (2, s.data_ptr())
    query = lambda dt: ctx.lib.skim_group_scratch_bytes_for(ctx.h, n, m, T, 2, x.data_ptr(), xt, ld, dt)  # noqa: E731
    need = query(0)
    assert need >= 8 * T * n and (T <= 64 or query(1) < need)
    scratch = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")       # (NaN wherever it is not written)
    mats = [gate["codes"].data_ptr(), gate["scales"].data_ptr(), up["codes"].data_ptr(), up["scales"].data_ptr(), n, m, group]

    def call(room):
        assert ctx.lib.skim_group_glu_backward(ctx.h, *mats, x.data_ptr(), xt, ld, sp, T, da.data_ptr(), n, dgate.data_ptr(), dup.data_ptr(), dx.data_ptr(), 0,
                                               scratch.data_ptr(), room) == 0
        return dx.cpu().double().numpy()

    got = call(need)
    assert (scratch[need:] == 0xFF).all()
    dg, du, eg, eu = gated_gradients(value, dav, Wg, Wu, m)
    want, size = dg @ Wg + du @ Wu, np.abs(dg) @ np.abs(Wg) + np.abs(du) @ np.abs(Wu)
    off = (eg + 2.0 ** -16 * np.abs(dg)) @ np.abs(Wg) + (eu + 2.0 ** -16 * np.abs(du)) @ np.abs(Wu) + loss(4 * n) * 1.01 * size
    assert np.all((np.abs(got - want) <= 1.01 * off + 2.0 ** -24 * np.abs(want))[: T - 1]) and np.isnan(got[T - 1]).all()
    if T > 64:
        got = call(query(1))
        sg, su = dgate.cpu().double().numpy(), dup.cpu().double().numpy()
        over = np.abs(got - (sg @ Wg + su @ Wu)) - loss(2 * n) * (np.abs(sg) @ np.abs(Wg) + np.abs(su) @ np.abs(Wu))
        assert np.all(over[: T - 1] <= 0) and np.isnan(got[T - 1]).all()


# ---- norm -----------------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,m", [(5, 100), (600, 1000), (600, 4097), (5, 9000), (5, 20000)])
def test_rms_norm_scales_of_products_that_are_no_numbers(ctx, dtype, T, m):
    """max |y| / 448 is a NaN where a y is: an infinity under a weight of 0, a weight that is a NaN, 0 under an infinite weight."""
    gen = torch.Generator(device="cuda").manual_seed(m)
    x = torch.randn((T, m), device="cuda", generator=gen).to(dtype)
    w = 1 + 0.1 * torch.randn(m, device="cuda", generator=gen)
    same = lambda o, ref, rows: all(torch.equal(o[k][rows].float(), ref[k][rows].float()) for k in ("scales", "q", "rstd"))  # noqa: E731
    no_number = lambda o, t: bool(torch.isnan(o["scales"][t]) and torch.isnan(o["q"][t].float()).all())  # noqa: E731
    others = [t for t in range(T) if t not in (1, T - 1)]
    for col in (0, m // 2, m - 1):
        pruned = w.clone()
        pruned[col] = 0
        bad = x.clone()
        bad[1, col], bad[T - 1, col] = float("inf"), float("-inf")
        o, ref = ctx.rms_norm(bad, pruned), ctx.rms_norm(x, pruned)
        assert no_number(o, 1) and no_number(o, T - 1) and same(o, ref, others), col
        o = ctx.rms_norm(bad, torch.zeros_like(w))             # ... alone: all other products are zeros
        assert no_number(o, 1) and no_number(o, T - 1) and (o["scales"][others] == 1).all() and not o["q"][others].float().any()
        without = w.clone()
        without[col] = float("nan")
        o = ctx.rms_norm(x, without)
        assert all(no_number(o, t) for t in range(0, T, max(1, T // 7))) and torch.isnan(o["scales"]).all()
        assert torch.equal(o["rstd"], ref["rstd"])
        endless, zero = w.clone(), x.clone()
        endless[col] = float("inf")
        zero[:, col] = 1
        zero[1, col] = zero[T - 1, col] = 0
        o = ctx.rms_norm(zero, endless)
        assert no_number(o, 1) and no_number(o, T - 1)
        assert torch.isinf(o["scales"][others]).all() and torch.isnan(o["q"][others, col].float()).all()
        rest = o["q"].float()[others]
        rest[:, col] = 0
        assert not rest.any()
    h, r = x.clone(), x.clone()                                # x + residual past the largest number, under a weight of 0
    big = torch.finfo(dtype).max
    pruned = w.clone()
    pruned[7] = 0
    h[1, 7] = r[1, 7] = big
    o = ctx.rms_norm(h, pruned, residual=r)
    assert torch.isinf(o["h"][1, 7]) and no_number(o, 1) and same(o, ctx.rms_norm(x, pruned, residual=x), [t for t in range(T) if t != 1])


# ---- values at the ends of the types' ranges --------------------------------------------------------------------------------

def scaled_matrix(rng, n, m, group, power):
    q, s = quantise(weights(rng, n, m) * np.float32(2.0) ** power, group)
    codes, scales = pack(q, s, group)
    return dict(codes=codes.cuda(), scales=scales.cuda(), n=n, m=m, group=group), dense(q, s, group)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 3, 17, 40, 64, 65, 130])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("power,of_x", [(-40, 124), (-100, 120), (110, -90), (125, -110), (-119, 40), (-8, -112)])
def test_products_of_large_and_small_values(ctx, T, group, power, of_x):
    """Weights of 2^power / 50 and x of 2^of_x: every product and sum of the formula is a normal float32, whatever its factors are, and so are the results of any
    number of tokens.  (125: groups with an outlier have scales of 2^121.  2^-119 / 50 / 7 is above the least scale, 2^-126, for a group's largest weight; groups below it have codes of 0 or 1, as the format says.)"""
    rng = np.random.default_rng(T + group)
    n, m = 150, 700
    gq, W = scaled_matrix(rng, n, m, group, power)
    x = torch.from_numpy(rng.standard_normal((T, m))).to(BF16).double() * 2.0 ** of_x      # (exact: a power of two)
    v = x.numpy()
    want, size = v @ W.T, np.abs(v) @ np.abs(W).T
    assert np.isfinite(want).all() and 2.0 ** -122 < np.abs(want).max() < 2.0 ** 100
    y = ctx.group_matmul(gq, x.to(BF16).cuda(), out_dtype=torch.float32)
    close(y, want, 2.0 ** -24 * np.abs(want) + loss(m) * size, "y")
    tq, V = scaled_matrix(rng, m, n, group, power)
    want, size = v @ V, np.abs(v) @ np.abs(V)
    close(ctx.group_matmul_dx(tq, x.to(BF16).cuda(), out_dtype=torch.float32), want, 2.0 ** -24 * np.abs(want) + loss(m) * size, "dx")


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 16, 33, 64, 65])
def test_gated_block_of_large_activations_and_small_weights(ctx, T):
    """g and u of a few units from x of 2^125 (and up to 2^127.3): sums of q x, without the scales, come past the largest float32."""
    rng = np.random.default_rng(T)
    n, m, group = 100, 600, 128
    (gate, Wg), (up, Wu) = scaled_matrix(rng, n, m, group, -122), scaled_matrix(rng, n, m, group, -122)
    x = torch.from_numpy(rng.standard_normal((T, m))).to(BF16).double() * 2.0 ** 125
    xb, value = x.to(BF16).cuda(), x.numpy()
    g, u, eg, eu = glu_errors(value, Wg, Wu, m)
    want = silu(g) * u
    a = ctx.group_glu(gate, up, xb, out_dtype=torch.float32)
    close(a, want, 1.1 * eg * np.abs(u) + np.abs(silu(g)) * eu + 1.1 * eg * eu + (U[torch.float32] * 1.01 + (8 + np.minimum(np.abs(g), 100)) * 2.0 ** -24) * np.abs(want), "a")
    da, dav = gradient(rng, T, n)
    o = ctx.group_glu_backward(gate, up, xb, da, want_dx=False)
    dg, du, eg, eu = gated_gradients(value, dav, Wg, Wu, m)
    close(o["dgate"], dg, eg + U[BF16] * 1.01 * (np.abs(dg) + eg), "dgate")
    close(o["dup"], du, eu + U[BF16] * 1.01 * (np.abs(du) + eu), "dup")


# ---- scratch ----------------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
def test_scratch_holds_a_copy_of_x_only_where_the_tiles_take_one(ctx):
    """The size for one call is that for any call less the copy, where rows lie on 16-byte borders; it is 0 for what the calls reject."""
    lib, h = ctx.lib, ctx.h
    of = lambda n, m, T, g, x, xt, ld, dt=1: lib.skim_group_scratch_bytes_for(h, n, m, T, g, x, xt, ld, dt)  # noqa: E731
    any_call = lambda n, m, T, g: lib.skim_group_scratch_bytes(h, n, m, T, g)  # noqa: E731
    copy = lambda columns, T: (-(-columns // 8) * 8 * T * 2 + 255) // 256 * 256  # noqa: E731
    for n, m, T in ((4096, 11008, 2048), (11008, 4096, 131072), (300, 1000, 90), (1021, 2999, 70)):
        as_it_is = m % 8 == 0
        assert any_call(n, m, T, 0) - of(n, m, T, 0, 1 << 20, 1, m) == (copy(m, T) if as_it_is else 0)
        assert any_call(n, m, T, 0) == of(n, m, T, 0, 1 << 20, 2, m) == of(n, m, T, 0, (1 << 20) + 2, 1, m) == of(n, m, T, 0, 1 << 20, 1, m + 1)
        assert any_call(n, m, T, 1) - of(n, m, T, 1, 1 << 20, 1, n) == (copy(n, T) if n % 8 == 0 else 0)
        assert any_call(n, m, T, 2) == of(n, m, T, 2, 1 << 20, 2, m) >= of(n, m, T, 2, 1 << 20, 1, m)
        assert of(n, m, T, 2, 1 << 20, 2, m, 0) > 8 * n * T                              # (dgate and dup in 16 bits)
    assert of(300, 1000, 64, 0, 1 << 20, 2, 1000) == 0 and of(300, 1000, 1, 1, 1 << 20, 1, 300) > 0
    for bad in ((0, 8, 90, 0, 0, 1, 8), (8, 0, 90, 0, 0, 1, 8), (8, 8, 0, 0, 0, 1, 8), (8, 8, 90, 3, 0, 1, 8), (8, 8, 90, -1, 0, 1, 8), (8, 8, 90, 0, 0, 0, 8), (8, 8, 90, 0, 0, 3, 8),
                (8, 16, 90, 0, 0, 2, 15), (16, 8, 90, 1, 0, 1, 15), (8, 8, 90, 1, 0, 2, 8), (8, 8, 90, 1, 0, 1, 8, 2), (8, 8, 90, 2, 0, 2, 8, 2), (1 << 24, 8, 90, 0, 0, 2, 8)):
        assert of(*bad) == 0, bad


@pytest.mark.gpu
def test_long_prompts_allocate_their_results_and_no_copies(ctx):
    rng = np.random.default_rng(2)
    T, n, m = 16384, 256, 2048
    gq, _ = matrix(rng, n, m, 128)
    x = torch.zeros((T, m), dtype=BF16, device="cuda")
    dy = torch.zeros((T, n), dtype=BF16, device="cuda")
    for call, result in ((lambda: ctx.group_matmul(gq, x), 2 * T * n), (lambda: ctx.group_glu(gq, gq, x), 2 * T * n), (lambda: ctx.group_matmul_dx(gq, dy), 2 * T * m)):
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        call()
        # (partial sums of at most 32 MB; a copy of x would be 67 MB, of dy 8)
        assert torch.cuda.max_memory_allocated() - before <= result + (32 << 20) + (1 << 20)
        aligned = ctx.lib.skim_group_scratch_bytes_for(ctx.h, n, m, T, 0, x.data_ptr(), 1, m, 1)
        assert torch.cuda.max_memory_allocated() - before <= result + max(aligned, ctx.lib.skim_group_scratch_bytes_for(ctx.h, n, m, T, 1, dy.data_ptr(), 1, n, 1)) + 4096


# ---- strides and alignment of the backward pass's inputs ------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 16, 40, 64, 65, 130])
@pytest.mark.parametrize("n", [96, 101, 200])
@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 0), (4, 4), (4, 2), (5, 3), (0, 1)])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_glu_backward_with_rows_of_any_stride(ctx, T, n, pad, offset, kind):
    """da and x on rows further apart than they are long (NaNs between them) and off every border, each with fours and octets on theirs and not."""
    rng = np.random.default_rng(T * 100 + n + 10 * pad + offset)
    m, group = 264, 64
    (gate, Wg), (up, Wu) = matrix(rng, n, m, group), matrix(rng, n, m, group)
    x, s, value = inputs(rng, T, m, kind, m + pad, offset)
    da, _, dav = inputs(rng, T, n, "bf16", n + pad, offset)
    dg, du, eg, eu = gated_gradients(value, dav, Wg, Wu, m)
    u = U[BF16] * 1.01
    want, size = dg @ Wg + du @ Wu, np.abs(dg) @ np.abs(Wg) + np.abs(du) @ np.abs(Wu)
    off = (eg + 2.0 ** -16 * np.abs(dg)) @ np.abs(Wg) + (eu + 2.0 ** -16 * np.abs(du)) @ np.abs(Wu) + loss(4 * n) * 1.01 * size
    o = ctx.group_glu_backward(gate, up, x, da, x_scales=s, out_dtype=torch.float32)
    close(o["dgate"], dg, eg + u * (np.abs(dg) + eg), "dgate")
    close(o["dup"], du, eu + u * (np.abs(du) + eu), "dup")
    close(o["dx"], want, 1.01 * off + 2.0 ** -24 * np.abs(want), "dx")
    o = ctx.group_glu_backward(gate, up, x, da, x_scales=s)
    sg, su = o["dgate"].cpu().double().numpy(), o["dup"].cpu().double().numpy()
    if T > 64:
        want, off = sg @ Wg + su @ Wu, loss(4 * n) * 1.01 * (np.abs(sg) @ np.abs(Wg) + np.abs(su) @ np.abs(Wu))
    close(o["dx"], want, u * (np.abs(want) + off) + 1.01 * off, "dx in bfloat16")


# ---- input validation -----------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("n,m,pad", [(1, 1, 0), (37, 300, 0), (5000, 256, 0), (40, 129, 3)])
def test_validation_mode_reports_weights_that_have_no_code(gpu_lib, n, m, pad):
    rng = np.random.default_rng(n)
    store = torch.full((n, m + pad), float("nan"), device="cuda")           # (NaNs between the rows are nobody's)
    W = store[:, :m]
    W.copy_(torch.from_numpy(weights(rng, n, m)))
    c = gpu_lib.Context(0)
    try:
        ref = c.group_quantize(W)
        c.validate_enable(True)
        for i, j in ((0, 0), (n // 2, m // 2), (n - 1, m - 1)):
            kept = W[i, j].item()
            for bad in (float("nan"), float("inf"), float("-inf"), 2.0 ** 127, -2.0 ** 127):
                W[i, j] = bad
                with pytest.raises(gpu_lib.SkimError, match="W holds") as e:
                    c.group_quantize(W)
                assert e.value.status == -6
            W[i, j] = 1.5 * 2.0 ** 126
            c.group_quantize(W)
            W[i, j] = kept
        got = c.group_quantize(W)
        assert torch.equal(got["codes"], ref["codes"]) and torch.equal(got["scales"].view(torch.int16), ref["scales"].view(torch.int16))
        c.validate_enable(False)
        W[0, 0] = float("nan")
        c.group_quantize(W)                                                 # off (the default): not looked for, no error
        torch.cuda.synchronize()
    finally:
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 70])
def test_refused_gradients_leave_their_outputs_alone(ctx, T):
    """Without scratch, dx of rows that are no multiple of 8 is refused, and dgate and dup are not written either."""
    rng = np.random.default_rng(T)
    n, m, group = 101, 264, 64
    (gate, _), (up, _) = matrix(rng, n, m, group), matrix(rng, n, m, group)
    x, _, _ = inputs(rng, T, m, "bf16")
    da, _ = gradient(rng, T, n)
    outs = [torch.full((T, k), 7.0, dtype=BF16, device="cuda") for k in (n, n, m)]
    mats = [gate["codes"].data_ptr(), gate["scales"].data_ptr(), up["codes"].data_ptr(), up["scales"].data_ptr(), n, m, group]
    call = lambda dx, scratch, room: ctx.lib.skim_group_glu_backward(ctx.h, *mats, x.data_ptr(), 1, m, None, T, da.data_ptr(), n, outs[0].data_ptr(), outs[1].data_ptr(),  # noqa: E731
                                                                     dx, 1, scratch, room)
    assert call(outs[2].data_ptr(), None, 0) == -4 and b"scratch" in ctx.lib.skim_last_error(ctx.h)
    torch.cuda.synchronize()
    assert all((o == 7).all() for o in outs)
    assert call(None, None, 0) == 0                                         # (without dx none is needed)
    torch.cuda.synchronize()
    assert not (outs[0] == 7).any() and (outs[2] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 16, 17, 64, 65])
@pytest.mark.parametrize("of_x", [-120, 124])
def test_scales_of_8_bit_activations_at_the_ends_of_float32(ctx, T, of_x):
    """Sums are taken before the token's scale: it is multiplied on at the end, however large or small."""
    rng = np.random.default_rng(T)
    n, m, group = 100, 700, 64
    gq, W = scaled_matrix(rng, n, m, group, 0 if of_x < 0 else -100)
    q, s, value = inputs(rng, T, m, "e4m3")
    s, value = s * 2.0 ** of_x, value * 2.0 ** of_x
    assert torch.isfinite(s).all() and (s > 0).all()
    want, size = value @ W.T, np.abs(value) @ np.abs(W).T
    close(ctx.group_matmul(gq, q, x_scales=s, out_dtype=torch.float32), want, 2.0 ** -23 * np.abs(want) + loss(m) * size, "y")
