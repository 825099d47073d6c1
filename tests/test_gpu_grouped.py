"""Weights of 4 bits with group scales, their products and the norm in front of them, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import grouped

pytestmark = pytest.mark.gpu

HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step, relative
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}   # half the smallest step


@pytest.fixture()
def ctx(skimlib):
    c = skimlib.Skim(device=0)
    c.set_workspace(torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    yield c
    assert c.get_status() == 0
    c.close()


def weights(rows, cols, seed=0):
    rng = np.random.default_rng([seed, rows, cols])
    w = rng.standard_normal((rows, cols)) * 0.02
    far = rng.random((rows, cols)) < 2e-3
    return np.where(far, w * 10, w).astype(np.float16)


def held(w, group, device="cuda"):
    """The oracle's stored form on the GPU, as grouped_quantize returns it, and the binary64 values."""
    codes, scale, zero = grouped.quantize(w, group)
    tiles = torch.from_numpy(grouped.store(codes, scale, zero, group)).to(device)
    return dict(tiles=tiles, rows=w.shape[0], cols=w.shape[1], group=group, err=None), grouped.values(codes, scale, zero, group)


def token_rows(tokens, cols, dtype, seed=1, pad=0, shift=0):
    """Rows on the GPU, `pad` NaN (or 8-bit extremes) behind each, `shift` elements behind an aligned address; their float64 values; the scales of 8-bit rows."""
    rng = np.random.default_rng([seed, tokens, cols])
    x = rng.standard_normal((tokens, cols)) * np.exp(0.5 * rng.standard_normal(cols))
    scale = None
    if dtype == torch.int8:
        scale = (np.abs(x).max(axis=1) / 127 if x.size else np.zeros(tokens)).astype(np.float32)
        x = np.rint(x / np.maximum(scale, 1e-30)[:, None])
    room = torch.full((tokens * (cols + pad) + shift,), -128 if dtype == torch.int8 else float("nan"), dtype=dtype, device="cuda")
    t = room[shift:].view(tokens, cols + pad)[:, :cols]
    t.copy_(torch.from_numpy(x).to(dtype))
    return t, t.double().cpu().numpy(), scale


def product_bound(cols, group, size, exact, dtype):
    """Binary32 additions of exact products: at most 17 operands (16 products and the sum) in each of a group's group / 16 instructions, a
    multiply-add a group, then at most 8 warps and 8 blocks; each may lose a whole unit of binary32, 2^-23 of the magnitudes' sum.  Two more for the scales
    and the token's scale, then the rounding of the result."""
    steps = 17 * (group // 16) + -(-cols // group) + 8 + 8 + 4
    off = steps * 2.0 ** -23 * size
    return off + HALF[dtype] * (np.abs(exact) + off) + TINY[dtype]


# ---------------------------------------------------------------- quantisation

SHAPES = [(1, 1), (1, 31), (3, 32), (8, 33), (15, 127), (16, 128), (17, 129), (40, 300), (64, 1000), (5, 3001), (200, 512)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_is_the_oracles_bytes(ctx, rows, cols, group):
    w = weights(rows, cols)
    g = np.exp(np.random.default_rng(5).standard_normal((rows, cols))).astype(np.float32)
    codes, scale, zero = grouped.quantize(w, group)
    want = grouped.store(codes, scale, zero, group)
    value = grouped.values(codes, scale, zero, group)
    W = torch.from_numpy(w).cuda()
    for importance in (None, g):
        out = dict(tiles=torch.full((len(want),), 0xA5, dtype=torch.uint8, device="cuda"), rows=rows, cols=cols, group=group, err=torch.full((rows,), -1.0, device="cuda"))
        q = ctx.grouped_quantize(W, group, importance=None if importance is None else torch.from_numpy(importance).cuda(), out=out)
        np.testing.assert_array_equal(q["tiles"].cpu().numpy(), want)
        # a lane adds at most 32 terms of every eighth record, then 2 + 7 sums; a term has at most four roundings
        exact = grouped.error(w, value, importance)
        steps = 32 * -(-cols // 1024) + 16
        np.testing.assert_allclose(q["err"].cpu().numpy(), exact, rtol=steps * 2.0 ** -24, atol=1e-30)
    plain = ctx.grouped_quantize(W, group)
    assert plain["err"] is None and torch.equal(plain["tiles"], q["tiles"])
    back = ctx.grouped_dequantize(q)
    np.testing.assert_array_equal(back.cpu().numpy().view(np.uint16) & 0x7fff | (back.cpu().numpy().view(np.uint16) & 0x8000) * (back.cpu().numpy() != 0),
                                  value.astype(np.float16).view(np.uint16) & 0x7fff | (value.astype(np.float16).view(np.uint16) & 0x8000) * (value.astype(np.float16) != 0))


@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantize_at_the_borders(ctx, group):
    """Quotients that are exactly k + 1/2, groups of one value, of zeros, of the smallest and the largest numbers, of one sign."""
    rng = np.random.default_rng(3)
    w = np.zeros((96, 384), np.float16)
    for i in range(32):                                   # s = 2^-5 or a value with 11 bits: ties
        s = np.float16(2.0 ** -5 if i % 2 else float(rng.integers(1024, 2048)) * 2.0 ** -16)
        k = rng.integers(0, 31, 384)
        w[i] = (k.astype(np.float64) / 2 * float(s)).astype(np.float16)
        w[i, ::32] = np.float16(15 * float(s))
    w[32:40] = (rng.integers(-3, 4, (8, 384)) * 2.0 ** -24).astype(np.float16)             # subnormal scales, or none
    w[40:48] = (rng.integers(-40, 41, (8, 384)) * 2.0 ** -24).astype(np.float16)
    w[48:56] = np.where(rng.random((8, 384)) < 0.5, 65504, -65504).astype(np.float16)
    w[56:60] = np.float16(0.3)
    w[60:64] = np.float16(-0.3)
    w[64:72] = -np.abs(rng.standard_normal((8, 384))).astype(np.float16)
    w[72:80] = np.float16(-0.0)
    w[80:88] = np.where(rng.random((8, 384)) < 0.01, 500, 1e-3 * rng.standard_normal((8, 384))).astype(np.float16)
    w[88:] = (rng.integers(-8, 8, (8, 384)) / 16).astype(np.float16)
    codes, scale, zero = grouped.quantize(w, group)
    q = ctx.grouped_quantize(torch.from_numpy(w).cuda(), group)
    np.testing.assert_array_equal(q["tiles"].cpu().numpy(), grouped.store(codes, scale, zero, group))


@pytest.mark.parametrize("ld,shift", [(304, 0), (303, 1), (307, 3)])
def test_quantize_strided_rows(ctx, ld, shift):
    w = weights(33, 300, seed=2)
    room = torch.full((33 * ld + shift,), float("nan"), dtype=torch.float16, device="cuda")
    W = room[shift:].view(33, ld)[:, :300]
    W.copy_(torch.from_numpy(w))
    imp = torch.full((33 * ld + shift,), float("nan"), device="cuda")
    G = imp[shift:].view(33, ld)[:, :300]
    g = np.exp(np.random.default_rng(6).standard_normal((33, 300))).astype(np.float32)
    G.copy_(torch.from_numpy(g))
    codes, scale, zero = grouped.quantize(w, 64)
    q = ctx.grouped_quantize(W, 64, importance=G, want_err=True)
    np.testing.assert_array_equal(q["tiles"].cpu().numpy(), grouped.store(codes, scale, zero, 64))
    np.testing.assert_allclose(q["err"].cpu().numpy(), grouped.error(w, grouped.values(codes, scale, zero, 64), g), rtol=64 * 2.0 ** -24)
    out = torch.full((33 * ld + shift,), 7.0, dtype=torch.float16, device="cuda")
    view = out[shift:].view(33, ld)
    ctx.grouped_dequantize(q, out=view[:, :300])
    np.testing.assert_array_equal(view[:, :300].cpu().numpy(), grouped.values(codes, scale, zero, 64).astype(np.float16))
    assert bool((view[:, 300:] == 7).all()) and bool((out[:shift] == 7).all())


def test_quantize_with_a_scale_vector(ctx):
    w = weights(48, 200, seed=4)
    alpha = np.exp(0.3 * np.random.default_rng(1).standard_normal(200)).astype(np.float32)
    ctx.apply_scale(torch.from_numpy(alpha).cuda())
    r = np.float32(1) / alpha
    codes, scale, zero = grouped.quantize(w, 32, r)
    q = ctx.grouped_quantize(torch.from_numpy(w).cuda(), 32, want_err=True)
    np.testing.assert_array_equal(q["tiles"].cpu().numpy(), grouped.store(codes, scale, zero, 32))
    np.testing.assert_allclose(q["err"].cpu().numpy(), grouped.error(w, grouped.values(codes, scale, zero, 32), None, r), rtol=64 * 2.0 ** -24)
    with pytest.raises(Exception, match="SKIM_ERR_SCALE"):
        ctx.grouped_quantize(torch.zeros((4, 64), dtype=torch.float16, device="cuda"), 32)


def test_quantize_bad_data_is_flagged(ctx):
    for bad, flag in ((float("nan"), 1), (float("inf"), 1), (float("-inf"), 1)):
        W = torch.zeros((4, 64), dtype=torch.float16, device="cuda")
        W[2, 33] = bad
        ctx.grouped_quantize(W, 32)
        assert ctx.get_status() == flag
    W = torch.ones((4, 64), dtype=torch.float16, device="cuda")
    for bad in (float("nan"), float("inf"), -1.0):
        G = torch.ones((4, 64), device="cuda")
        G[1, 5] = bad
        ctx.grouped_quantize(W, 32, importance=G, want_err=True)
        assert ctx.get_status() == 2


# ---------------------------------------------------------------- products

TOKENS_SHAPES = [(1, 1, 1), (1, 16, 128), (2, 17, 129), (3, 100, 64), (7, 33, 1000), (8, 250, 2100), (9, 48, 384), (16, 64, 256), (17, 130, 520),
                 (31, 128, 128), (33, 129, 640), (64, 200, 1001), (65, 256, 256), (130, 300, 513), (257, 140, 2048)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.int8])
@pytest.mark.parametrize("tokens,rows,cols", TOKENS_SHAPES)
def test_matvec(ctx, tokens, rows, cols, dtype):
    for n, group in enumerate((32, 64, 128)):
        q, value = held(weights(rows, cols, seed=n), group)
        x, xv, xs = token_rows(tokens, cols, dtype, seed=n, pad=8 * n)
        out_dtype = (torch.float32, torch.float16, torch.bfloat16)[(n + rows) % 3]
        y = ctx.grouped_matvec(q, x, x_scale=None if xs is None else torch.from_numpy(xs).cuda(), out_dtype=out_dtype)
        assert y.shape == (tokens, rows) and y.dtype == out_dtype
        exact, size = grouped.product(value, xv, xs)
        assert np.all(np.abs(y.double().cpu().numpy() - exact) <= product_bound(cols, group, size, exact, out_dtype))


def gated_bound(cols, group, act, g, gs, u, us, dtype):
    """The products' errors through the gate: |act'| is at most 1.2 (both activations), |act| at most |g|.  The activation itself: exp, a division and
    the products (tanh: the sum 1 + tanh, an error of 2^-23 of 1 and less than 2^-20 of its argument's effect) stay under 2^-20 |g|."""
    dg = product_bound(cols, group, gs, g, torch.float32)
    du = product_bound(cols, group, us, u, torch.float32)
    a = grouped.activation(act, g)
    off = (1.2 * dg + 2.0 ** -20 * (np.abs(g) + dg)) * (np.abs(u) + du) + np.abs(a) * du
    exact = a * u
    return exact, off * (1 + 2.0 ** -22) + HALF[dtype] * (np.abs(exact) + off) + TINY[dtype]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.int8])
@pytest.mark.parametrize("tokens,rows,cols", TOKENS_SHAPES)
def test_gated(ctx, tokens, rows, cols, dtype):
    for n, group in enumerate((32, 64, 128)):
        act = ("silu", "gelu")[(n + tokens) % 2]
        qg, vg = held(weights(rows, cols, seed=10 + n), group)
        qu, vu = held(weights(rows, cols, seed=20 + n), group)
        x, xv, xs = token_rows(tokens, cols, dtype, seed=n)
        out_dtype = (torch.float32, torch.float16, torch.bfloat16)[(n + rows) % 3]
        y = ctx.grouped_gated(qg, qu, x, x_scale=None if xs is None else torch.from_numpy(xs).cuda(), activation=act, out_dtype=out_dtype)
        g, gs = grouped.product(vg, xv, xs)
        u, us = grouped.product(vu, xv, xs)
        exact, bound = gated_bound(cols, group, act, g, gs, u, us, out_dtype)
        assert np.all(np.abs(y.double().cpu().numpy() - exact) <= bound)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gate_far_out(ctx, act):
    """Gates from -1e4 to 1e4: no overflow on the way, the negative side goes to zero."""
    w = np.zeros((16, 32), np.float16)
    w[:, 0] = np.linspace(-1, 1, 16)
    one = np.zeros((16, 32), np.float16)
    one[:, 1] = 1
    x = np.zeros((40, 32))
    x[:, 0] = np.concatenate([-np.logspace(-3, 4, 20), np.logspace(-3, 4, 20)])
    x[:, 1] = 1
    t = torch.from_numpy(x).half().cuda()
    qg, vg = held(w, 32)
    qu, vu = held(one, 32)
    g, gs = grouped.product(vg, t.double().cpu().numpy())
    u, us = grouped.product(vu, t.double().cpu().numpy())
    with np.errstate(over="ignore"):
        exact, bound = gated_bound(32, 32, act, g, gs, u, us, torch.float32)
    for rows in (t[:3], t[:12], t):
        y = ctx.grouped_gated(qg, qu, rows.contiguous(), activation=act).double().cpu().numpy()
        assert np.all(np.abs(y - exact[:len(rows)]) <= bound[:len(rows)])


@pytest.mark.parametrize("tokens", [1, 5, 40, 70])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.int8])
@pytest.mark.parametrize("pad,shift", [(0, 0), (1, 0), (8, 3), (3, 1)])
def test_rows_at_any_address_and_the_rows_between(ctx, tokens, dtype, pad, shift):
    """Rows of x anywhere, NaN between them; what lies between and behind the rows of y stays."""
    rows, cols = 50, 264
    q, value = held(weights(rows, cols), 64)
    x, xv, xs = token_rows(tokens, cols, dtype, pad=pad, shift=shift)
    room = torch.full((tokens + 1, rows + 5), 3.0, device="cuda")
    y = ctx.grouped_matvec(q, x, x_scale=None if xs is None else torch.from_numpy(xs).cuda(), out=room[:tokens, :rows])
    exact, size = grouped.product(value, xv, xs)
    assert np.all(np.abs(y.double().cpu().numpy() - exact) <= product_bound(cols, 64, size, exact, torch.float32))
    assert bool((room[:, rows:] == 3).all()) and bool((room[tokens:] == 3).all())


@pytest.mark.parametrize("tokens", [3, 12, 90])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_what_is_not_finite_stays_in_its_row(ctx, tokens, dtype):
    rows, cols = 40, 300
    q, value = held(weights(rows, cols), 128)
    x, _, _ = token_rows(tokens, cols, dtype)
    clean = ctx.grouped_matvec(q, x)
    x[1, 7] = float("nan")
    x[2, 299] = float("inf")
    y = ctx.grouped_matvec(q, x)
    keep = [t for t in range(tokens) if t not in (1, 2)]
    assert torch.equal(y[keep], clean[keep]) and bool(y[1].isnan().all())
    want = np.where(value[:, 299] == 0, np.nan, np.inf * np.sign(value[:, 299]))
    np.testing.assert_array_equal(y[2].cpu().numpy().astype(np.float64), want)


def test_few_rows_and_long_rows_share_the_columns(ctx):
    """Few rows: blocks of a cluster share the columns.  8-bit rows without a scale and whole weights give whole sums below 2^24: no rounding anywhere."""
    for rows, cols, tokens in [(16, 4096, 1), (5, 16384, 8), (33, 22016, 3), (16, 9000, 16), (16, 8200, 33), (128, 8192, 70), (20, 131072, 17)]:
        rng = np.random.default_rng(cols)
        w = rng.integers(-1, 15, (rows, cols))
        w[:, 0::32] = -1
        w[:, 1::32] = 14                                  # high - low = 15: s = 1, z = 1, and the values are the weights
        q = ctx.grouped_quantize(torch.from_numpy(w).half().cuda(), 32)
        x = rng.integers(-16, 17, (tokens, cols))
        y = ctx.grouped_matvec(q, torch.from_numpy(x).to(torch.int8).cuda())
        np.testing.assert_array_equal(y.cpu().numpy(), (x @ w.T).astype(np.float64))
        up = ctx.grouped_gated(q, q, torch.from_numpy(np.sign(x) * 127).to(torch.int8).cuda())
        g = (np.sign(x) * 127) @ w.T
        far = np.abs(g) > 100
        np.testing.assert_allclose(up.cpu().numpy()[far], np.where(g > 0, g.astype(np.float64) ** 2, 0.0)[far], rtol=2.0 ** -23, atol=1e-30)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.int8])
@pytest.mark.parametrize("rows,cols,tokens,pad,runs", [(11008, 1024, 600, 0, 5),          # several tiles one after another on every SM
                                                       (3001, 520, 700, 16, 2),           # ragged in every direction
                                                       (520, 4101, 300, 11, 2),           # few tiles: four pairs of blocks share the columns
                                                       (1030, 4096, 601, 0, 2),           # two pairs
                                                       (12000, 2000, 20, 0, 2),           # few tokens, many rows
                                                       (3001, 519, 700, 2, 2),            # rows at odd addresses, copied first
                                                       (4100, 4099, 9, 0, 2)])
def test_many_tokens(ctx, rows, cols, tokens, pad, runs, dtype, group):
    """All rows and tokens, run by run, against 64 bits (products on the GPU, of the oracle's values)."""
    w = [weights(rows, cols, seed) for seed in (1, 2)]
    qs = [ctx.grouped_quantize(torch.from_numpy(v).cuda(), group) for v in w]
    values = [torch.from_numpy(grouped.values(*grouped.quantize(v, group), group)).cuda() for v in w]
    x, xv, scale = token_rows(tokens, cols, dtype, pad=pad)
    xs = None if scale is None else torch.from_numpy(scale).cuda()
    xd = torch.from_numpy(xv).cuda() * (1.0 if xs is None else xs.double()[:, None])
    exact = [xd @ v.t() for v in values]
    size = [xd.abs() @ v.abs().t() for v in values]
    as_np = lambda v: v.cpu().numpy()
    bound = product_bound(cols, group, as_np(size[0]), as_np(exact[0]), torch.float32)
    want, gated = gated_bound(cols, group, "gelu", as_np(exact[0]), as_np(size[0]), as_np(exact[1]), as_np(size[1]), torch.bfloat16)
    for _ in range(runs):
        assert np.all(np.abs(as_np(ctx.grouped_matvec(qs[0], x, x_scale=xs).double()) - as_np(exact[0])) <= bound)
        assert np.all(np.abs(as_np(ctx.grouped_gated(qs[0], qs[1], x, x_scale=xs, activation="gelu", out_dtype=torch.bfloat16).double()) - want) <= gated)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_many_tokens_not_finite_and_the_rows_between(ctx, dtype):
    rows, cols, tokens = 3001, 520, 700
    q = ctx.grouped_quantize(torch.from_numpy(weights(rows, cols)).cuda(), 128)
    x, _, _ = token_rows(tokens, cols, dtype, pad=8)
    room = torch.full((tokens + 1, rows + 3), 5.0, device="cuda")
    clean = ctx.grouped_matvec(q, x)
    gate = ctx.grouped_gated(q, q, x)
    x[1, 7], x[600, 519] = float("nan"), float("-inf")
    y = ctx.grouped_matvec(q, x, out=room[:tokens, :rows])
    keep = [t for t in range(tokens) if t not in (1, 600)]
    assert torch.equal(y[keep], clean[keep]) and bool(y[1].isnan().all()) and not bool(y[600].isfinite().any())
    assert torch.equal(ctx.grouped_gated(q, q, x)[keep], gate[keep])
    assert bool((room[:, rows:] == 5).all()) and bool((room[tokens] == 5).all())


def test_room_for_a_copy_given_or_too_small(ctx):
    q = ctx.grouped_quantize(torch.from_numpy(weights(2000, 1000)).cuda(), 128)
    x, xv, _ = token_rows(500, 1000, torch.float16, pad=3)
    value = grouped.values(*grouped.quantize(weights(2000, 1000), 128), 128)
    exact, size = grouped.product(value, xv)
    bound = product_bound(1000, 128, size, exact, torch.float32)
    for n in (500 * 1000 * 2, 500 * 1000 * 2 - 1, 0):
        room = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        y = ctx.grouped_matvec(q, x, scratch=room[:n])
        assert np.all(np.abs(y.double().cpu().numpy() - exact) <= bound)
        assert bool((room[n:] == 0xA5).all()) and (n == 500 * 1000 * 2 or bool((room == 0xA5).all()))
    with pytest.raises(Exception, match="SKIM_ERR_WORKSPACE"):
        ctx.grouped_matvec(q, x, scratch=torch.empty(2000000, dtype=torch.uint8, device="cuda")[8:])


def test_rows_far_apart(ctx):
    """Rows of x and of y, and of the norm, more than 2^31 elements from the first one."""
    cols, rows, far = 256, 48, (1 << 30) + 64
    room = torch.empty(3 * far, dtype=torch.float16, device="cuda")
    x = room.view(3, far)[:, :cols]
    near, xv, _ = token_rows(3, cols, torch.float16)
    x.copy_(near)
    q, _ = held(weights(rows, cols), 64)
    y = room.view(3, far)[:, 512:512 + rows]
    ctx.grouped_matvec(q, x, out=y)
    assert torch.equal(y, ctx.grouped_matvec(q, near, out_dtype=torch.float16))
    out = room.view(3, far)[:, 1024:1024 + cols]
    ctx.add_rmsnorm(x, residual=x, out=out)
    assert torch.equal(out, ctx.add_rmsnorm(near, residual=near)[0])
    W = room.view(3, far)[:, 2048:2048 + cols]
    w = torch.from_numpy(weights(3, cols)).cuda()
    W.copy_(w)
    assert torch.equal(ctx.grouped_quantize(W, 32)["tiles"], ctx.grouped_quantize(w, 32)["tiles"])


def test_a_vector_and_one_row_are_the_same_and_runs_repeat(ctx):
    q, _ = held(weights(70, 700), 64)
    x, _, _ = token_rows(1, 700, torch.float16)
    a, b = ctx.grouped_matvec(q, x), ctx.grouped_matvec(q, x[0])
    assert b.shape == (70,) and torch.equal(a[0], b)
    many, _, _ = token_rows(100, 700, torch.bfloat16)
    assert torch.equal(ctx.grouped_matvec(q, many), ctx.grouped_matvec(q, many))


def test_nothing_to_do(ctx):
    q, _ = held(weights(20, 64), 32)
    empty = torch.empty((0, 64), dtype=torch.float16, device="cuda")
    assert ctx.grouped_matvec(q, empty).shape == (0, 20) and ctx.grouped_gated(q, q, empty).shape == (0, 20)
    none = ctx.grouped_quantize(torch.empty((0, 64), dtype=torch.float16, device="cuda"), 32, want_err=True)
    assert none["tiles"].numel() == 0 and ctx.grouped_dequantize(none).shape == (0, 64)
    assert ctx.grouped_matvec(none, torch.ones((3, 64), dtype=torch.float16, device="cuda")).shape == (3, 0)
    out, scale, stream = ctx.add_rmsnorm(empty, residual=empty, out_dtype=torch.int8)
    assert out.shape == (0, 64) and scale.shape == (0,) and stream.shape == (0, 64)


# ---------------------------------------------------------------- the norm

def norm_rows(rows, cols, dtype, seed, pad=0, shift=0, size=1.0):
    room = torch.full((rows * (cols + pad) + shift,), float("nan"), dtype=dtype, device="cuda")
    t = room[shift:].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.from_numpy(np.random.default_rng([seed, rows, cols]).standard_normal((rows, cols)) * size).to(dtype))
    return t


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (2, 7, 0, 0), (3, 8, 0, 0), (1, 4096, 0, 0), (200, 512, 8, 0), (300, 8192, 0, 0), (170, 4104, 0, 0),
                                                 (5, 1000, 3, 1), (160, 11008, 0, 0), (2, 32768, 0, 0), (2, 32776, 0, 0), (3, 40001, 1, 1), (1000, 64, 0, 0)])
def test_add_rmsnorm(ctx, rows, cols, pad, shift, dtype, eight):
    x, r = norm_rows(rows, cols, dtype, 1, pad, shift), norm_rows(rows, cols, dtype, 2, pad, shift, 3.0)
    w = norm_rows(1, cols, dtype, 3, size=0.5)[0] + 1
    for residual, weight in ((r, w), (None, w), (r, None)):
        h, want, codes, scale = grouped.add_rmsnorm(x.float().cpu().numpy(), None if residual is None else residual.float().cpu().numpy(),
                                                    None if weight is None else weight.float().cpu().numpy(), 1e-5)
        out, s, stream = ctx.add_rmsnorm(x, weight, eps=1e-5, residual=residual, out_dtype=torch.int8 if eight else None)
        # the sum of squares: at most 8 * ceil(cols / 8192) * 4 terms a lane (rows read again: more) and 10 exchanges; half of that in rstd, and a few products
        rel = (8 * max(4, -(-cols // 8192)) + 10 + 12) * 2.0 ** -24
        if eight:
            assert out.dtype == torch.int8
            np.testing.assert_array_equal(out.cpu().numpy(), codes)
            np.testing.assert_allclose(s.double().cpu().numpy(), scale, rtol=rel)
        else:
            assert s is None and out.dtype == dtype
            off = rel * np.abs(want)
            assert np.all(np.abs(out.double().cpu().numpy() - want) <= off + HALF[dtype] * (np.abs(want) + off) + TINY[dtype])
        if residual is None:
            assert stream is None
        else:
            assert torch.equal(stream, (x.float() + residual.float()).to(dtype))


def test_norm_codes_at_the_borders(ctx):
    """127 p / a exactly k + 1/2 (a = 254 or 127 / 2^n), rows of zeros, of the smallest numbers."""
    k = np.arange(-126, 127)
    rows = np.zeros((6, 256), np.float32)
    rows[0, :253], rows[0, 255] = k + 0.5, 127
    rows[1, :253], rows[1, 255] = (k + 0.5) * 2, -254
    rows[2, :253], rows[2, 255] = (k + 0.5) / 64, 127 / 64
    rows[4] = np.random.default_rng(1).integers(-60, 61, 256) * 2.0 ** -24
    rows[5, 3] = 2.0 ** -24
    for dtype in (torch.float16, torch.bfloat16):
        x = torch.from_numpy(rows).to(dtype).cuda()
        _, _, codes, scale = grouped.add_rmsnorm(x.float().cpu().numpy(), None, None, 0.0 if False else 1e-12)
        out, s, _ = ctx.add_rmsnorm(x, eps=1e-12, out_dtype=torch.int8)
        np.testing.assert_array_equal(out.cpu().numpy(), codes)
        np.testing.assert_allclose(s.double().cpu().numpy(), scale, rtol=1e-6)
        assert s[3] == 0
    tiny = torch.full((1, 64), 2.0 ** -130, dtype=torch.bfloat16, device="cuda")             # 127 / a overflows
    tiny[0, 1] = 2.0 ** -131
    out, s, _ = ctx.add_rmsnorm(tiny, eps=1e-5, out_dtype=torch.int8)
    assert out[0, 0] == 127 and out[0, 1] == 64


def test_norm_in_place_and_what_lies_between(ctx):
    for cols in (512, 515, 33000):
        x, r = norm_rows(3, cols, torch.float16, 1, pad=5), norm_rows(3, cols, torch.float16, 2, pad=5)
        want, _, stream = ctx.add_rmsnorm(x.contiguous(), residual=r.contiguous())
        room = torch.full((4, cols + 3), 9.0, dtype=torch.float16, device="cuda")
        out, _, s = ctx.add_rmsnorm(x, residual=r, sum_out=r, out=room[:3, :cols])
        assert torch.equal(out, want) and torch.equal(r, stream) and s.data_ptr() == r.data_ptr()
        assert bool((room[:, cols:] == 9).all()) and bool((room[3] == 9).all())
        out, _, _ = ctx.add_rmsnorm(x, residual=r, sum_out=r, out=x)                       # (the residual has become the sum)
        again, _, _ = ctx.add_rmsnorm(norm_rows(3, cols, torch.float16, 1), residual=stream)
        assert torch.equal(out, again)


def test_norm_of_what_is_not_finite(ctx):
    x = torch.ones((4, 100), dtype=torch.float16, device="cuda")
    x[1, 3], x[2, 4] = float("nan"), float("inf")
    out, s, _ = ctx.add_rmsnorm(x, out_dtype=torch.int8)
    assert bool(s[0].isfinite()) and bool(s[3].isfinite()) and not bool(s[1].isfinite()) and not bool(s[2].isfinite())
    assert torch.equal(out[0], out[3]) and int(out[1, 3]) == 0 and int(out[2, 4]) == 0
    y, _, _ = ctx.add_rmsnorm(x)
    assert bool(y[1].isnan().all()) and bool(y[2, 4].isnan()) and torch.equal(y[0], y[3])


# ---------------------------------------------------------------- a run of them, as a decoder's layer makes it

def oracle_feed_forward(x, r, w, gate, up, down, act, eight, dtype):
    h, rows, codes, scale = grouped.add_rmsnorm(x, r, w, 1e-5)
    if eight:
        rows = codes * scale[:, None]
    g, u = rows @ gate.T, rows @ up.T
    return h, (grouped.activation(act, g) * u) @ down.T, np.abs(grouped.activation(act, g) * u) @ np.abs(down).T


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("tokens", [1, 4, 20, 75])
def test_feed_forward(ctx, tokens, eight, dtype):
    cols, hidden = 256, 700
    gate, vg = held(weights(hidden, cols, 1), 64)
    up, vu = held(weights(hidden, cols, 2), 64)
    down, vd = held(weights(cols, hidden, 3), 64)
    x, r = norm_rows(tokens, cols, dtype, 4), norm_rows(tokens, cols, dtype, 5)
    w = (norm_rows(1, cols, dtype, 6, size=0.2)[0] + 1).contiguous()
    y, stream = ctx.feed_forward(x, w, gate, up, down, residual=r, eight_bit=eight)
    h, want, size = oracle_feed_forward(x.double().cpu().numpy(), r.double().cpu().numpy(), w.double().cpu().numpy(), vg, vu, vd, "silu", eight, dtype)
    assert torch.equal(stream, (x.float() + r.float()).to(dtype))
    # the hidden rows are rounded to `dtype`, and without 8 bits the normalised ones too (an error of half a step in every term of the gate's and the
    # up's sums, which the gate's slope of at most 1.2 passes on): half a step of the last sum's magnitudes for the first, of the products of magnitudes for the second
    off = 2 * HALF[dtype] * size
    if not eight:
        rows = np.abs(grouped.add_rmsnorm(x.double().cpu().numpy(), r.double().cpu().numpy(), w.double().cpu().numpy(), 1e-5)[1])
        gs, us = rows @ np.abs(vg).T, rows @ np.abs(vu).T
        off = off + HALF[dtype] * (2.2 * (gs * us)) @ np.abs(vd).T * 1.1
    assert np.all(np.abs(y.double().cpu().numpy() - want) <= off + HALF[dtype] * np.abs(want) + 1e-5 * size + TINY[dtype])


def test_what_the_quantiser_wrote_is_read_at_once(ctx):
    """Quantiser, dequantiser and products enqueued one behind the other without a wait, on matrices that follow one another."""
    x, xv, _ = token_rows(4, 2048, torch.float16)
    got = []
    for n in range(6):
        q = ctx.grouped_quantize(torch.from_numpy(weights(512, 2048, n)).cuda(), 128)
        got.append((ctx.grouped_dequantize(q), ctx.grouped_matvec(q, x), ctx.grouped_gated(q, q, x)))
    for n, (value, y, gated) in enumerate(got):
        codes, scale, zero = grouped.quantize(weights(512, 2048, n), 128)
        v = grouped.values(codes, scale, zero, 128)
        np.testing.assert_array_equal(value.cpu().numpy(), v.astype(np.float16))
        exact, size = grouped.product(v, xv)
        assert np.all(np.abs(y.double().cpu().numpy() - exact) <= product_bound(2048, 128, size, exact, torch.float32))
        want, bound = gated_bound(2048, 128, "silu", exact, size, exact, size, torch.float32)
        assert np.all(np.abs(gated.double().cpu().numpy() - want) <= bound)


def test_captured_and_replayed_on_a_stream_of_its_own(skimlib):
    """Two graphs that share a context and its workspace, replayed on new inputs; an eager call between them."""
    s = torch.cuda.Stream()
    c = skimlib.Skim(device=0, stream=s)
    c.set_workspace(torch.empty(4096, dtype=torch.uint8, device="cuda"))
    cols, hidden = 512, 1100
    gate, up, down = (held(weights(*shape, n), 128)[0] for n, shape in enumerate([(hidden, cols), (hidden, cols), (cols, hidden)]))
    w = torch.ones(cols, dtype=torch.float16, device="cuda")
    graphs = []
    torch.cuda.synchronize()
    for tokens in (2, 70, 1500):
        x, r = norm_rows(tokens, cols, torch.float16, 1), norm_rows(tokens, cols, torch.float16, 2)
        with torch.cuda.stream(s):
            c.feed_forward(x, w, gate, up, down, residual=r)
            s.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                y, stream = c.feed_forward(x, w, gate, up, down, residual=r)
        graphs.append((graph, x, r, y, stream))
    for seed in (11, 12):
        for graph, x, r, y, stream in graphs:
            with torch.cuda.stream(s):
                x.copy_(norm_rows(x.shape[0], cols, torch.float16, seed))
                graph.replay()
                eager, eager_stream = c.feed_forward(x, w, gate, up, down, residual=r)
            s.synchronize()
            assert torch.equal(y, eager) and torch.equal(stream, eager_stream)
    assert c.get_status() == 0
    c.close()


def test_results_are_made_on_the_contexts_stream(ctx):
    """Another stream is the current one: results and scratch come from the context's stream, so what was freed there is not written over early."""
    q = ctx.grouped_quantize(torch.from_numpy(weights(2000, 1000)).cuda(), 128)
    x, _, _ = token_rows(300, 1000, torch.float16, pad=3)
    want = ctx.grouped_matvec(q, x)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = [ctx.grouped_matvec(q, x) for _ in range(8)]
        out, scale, stream = ctx.add_rmsnorm(x, residual=x, out_dtype=torch.int8)
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in got) and torch.equal(stream, x + x)


def test_the_most_tokens(ctx):
    rows, cols, tokens = 33, 40, 1048560
    w = weights(rows, cols)
    q = ctx.grouped_quantize(torch.from_numpy(w).cuda(), 32)
    value = torch.from_numpy(grouped.values(*grouped.quantize(w, 32), 32)).cuda()
    x = torch.randn((tokens, cols), device="cuda").half()
    y = ctx.grouped_matvec(q, x)
    exact, size = x.double() @ value.t(), x.double().abs() @ value.abs().t()
    steps = 17 * 2 + 2 + 8 + 8 + 4                         # as product_bound counts them
    off = steps * 2.0 ** -23 * size
    assert bool(((y.double() - exact).abs() <= off + 2.0 ** -24 * (exact.abs() + off)).all())
    out, scale, _ = ctx.add_rmsnorm(x, out_dtype=torch.int8)
    assert int(out.abs().amax(dim=1).amin()) == 127 and bool(scale.isfinite().all())
    with pytest.raises(Exception, match="SKIM_ERR_SHAPE"):
        ctx.grouped_matvec(q, torch.zeros((tokens + 1, cols), dtype=torch.float16, device="cuda"))


def test_three_contexts_on_streams_of_their_own_at_once(skimlib):
    streams = [torch.cuda.Stream() for _ in range(3)]
    w = weights(3000, 1536)
    tiles, value = held(w[:16], 64)[0], grouped.values(*grouped.quantize(w, 64), 64)
    maker = skimlib.Skim(device=0)
    maker.set_workspace(torch.empty(4096, dtype=torch.uint8, device="cuda"))
    q = maker.grouped_quantize(torch.from_numpy(w).cuda(), 64)
    assert torch.equal(q["tiles"][:tiles["tiles"].numel()], tiles["tiles"])
    xs = [token_rows(t, 1536, torch.bfloat16, seed=t) for t in (3, 48, 500)]
    torch.cuda.synchronize()
    ctxs = [skimlib.Skim(device=0, stream=s) for s in streams]
    for c in ctxs:
        c.set_workspace(torch.empty(4096, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    got = [[c.grouped_matvec(q, x[0]) for c, x in zip(ctxs, xs)] for _ in range(20)]
    torch.cuda.synchronize()
    for ys in got:
        for y, x in zip(ys, xs):
            exact, size = grouped.product(value, x[1])
            assert np.all(np.abs(y.double().cpu().numpy() - exact) <= product_bound(1536, 64, size, exact, torch.float32))
    for c in ctxs:
        assert c.get_status() == 0
        c.close()


# ---------------------------------------------------------------- refusals of the binding

def test_binding_refuses(ctx):
    q, _ = held(weights(20, 64), 32)
    x = torch.zeros((2, 64), dtype=torch.float16, device="cuda")
    for bad in (x.cpu(), x.float(), x[:, :63], torch.zeros((64, 2), dtype=torch.float16, device="cuda").t(), x[None]):
        with pytest.raises(TypeError):
            ctx.grouped_matvec(q, bad)
    with pytest.raises(Exception, match="SKIM_ERR_SHAPE"):
        ctx.grouped_matvec(q, x[:1].expand(2, 64))                     # rows on top of one another
    with pytest.raises(Exception, match="SKIM_ERR_TYPE"):
        ctx.grouped_matvec(q, x, out_dtype=torch.int8)
    with pytest.raises(Exception, match="SKIM_ERR_TYPE"):
        ctx.grouped_gated(q, q, x, activation="relu")
    with pytest.raises(TypeError):
        ctx.grouped_matvec(dict(q, rows=40), x)
    with pytest.raises(TypeError):
        ctx.grouped_matvec(dict(q, group=16), x)
    with pytest.raises(TypeError):
        ctx.grouped_gated(q, held(weights(36, 64), 32)[0], x)
    with pytest.raises(TypeError):
        ctx.grouped_matvec(q, x, x_scale=torch.ones(3, device="cuda"))
    with pytest.raises(TypeError):
        ctx.grouped_matvec(q, x, out=torch.empty((3, 20), device="cuda"))
    with pytest.raises(TypeError):
        ctx.add_rmsnorm(x, torch.ones(64, device="cuda"))
    with pytest.raises(TypeError):
        ctx.add_rmsnorm(x, residual=x[:1])
    with pytest.raises(Exception, match="SKIM_ERR_TYPE"):
        ctx.add_rmsnorm(x, out_dtype=torch.float32)
    with pytest.raises(TypeError):
        ctx.grouped_quantize(x, 32, importance=torch.ones((2, 65), device="cuda")[:, :64])
    with pytest.raises(Exception, match="SKIM_ERR_TYPE"):
        ctx.grouped_quantize(x, 16)


def test_products_need_a_workspace(skimlib):
    c = skimlib.Skim(device=0)
    q, _ = held(weights(20, 64), 32)
    with pytest.raises(Exception, match="SKIM_ERR_WORKSPACE"):
        c.grouped_matvec(q, torch.zeros((2, 64), dtype=torch.float16, device="cuda"))
    c.close()
