"""The norm where values are not finite, or their squares leave the binary32 range, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import grouped

pytestmark = pytest.mark.gpu

HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}      # half a step, relative
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}    # half the smallest step

# rows and columns that take the kernel's forms: one, two and four pieces a thread, rows read again, whole pieces and odd ones
SHAPES = [(9, 7), (9, 100), (9, 512), (9, 9000), (300, 8192), (300, 5000), (9, 40001), (9, 40000)]


def rows_of(values, dtype):
    return torch.from_numpy(np.asarray(values, dtype=np.float64)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_eight_bit_rows_say_that_they_are_not_finite(ctx, rows, cols, dtype):
    """Infinities and NaN in x, in the residual and in the weight, under weights of 0 too: the row's scale is not finite, so none of its values is."""
    rng = np.random.default_rng([rows, cols])
    x, r = rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols))
    w = 1 + 0.2 * rng.standard_normal(cols)
    zero, last = cols // 2, cols - 1
    w[zero] = 0.0
    x[1, zero], x[2, zero], r[3, zero], x[4, last], r[5, 0] = np.nan, np.inf, -np.inf, np.inf, np.nan
    x[6, 1], r[6, 1] = np.inf, -np.inf
    bad = np.zeros(rows, bool)
    bad[1:7] = True
    X, R = rows_of(x, dtype), rows_of(r, dtype)
    for far, kind in ((None, None), (last, np.nan), (last, np.inf), (0, -np.inf)):
        weight = w.copy()
        expect = bad.copy()
        if far is not None:
            weight[far] = kind
            expect[:] = True
        for residual in (R, None):
            if residual is None and far is None:
                expect = bad & ~np.isin(np.arange(rows), (3, 5))
            out, scale, _ = ctx.add_rmsnorm(X, rows_of(weight, dtype), residual=residual, out_dtype=torch.int8)
            np.testing.assert_array_equal(~scale.isfinite().cpu().numpy(), expect)
            assert int(out.to(torch.int32).abs().max()) <= 127
            assert not bool((out.float() * scale[:, None])[torch.from_numpy(expect).cuda()].isfinite().any())
    # a weight that is infinite where the row is 0: their product is not a number
    x[:], weight = 0.0, np.ones(cols)
    x[:, 1], weight[0] = 1.0, np.inf
    out, scale, _ = ctx.add_rmsnorm(rows_of(x, dtype), rows_of(weight, dtype), out_dtype=torch.int8)
    assert bool(scale.isnan().all())


def far_rows(rows, cols, seed, eps):
    """Rows whose sum of squares leaves the binary32 range above (all values, one, only all together) or, with an eps that does not hide it, below; others between them."""
    rng = np.random.default_rng([seed, rows, cols])
    x = rng.standard_normal((rows, cols))
    kind = np.arange(rows) % 9
    x[kind == 1] *= 1e20
    x[kind == 2] *= 2.0 ** 126 / 6
    x[kind == 3, cols // 3] = -2e38
    x[kind == 4] = np.where(rng.random((int((kind == 4).sum()), cols)) < 0.5, 1, -1) * 2.0 ** (64 - np.log2(cols) / 2 + 1)
    x[kind == 5, cols - 1] = 3e19
    if eps < 1e-30:
        x[kind == 6] *= 1e-25
        x[kind == 7] *= 2.0 ** -131
        x[kind == 8] = 0.0
        x[kind == 8, cols // 2] = 2.0 ** -133
    else:
        x[kind == 8] = 0.0
    return rows_of(x, torch.bfloat16)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("eps", [1e-5, 0.0, 1e-38])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_squares_out_of_the_binary32_range(ctx, rows, cols, eps, eight):
    x = far_rows(rows, cols, 1, eps)
    w = rows_of(np.random.default_rng(2).uniform(0.5, 1.5, cols), torch.bfloat16)
    r = far_rows(rows, cols, 3, eps) * 0.25
    # the sum of squares as the norm's other test counts it, half of that in rstd, and a few products; a reciprocal root below 2^-126 (rows about 2^126)
    # has steps of 2^-149: half of one is at most 2^-21 of 2^-129
    rel = (8 * max(4, -(-cols // 8192)) + 10 + 12) * 2.0 ** -24 + 2.0 ** -21
    for residual, weight in ((None, w), (r, w), (r, None)):
        as_np = lambda t: None if t is None else t.float().cpu().numpy()
        eps32 = float(np.float32(eps))
        with np.errstate(over="ignore", invalid="ignore"):
            h, want, codes, scale = grouped.add_rmsnorm(as_np(x), as_np(residual), as_np(weight), eps32)
            p = (as_np(x) if residual is None else as_np(x) + as_np(residual)) * (np.float32(1) if weight is None else as_np(weight))
        over = np.isinf(p)                                   # products with the weight that leave the binary32 range: infinite, and so is or NaN the row's scale
        row_over = over.any(axis=1)
        assert np.isfinite(want).all() and np.isfinite(scale[~row_over]).all()
        held = None if residual is None else residual.clone()
        out, s, stream = ctx.add_rmsnorm(x, weight, eps=eps, residual=held, sum_out=held, out_dtype=torch.int8 if eight else None)
        if residual is not None:
            assert torch.equal(stream, (x.float() + residual.float()).to(torch.bfloat16))
        if eight:
            got = s.double().cpu().numpy()
            np.testing.assert_array_equal(out.cpu().numpy()[~row_over], codes[~row_over])
            np.testing.assert_allclose(got[~row_over], scale[~row_over], rtol=rel, atol=2.0 ** -149)
            assert not np.isfinite(got[row_over]).any()
        else:
            got = out.double().cpu().numpy()
            off = rel * np.abs(want)
            assert np.all((np.abs(got - want) <= off + HALF[torch.bfloat16] * (np.abs(want) + off) + TINY[torch.bfloat16]) | over)
            np.testing.assert_array_equal(got[over], p[over])
