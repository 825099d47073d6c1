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
