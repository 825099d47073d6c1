"""Importances of the quantiser with group scales where no error is asked for, and errors asked for of a result that has no place for them."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx(skimlib):
    c = skimlib.Skim(device=0)
    c.set_workspace(torch.empty(4096, dtype=torch.uint8, device="cuda"))
    yield c
    c.close()


def test_bad_importances_are_reported_without_an_error_asked_for(ctx):
    W = torch.ones((20, 300), dtype=torch.float16, device="cuda")
    plain = ctx.grouped_quantize(W, 64)["tiles"]
    for bad in (None, float("nan"), float("inf"), -1.0):
        G = torch.ones((20, 300), device="cuda")
        if bad is not None:
            G[19, 299] = bad
        for out in (None, dict(tiles=torch.empty_like(plain), rows=20, cols=300, group=64, err=None), dict(tiles=torch.empty_like(plain), rows=20, cols=300, group=64)):
            q = ctx.grouped_quantize(W, 64, importance=G, out=out)
            assert torch.equal(q["tiles"], plain) and q.get("err") is None
            assert ctx.get_status() == (0 if bad is None else 2)


def test_an_error_asked_for_is_made_where_the_given_result_has_none(ctx):
    w = np.random.default_rng(1).standard_normal((20, 300)).astype(np.float16)
    W = torch.from_numpy(w).cuda()
    want = ctx.grouped_quantize(W, 64, want_err=True)
    for held in (dict(err=None), {}):
        out = dict(tiles=torch.empty_like(want["tiles"]), rows=20, cols=300, group=64, **held)
        got = ctx.grouped_quantize(W, 64, want_err=True, out=out)
        assert got is out and torch.equal(got["err"], want["err"]) and torch.equal(got["tiles"], want["tiles"])
