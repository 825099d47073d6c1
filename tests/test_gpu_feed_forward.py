"""The feed-forward half of a layer: odd sizes, results and room given, nothing to do, refusals; scales that are not finite; where results and scratch are made."""
import numpy as np
import pytest
import torch

from oracle import grouped
from test_gpu_grouped import HALF, TINY, ctx, held, norm_rows, oracle_feed_forward, token_rows, weights  # noqa: F401 (ctx: the fixture)

pytestmark = pytest.mark.gpu


def layer(cols, hidden, group):
    """(gate, up, down) in the stored form and their values"""
    made = [held(weights(*shape, n), group) for n, shape in ((1, (hidden, cols)), (2, (hidden, cols)), (3, (cols, hidden)))]
    return [m[0] for m in made], [m[1] for m in made]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("tokens,cols,hidden,group", [(1, 33, 7, 32), (3, 255, 701, 64), (19, 129, 300, 32), (40, 1001, 513, 128), (150, 520, 1111, 64)])
def test_odd_sizes_into_what_is_given(ctx, tokens, cols, hidden, group, eight, dtype):  # noqa: F811
    """Rows at odd addresses, the sum in place of the residual, the result between other values, scratch of the bytes named."""
    held_, (vg, vu, vd) = layer(cols, hidden, group)
    x, r = norm_rows(tokens, cols, dtype, 4, pad=3, shift=1), norm_rows(tokens, cols, dtype, 5, pad=5)
    w = (norm_rows(1, cols, dtype, 6, size=0.2)[0] + 1).contiguous()
    before = r.clone()
    plain, plain_stream = ctx.feed_forward(x, w, *held_, residual=before, eight_bit=eight, activation="gelu")
    need = ctx.feed_forward_bytes(tokens, cols, hidden)
    scratch = torch.full((need + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    room = torch.full((tokens + 1, cols + 4), 3.0, dtype=dtype, device="cuda")
    y, stream = ctx.feed_forward(x, w, *held_, residual=r, sum_out=r, out=room[:tokens, :cols], scratch=scratch[:need], eight_bit=eight, activation="gelu")
    assert stream is r and torch.equal(r, (x.float() + before.float()).to(dtype)) and torch.equal(plain_stream, r)
    assert y.data_ptr() == room.data_ptr() and torch.equal(y, plain)
    assert bool((room[:, cols:] == 3).all()) and bool((room[tokens] == 3).all()) and bool((scratch[need:] == 0xA5).all())
    as64 = lambda t: t.double().cpu().numpy()
    h, want, size = oracle_feed_forward(as64(x), as64(before), as64(w), vg, vu, vd, "gelu", eight, dtype)
    # as counted for the layer of whole pieces: the hidden rows' rounding, without 8 bits the normalised rows' too, the result's
    off = 2 * HALF[dtype] * size
    if not eight:
        rows = np.abs(grouped.add_rmsnorm(as64(x), as64(before), as64(w), 1e-5)[1])
        off = off + HALF[dtype] * (2.2 * ((rows @ np.abs(vg).T) * (rows @ np.abs(vu).T))) @ np.abs(vd).T * 1.1
    assert np.all(np.abs(as64(y) - want) <= off + HALF[dtype] * np.abs(want) + 1e-5 * size + TINY[dtype])


def test_a_vector_and_no_residual(ctx):  # noqa: F811
    held_, _ = layer(100, 60, 32)
    x = norm_rows(1, 100, torch.float16, 1)
    y, stream = ctx.feed_forward(x[0], None, *held_)
    want, _ = ctx.feed_forward(x, None, *held_)
    assert y.shape == (100,) and stream is None and torch.equal(y, want[0])
    total = torch.empty_like(x[0])
    again, stream = ctx.feed_forward(x[0], None, *held_, sum_out=total)
    assert stream is total and torch.equal(total, x[0]) and torch.equal(again, y)


def test_no_tokens(ctx):  # noqa: F811
    held_, _ = layer(100, 60, 32)
    x = torch.empty((0, 100), dtype=torch.bfloat16, device="cuda")
    for eight in (False, True):
        y, stream = ctx.feed_forward(x, None, *held_, residual=x, eight_bit=eight)
        assert y.shape == (0, 100) and stream.shape == (0, 100)
    assert ctx.feed_forward_bytes(0, 100, 60) == 0


def test_refused_before_anything_is_written(ctx):  # noqa: F811
    held_, _ = layer(96, 64, 32)
    x, r = norm_rows(5, 96, torch.float16, 1), norm_rows(5, 96, torch.float16, 2)
    before = r.clone()
    need = ctx.feed_forward_bytes(5, 96, 64)
    out = torch.full((5, 96), 3.0, dtype=torch.float16, device="cuda")
    room = torch.empty(need + 512, dtype=torch.uint8, device="cuda")
    for bad in (dict(scratch=room[:need - 1]), dict(scratch=room[128:128 + need]), dict(activation="relu"), dict(eps=-1.0), dict(eps=float("nan"))):
        with pytest.raises(Exception, match="SKIM_ERR"):
            ctx.feed_forward(x, None, *held_, residual=r, sum_out=r, out=out, **bad)
    gate, up, down = held_
    other = held(weights(64, 96), 64)[0]
    for bad in ((gate, up, gate), (down, up, down), (gate, other, down), (gate, up, held(weights(96, 65), 32)[0])):
        with pytest.raises(TypeError):
            ctx.feed_forward(x, None, *bad, residual=r, sum_out=r, out=out)
    with pytest.raises(TypeError):
        ctx.feed_forward(x, None, *held_, residual=r.bfloat16(), out=out)
    with pytest.raises(TypeError):
        ctx.feed_forward(x, None, *held_, out=out[:, :95])
    assert torch.equal(r, before) and bool((out == 3).all())


@pytest.mark.parametrize("tokens,rows,cols", [(4, 40, 300), (12, 100, 1000), (30, 50, 264), (300, 3001, 520)])
def test_scales_that_are_not_finite_stay_in_their_rows(ctx, tokens, rows, cols):  # noqa: F811
    w = weights(rows, cols)
    q = ctx.grouped_quantize(torch.from_numpy(w).cuda(), 64)
    x, _, xs = token_rows(tokens, cols, torch.int8)
    scale = torch.from_numpy(xs).cuda()
    clean, gate = ctx.grouped_matvec(q, x, x_scale=scale), ctx.grouped_gated(q, q, x, x_scale=scale)
    bad = scale.clone()
    bad[1], bad[3] = float("inf"), float("nan")
    keep = [t for t in range(tokens) if t not in (1, 3)]
    y, g = ctx.grouped_matvec(q, x, x_scale=bad), ctx.grouped_gated(q, q, x, x_scale=bad)
    assert torch.equal(y[keep], clean[keep]) and torch.equal(g[keep], gate[keep])
    assert bool(y[3].isnan().all()) and bool(g[3].isnan().all())
    # infinity times a sum of 0 is not a number, times any other one infinite with its sign
    whole = x[1].double() @ torch.from_numpy(grouped.values(*grouped.quantize(w, 64), 64)).cuda().t()
    assert not bool(y[1].isfinite().any()) and not bool(g[1].isfinite().any())
    sure = (whole.abs() > 1.0)
    assert torch.equal(torch.sign(y[1][sure]).double(), torch.sign(whole[sure])) and bool(y[1][sure].isinf().all())


def test_results_and_scratch_come_from_the_contexts_stream(skimlib):
    """Another stream is the current one: every tensor made by the calls, the room for a copy and the feed-forward's scratch among them, belongs to the context's
    stream, on which the kernels write it."""
    mine, other = torch.cuda.Stream(), torch.cuda.Stream()
    assert mine.cuda_stream != other.cuda_stream
    c = skimlib.Skim(device=0, stream=mine)
    c.set_workspace(torch.empty(4096, dtype=torch.uint8, device="cuda"))
    W = torch.from_numpy(weights(2000, 1000)).cuda()
    x, _, _ = token_rows(300, 1000, torch.float16, pad=3)
    held_, _ = layer(100, 60, 32)
    rows = norm_rows(70, 100, torch.float16, 1)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()

    def on(stream):
        return sorted((s["address"], s["total_size"], s["allocated_size"]) for s in torch.cuda.memory_snapshot() if s["stream"] == stream.cuda_stream)

    before = on(other)
    calls = torch.cuda.memory_stats()["allocation.all.allocated"]
    with torch.cuda.stream(other):
        q = c.grouped_quantize(W, 128, want_err=True)
        made = [q["tiles"], q["err"], c.grouped_dequantize(q), c.grouped_matvec(q, x), c.grouped_gated(q, q, x)]
        made += [t for t in c.add_rmsnorm(rows, residual=rows, out_dtype=torch.int8)] + list(c.feed_forward(rows, None, *held_, residual=rows))
    # ten results, two rooms for copies, one scratch
    assert torch.cuda.memory_stats()["allocation.all.allocated"] - calls == len(made) + 3
    assert on(other) == before
    segments = [s for s in torch.cuda.memory_snapshot() if s["stream"] == mine.cuda_stream]
    for t in made:
        assert any(s["address"] <= t.data_ptr() < s["address"] + s["total_size"] for s in segments)
    torch.cuda.synchronize()
    assert c.get_status() == 0
    c.close()
