"""Pins of the oracle of the weights with group scales and of the norm, and the refusals of their calls (no GPU)."""
import ctypes as C

import numpy as np
import pytest

from oracle import grouped


def test_hand_worked_group():
    # low -0.5, high 1.0: s = 1.5 / 15 = 0.1 in binary16 = 0.0999755859375; z = rint(5.00122) = 5; 0.25 / s = 2.5006 -> 3, 1 / s = 10.0024 -> 10
    w = np.zeros((1, 32), np.float16)
    w[0, :4] = [-0.5, 1.0, 0.25, 0.0]
    codes, scale, zero = grouped.quantize(w, 32)
    assert float(scale[0, 0]) == 0.0999755859375 and zero[0, 0] == 5
    assert codes[0, :4].tolist() == [0, 15, 8, 5] and set(codes[0, 4:].tolist()) == {5}
    assert grouped.values(codes, scale, zero, 32)[0, :3].tolist() == [-5 * 0.0999755859375, 10 * 0.0999755859375, 3 * 0.0999755859375]


def test_values_are_within_half_a_step():
    w = (np.random.default_rng(0).standard_normal((40, 300)) * 0.02).astype(np.float16)
    for group in (32, 64, 128):
        codes, scale, zero = grouped.quantize(w, group)
        step = scale.astype(np.float64)[:, np.arange(300) // group]
        # half a step, where neither the scale's rounding (15 steps of 2^-11 relative) nor the zero point's clips the range
        off = np.abs(grouped.values(codes, scale, zero, group) - w.astype(np.float64))
        assert np.all(off <= step * (0.5 + 0.5 + 15 * 2.0 ** -11))
        assert np.mean(off <= 0.5 * step) > 0.95


def test_groups_of_one_sign_and_of_nothing():
    w = np.zeros((3, 64), np.float16)
    w[0] = 0.75                       # low stays 0: z = 0, the top code is the value
    w[1] = -0.75
    codes, scale, zero = grouped.quantize(w, 64)
    assert zero[:, 0].tolist() == [0, 15, 0] and codes[0, 0] == 15 and codes[1, 0] == 0 and codes[2, 0] == 0
    assert scale[2, 0] == 0 and not grouped.values(codes, scale, zero, 64)[2].any()


def test_stored_words():
    """Column e of the eight behind 32 t + 8 p lies in nibble 4 (e & 1) + e / 2 of word 16 i + 4 p + t."""
    codes = np.zeros((17, 130), np.int64)
    codes[1, 32 * 2 + 8 * 3 + 5] = 9
    codes[16, 129] = 7
    scale, zero = np.ones((17, 2), np.float16), np.full((17, 2), 4)
    words = grouped.store(codes, scale, zero, 128).view(np.uint32).reshape(2, 2, 272)
    assert words[0, 0, 16 * 1 + 4 * 3 + 2] == 9 << (4 * 6) and words[1, 1, 0] == 7 << 16
    assert words[0, 0, 256] == 0x3c00 | 4 << 16 and words[1, 0, 256] == 0x3c00 | 4 << 16 and words[1, 0, 257] == 0
    assert np.count_nonzero(words) == 2 + 17 * 2


def test_products_and_norm_by_hand():
    value = np.array([[1.0, -2.0], [0.5, 4.0]])
    y, size = grouped.product(value, np.array([[3.0, 1.0]]), np.array([2.0], np.float32))
    assert y.tolist() == [[2.0, 11.0]] and size.tolist() == [[10.0, 11.0]]
    assert grouped.activation("silu", np.array([0.0]))[0] == 0.0 and abs(grouped.activation("gelu", np.array([1.0]))[0] - 0.8411919906) < 1e-9
    h, out, codes, scale = grouped.add_rmsnorm(np.array([[3.0, 0.0]]), np.array([[0.0, 4.0]]), None, 0.0)
    assert h.tolist() == [[3.0, 4.0]] and np.allclose(out, np.array([[3.0, 4.0]]) / np.sqrt(12.5))
    assert codes.tolist() == [[95, 127]] and np.isclose(scale[0], 4 / np.sqrt(12.5) / 127)


# ---------------------------------------------------------------- refusals: found on the host, before anything is launched

NULL, SHAPE, WORKSPACE, ALIGN, TYPE = -1, -2, -5, -9, -11


@pytest.fixture(scope="module")
def lib():
    from paper_2412_04180_b200 import build, skim
    build.build()
    return skim.lib()


@pytest.fixture()
def handle():
    """A context of zeros: device 0, no workspace.  Calls end at the missing workspace at the latest."""
    buf = C.create_string_buffer(65536)
    return C.addressof(buf), buf


A = 4096      # an aligned address that is never read


def test_grouped_bytes(lib):
    from paper_2412_04180_b200.skim import Skim
    assert Skim.grouped_bytes(0, 1, 128) == 0
    assert Skim.grouped_bytes(16, 128, 128) == 1088 and Skim.grouped_bytes(17, 129, 64) == 4 * 1152 and Skim.grouped_bytes(1, 1, 32) == 1280
    n = C.c_size_t()
    assert lib.skim_grouped_bytes(1, 1, 32, None) == NULL
    for rows, cols, group, code in [(-1, 1, 32, SHAPE), (1, 0, 32, SHAPE), (1, 131073, 32, SHAPE), (1 << 31, 1, 32, SHAPE), (1, 1, 16, TYPE), (1, 1, 256, TYPE)]:
        assert lib.skim_grouped_bytes(rows, cols, group, C.byref(n)) == code


def test_quantize_and_dequantize_refusals(lib, handle):
    h = handle[0]
    f = lib.skim_grouped_quantize
    assert f(None, A, None, 4, 64, 64, 32, A, None) == NULL
    assert f(h, None, None, 4, 64, 64, 32, A, None) == NULL and f(h, A, None, 4, 64, 64, 32, None, None) == NULL
    assert f(h, A, None, 4, 64, 63, 32, A, None) == SHAPE and f(h, A, None, 4, 64, 64, 48, A, None) == TYPE
    assert f(h, A, None, 4, 64, 64, 32, A + 8, None) == ALIGN and f(h, A + 1, None, 4, 64, 64, 32, A, None) == ALIGN
    assert f(h, A, A + 2, 4, 64, 64, 32, A, None) == ALIGN and f(h, A, None, 4, 64, 64, 32, A, A + 2) == ALIGN
    assert f(h, A, A, 4, 64, 64, 32, A, A) == WORKSPACE
    f = lib.skim_grouped_dequantize
    assert f(h, None, 4, 64, 32, A, 64) == NULL and f(h, A, 4, 64, 32, None, 64) == NULL and f(None, A, 4, 64, 32, A, 64) == NULL
    assert f(h, A, 4, 64, 32, A, 63) == SHAPE and f(h, A, 4, 64, 33, A, 64) == TYPE and f(h, A, 4, 64, 32, A + 1, 64) == ALIGN


def test_product_refusals(lib, handle):
    h = handle[0]

    def both(code, ctx=h, tiles=A, rows=4, cols=64, group=32, act=0, x=A, xt=0, ldx=64, xs=None, tokens=2, y=A, yt=2, ldy=4):
        assert lib.skim_grouped_matvec(ctx, tiles, rows, cols, group, x, xt, ldx, xs, tokens, y, yt, ldy, None, 0) == code
        assert lib.skim_grouped_gated(ctx, A, tiles, rows, cols, group, act, x, xt, ldx, xs, tokens, y, yt, ldy, None, 0) == code
        assert lib.skim_grouped_gated(ctx, tiles, A, rows, cols, group, act, x, xt, ldx, xs, tokens, y, yt, ldy, None, 0) == code

    both(WORKSPACE)
    for bad in (dict(ctx=None), dict(tiles=None), dict(x=None), dict(y=None)):
        both(NULL, **bad)
    for bad in (dict(rows=-1), dict(cols=0), dict(cols=131073, ldx=1 << 30), dict(ldx=63), dict(ldy=3), dict(tokens=-1), dict(tokens=1048561)):
        both(SHAPE, **bad)
    for bad in (dict(group=0), dict(group=96), dict(xt=2), dict(xt=4), dict(xt=-1), dict(yt=3), dict(yt=-1)):
        both(TYPE, **bad)
    for bad in (dict(tiles=A + 8), dict(x=A + 1), dict(xt=1, x=A + 1), dict(y=A + 2), dict(yt=0, y=A + 1), dict(xs=A + 2)):
        both(ALIGN, **bad)
    for act in (-1, 2):
        assert lib.skim_grouped_gated(h, A, A, 4, 64, 32, act, A, 0, 64, None, 2, A, 2, 4, None, 0) == TYPE
    both(WORKSPACE, xt=3, x=A + 1, xs=A)


def test_scratch_bytes(lib, handle):
    """Bytes only where rows lie at odd addresses and there is work enough."""
    h, n = handle[0], C.c_size_t(7)
    f = lambda *a: (lib.skim_grouped_scratch_bytes(h, *a, C.byref(n)), n.value)
    assert f(4096, 4096, 128, 0, A, 0, 4096, 300) == (0, 0)                                # at multiples of 16 bytes
    assert f(4096, 4096, 128, 0, A, 0, 4099, 1) == (0, 0) and f(64, 64, 32, 0, A, 0, 67, 2) == (0, 0)
    assert f(4096, 4097, 128, 0, A, 0, 4099, 8) == (0, 8 * 4104 * 2) and f(4096, 4097, 64, 1, A + 1, 3, 4097, 8) == (0, 8 * 4112)
    assert f(4096, 4096, 128, 0, A, 3, 4104, 8) == (0, 0)                                  # 8 bytes are enough for few 8-bit rows
    assert lib.skim_grouped_scratch_bytes(h, 1, 1, 32, 0, A, 0, 1, 1, None) == NULL and lib.skim_grouped_scratch_bytes(None, 1, 1, 32, 0, A, 0, 1, 1, C.byref(n)) == NULL
    assert f(4, 64, 32, 0, A, 2, 64, 1)[0] == TYPE and f(4, 64, 48, 0, A, 0, 64, 1)[0] == TYPE
    assert f(4, 64, 32, 0, A, 0, 63, 1)[0] == SHAPE and f(4, 64, 32, 0, A, 0, 64, -1)[0] == SHAPE


def test_norm_refusals(lib, handle):
    h = handle[0]

    def f(ctx=h, x=A, ldx=64, r=None, ldr=0, w=None, kind=0, rows=2, cols=64, eps=1e-5, s=None, lds=0, out=A, ot=0, ldo=64, scale=None):
        return lib.skim_add_rmsnorm(ctx, x, ldx, r, ldr, w, kind, rows, cols, eps, s, lds, out, ot, ldo, scale)

    for bad in (dict(ctx=None), dict(x=None), dict(out=None), dict(ot=3)):
        assert f(**bad) == NULL
    for bad in (dict(rows=-1), dict(cols=0), dict(ldx=63), dict(ldo=63), dict(r=A, ldr=63), dict(s=A, lds=63), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert f(**bad) == SHAPE
    for bad in (dict(kind=2), dict(kind=3), dict(ot=1), dict(ot=2), dict(kind=1, ot=0)):
        assert f(**bad) == TYPE
    for bad in (dict(x=A + 1), dict(r=A + 1, ldr=64), dict(w=A + 1), dict(s=A + 1, lds=64), dict(out=A + 1), dict(ot=3, scale=A + 2)):
        assert f(**bad) == ALIGN


def test_feed_forward_refusals(lib, handle):
    h = handle[0]
    n = C.c_size_t()
    assert lib.skim_feed_forward_bytes(3, 100, 50, C.byref(n)) == 0 and n.value == 768 + 256 + 512
    assert lib.skim_feed_forward_bytes(3, 100, 50, None) == NULL and lib.skim_feed_forward_bytes(3, 0, 50, C.byref(n)) == SHAPE
    assert lib.skim_feed_forward_bytes(1048561, 100, 50, C.byref(n)) == SHAPE and lib.skim_feed_forward_bytes(3, 100, 131073, C.byref(n)) == SHAPE

    def f(ctx=h, x=A, ldx=100, r=None, ldr=0, w=None, kind=0, tokens=3, cols=100, hidden=50, eps=1e-5, gate=A, up=A, down=A, group=32, act=0, eight=1, scratch=A,
          size=1 << 20, s=None, lds=0, y=A, ldy=100):
        return lib.skim_feed_forward(ctx, x, ldx, r, ldr, w, kind, tokens, cols, hidden, eps, gate, up, down, group, act, eight, scratch, size, s, lds, y, ldy)

    assert f() == WORKSPACE
    for bad in (dict(ctx=None), dict(x=None), dict(gate=None), dict(up=None), dict(down=None), dict(scratch=None), dict(y=None)):
        assert f(**bad) == NULL
    for bad in (dict(tokens=-1), dict(cols=0), dict(hidden=0), dict(hidden=131073), dict(ldy=99)):
        assert f(**bad) == SHAPE
    for bad in (dict(kind=2), dict(kind=3), dict(act=2), dict(group=48)):
        assert f(**bad) == TYPE
    for bad in (dict(gate=A + 8), dict(up=A + 8), dict(down=A + 8), dict(y=A + 1)):
        assert f(**bad) == ALIGN


def test_every_refusal_has_words(lib):
    assert b"type" in lib.skim_strerror(TYPE)
