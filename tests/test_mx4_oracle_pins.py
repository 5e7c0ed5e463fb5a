"""Pins of the MXFP4 and RMS norm oracle against hand-worked values, and the
refusals of the entry points (which need no GPU)."""
import numpy as np
import pytest

import paper_2603_04359_amd as cat
from oracle import mx4_oracle as mo
from paper_2603_04359_amd import binding as B

P = 1 << 20         # fake aligned address: the calls below fail before using it


def _block(*head):
    x = np.zeros((1, 32))
    x[0, :len(head)] = head
    return x


def test_every_level_and_tie():
    # amax 6: e = 2 - 2 = 0, so the elements are rounded to the levels as they are
    vals = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -5.0, 0.2500001, 4.9999, 5.0001, -0.0]
    want = [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -0.0, -1.0, -4.0, 0.5, 4.0, 6.0, -0.0]
    c, s = mo.quantize(_block(*vals))
    assert s[0, 0] == 127
    assert mo.dequantize(c, s)[0, :len(want)].tolist() == want
    assert c[0, 0] == 7 + 16 * 0 and c[0, 4] == 8 + 16 * 10      # -0.25 keeps its sign


@pytest.mark.parametrize("amax,byte,top", [(7.99, 127, 6.0), (8.0, 128, 8.0), (4.0, 127, 4.0),
                                           (3.99, 126, 3.0), (1.0, 125, 1.0),
                                           (2.0 ** -125, 0, 2.0 ** -125),
                                           (2.0 ** -126, 0, 2.0 ** -126), (2.0 ** -128, 0, 2.0 ** -128),
                                           (2.0 ** -130, 0, 0.0), (0.0, 0, 0.0),
                                           (3e38, 252, 1.5 * 2.0 ** 127)])
def test_scale_byte(amax, byte, top):
    c, s = mo.quantize(_block(amax))
    assert s[0, 0] == byte
    assert mo.dequantize(c, s)[0, 0] == top


def test_non_finite_block_is_nan_and_leaves_others():
    x = np.ones((1, 96))
    x[0, 5], x[0, 40] = np.inf, np.nan
    c, s = mo.quantize(x)
    assert s.tolist() == [[255, 255, 125]]
    v = mo.dequantize(c, s)[0]
    assert np.isnan(v[:64]).all() and (v[64:] == 1.0).all()


def test_round_trip_is_idempotent():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((7, 96)) * np.exp(3 * rng.standard_normal((7, 1)))
    v = mo.dequantize(*mo.quantize(x))
    c2, s2 = mo.quantize(v)
    assert np.array_equal(mo.dequantize(c2, s2), v)


def test_grouped_is_linear_per_group():
    rng = np.random.default_rng(1)
    cx, sx = mo.quantize(rng.standard_normal((9, 64)))
    cw, sw = zip(*(mo.quantize(rng.standard_normal((5, 64))) for _ in range(3)))
    cw, sw = np.stack(cw), np.stack(sw)
    y, _ = mo.linear_grouped(cx, sx, [1, 4, 4, 8], cw, sw, 9)
    x, w = mo.dequantize(cx, sx), mo.dequantize(cw, sw)
    assert np.isnan(y[[0, 8]]).all()
    assert np.allclose(y[1:4], x[1:4] @ w[0].T) and np.allclose(y[4:8], x[4:8] @ w[2].T)


def test_rmsnorm_by_hand():
    h, y = mo.rmsnorm([[3.0, 4.0]], [1.0, 2.0], [[0.0, 0.0]], eps=0.0)
    r = 1 / np.sqrt(12.5)
    assert np.allclose(y, [[3 * r, 8 * r]], rtol=1e-15)
    q, s = mo.quantize_int8(np.float32([[1.0, -127.0, 0.5, 1.5], [0, 0, 0, 0]]))
    assert q.tolist() == [[1, -127, 0, 2], [0, 0, 0, 0]] and s.tolist() == [1.0, 0.0]


# ---------------------------------------------------------------- refusals
def _err(rc, code, word=None):
    assert rc == code
    if word:
        assert word in cat.cat_last_error()


@pytest.mark.parametrize("fn", ["cat_rmsnorm_quant", "cat_rmsnorm_mx4"])
def test_rmsnorm_refusals(fn):
    f = getattr(cat.lib(), fn)
    ok = dict(x=P, xd=1, n=2, d=64, r=P, ro=P, w=P, wd=1, eps=1e-6, c=P, s=P)

    def call(**kw):
        a = dict(ok, **kw)
        return f(a["x"], a["xd"], a["n"], a["d"], a["r"], a["ro"], a["w"], a["wd"], a["eps"], a["c"],
                 a["s"], None)
    inv = B.CAT_ERR_INVALID_ARG
    for name in ("x", "w", "c", "s"):
        _err(call(**{name: None}), inv, "NULL")
    _err(call(r=None), inv, "together")
    _err(call(ro=None), inv, "together")
    _err(call(xd=2), inv, "dtype")
    _err(call(wd=-1), inv, "dtype")
    _err(call(n=0), inv)
    _err(call(d=0), inv)
    for eps in (-1e-9, float("nan"), float("inf")):
        _err(call(eps=eps), inv, "eps")
    for name in ("x", "r", "ro", "w", "c", "s"):
        _err(call(**{name: P + 8}), inv, "aligned")
    if fn == "cat_rmsnorm_mx4":
        _err(call(d=48), inv, "32")


def test_mx4_convert_refusals():
    L, inv = cat.lib(), B.CAT_ERR_INVALID_ARG
    for q in (lambda x=P, t=1, n=2, d=64, c=P, s=P: L.cat_mx4_quant(x, t, n, d, c, s, None),
              lambda x=P, t=1, n=2, d=64, c=P, s=P: L.cat_mx4_dequant(c, s, n, d, x, t, None)):
        _err(q(x=None), inv, "NULL")
        _err(q(c=None), inv, "NULL")
        _err(q(s=None), inv, "NULL")
        _err(q(t=3), inv, "dtype")
        _err(q(n=0), inv)
        _err(q(d=0), inv)
        _err(q(d=80), inv, "32")
        _err(q(x=P + 4), inv, "aligned")
        _err(q(c=P + 4), inv, "aligned")
        _err(q(s=P + 1), inv, "aligned")


def test_mx4_linear_refusals():
    L, inv, uns = cat.lib(), B.CAT_ERR_INVALID_ARG, B.CAT_ERR_UNSUPPORTED
    ok = dict(cx=P, ex=P, cw=P, ew=P, n=4, k=64, o=8, y=P, t=0)

    def call(**kw):
        a = dict(ok, **kw)
        return L.cat_mx4_linear(a["cx"], a["ex"], a["cw"], a["ew"], a["n"], a["k"], a["o"], a["y"],
                                a["t"], None)
    for name in ("cx", "ex", "cw", "ew", "y"):
        _err(call(**{name: None}), inv, "NULL")
        _err(call(**{name: P + 2}), inv, "aligned")
    for name in ("n", "k", "o"):
        _err(call(**{name: 0}), inv)
        _err(call(**{name: -32}), inv)
    _err(call(k=48), inv, "32")
    _err(call(t=7), inv, "dtype")
    _err(call(k=B.CAT_MAX_D_IN + 32), uns)
    _err(call(n=2 ** 30 + 1), uns)
    _err(call(o=2 ** 30 + 1), uns)


def test_mx4_grouped_refusals():
    L, inv, uns = cat.lib(), B.CAT_ERR_INVALID_ARG, B.CAT_ERR_UNSUPPORTED
    ok = dict(cx=P, ex=P, n=4, ids=P, m=6, off=P, g=2, cw=P, ew=P, k=64, o=8, y=P, t=0)

    def call(**kw):
        a = dict(ok, **kw)
        return L.cat_mx4_linear_grouped(a["cx"], a["ex"], a["n"], a["ids"], a["m"], a["off"], a["g"],
                                        a["cw"], a["ew"], a["k"], a["o"], a["y"], a["t"], None)
    for name in ("cx", "ex", "off", "cw", "ew", "y"):
        _err(call(**{name: None}), inv, "NULL")
    for name in ("cx", "ex", "ids", "off", "cw", "ew", "y"):
        _err(call(**{name: P + 4}), inv, "aligned")
    for name in ("n", "m", "g", "k", "o"):
        _err(call(**{name: 0}), inv)
    _err(call(g=B.CAT_MAX_GROUPS + 1), inv, "groups")
    _err(call(ids=None), inv, "row_ids")        # 6 rows of y from 4 of codes_x
    _err(call(m=2 ** 30 + 1), uns)
    _err(call(k=B.CAT_MAX_D_IN + 32), uns)


def test_binding_refuses_cpu_tensors_and_wrong_types():
    torch = pytest.importorskip("torch")
    u8 = torch.zeros(2, 32, dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        cat.cat_mx4_quant(torch.zeros(2, 64), u8, u8)
    with pytest.raises(TypeError, match="tensor"):
        cat.cat_mx4_dequant([1], u8, torch.zeros(2, 64))
    with pytest.raises(ValueError, match="required"):
        cat.cat_mx4_quant(None, u8, u8)
