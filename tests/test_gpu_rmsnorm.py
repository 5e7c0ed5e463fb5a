"""RMS norm with the residual's addition and quantized output against the
oracle.

Every rounding of the operator is stated (h, r and y in fp32, the sum of
squares in fp64), so codes, scales and the updated residual are compared for
equality with the oracle in the same roundings; fp64 sums in another order
differ by 2^-53 or so and move the fp32 r only next to a rounding border.
Against plain fp64: h, fl(h w), r and y carry four roundings of 2^-24, the
scale and the code factor up to six more, so a code lies within 1/2 + 127 *
10 * 2^-24 of y / s and s within 8 * 2^-24 of its value."""
import numpy as np
import pytest

from oracle import mx4_oracle as mo
from tests.gpu_common import torch_mod
from tests.test_gpu_mx4 import _cat, _dev, _rows, _to

pytestmark = pytest.mark.gpu


def _run(n, d, dtype, wdtype, residual, mx4, seed=0, eps=1e-5, x=None, w=None, res=None,
         inplace=None):
    torch = torch_mod()
    rng = np.random.default_rng(seed + 1)
    xd, x = _to(_rows(n, d, seed) if x is None else x, dtype)
    wd, w = _to(np.float32(1 + 0.2 * rng.standard_normal(d)) if w is None else w, wdtype)
    rd = ro = None
    if residual:
        rd, res = _to(_rows(n, d, seed + 2) if res is None else res, dtype)
        ro = torch.full_like(rd, 7.0)
        if inplace == "residual":
            ro = rd
        elif inplace == "x":
            ro = xd
    if mx4:
        c = torch.full((n, d // 2), 0xAB, dtype=torch.uint8, device="cuda")
        s = torch.full((n, d // 32), 0xCD, dtype=torch.uint8, device="cuda")
        _cat().cat_rmsnorm_mx4(xd, wd, c, s, residual=rd, residual_out=ro, eps=eps)
    else:
        c = torch.full((n, d), 0x55, dtype=torch.int8, device="cuda")
        s = torch.full((n,), 7.0, device="cuda")
        _cat().cat_rmsnorm_quant(xd, wd, c, s, residual=rd, residual_out=ro, eps=eps)
    torch.cuda.synchronize()
    return (x, w, res), c.cpu().numpy(), s.cpu().numpy(), None if ro is None else ro.float().cpu().numpy()


def _check(n, d, dtype, wdtype, residual, mx4, eps=1e-5, **kw):
    (x, w, res), c, s, ro = _run(n, d, dtype, wdtype, residual, mx4, eps=eps, **kw)
    h32, y32 = mo.rmsnorm_f32(x, w, res if residual else None, eps)
    if residual:
        assert np.array_equal(ro, mo.round_bf16(h32) if dtype == "bf16" else h32)
    _, y64 = mo.rmsnorm(x, w, res if residual else None, eps)
    if mx4:
        co, so = mo.quantize(y32)
        assert np.array_equal(s, so) and np.array_equal(c, co)
        # within half a step of the fp64 value, or beyond the largest level
        v, scale = mo.dequantize(c, s), np.repeat(np.exp2(s.astype(np.float64) - 127), 32, 1)
        u, near = np.abs(y64) / scale, 1e-6
        half = np.where(u < 2, 0.25, np.where(u < 4, 0.5, 1.0))
        assert ((np.abs(v - y64) / scale <= half + near) | ((u >= 6) & (np.abs(v) == 6 * scale))).all()
        assert (u < 8 * (1 + near)).all()
    else:
        qo, so = mo.quantize_int8(y32)
        assert np.array_equal(s, so) and np.array_equal(c, qo)
        s64 = np.abs(y64).max(1) / 127
        assert (np.abs(s - s64) <= 8 * 2.0 ** -24 * s64).all()
        u = y64 / np.where(s64 > 0, s64, 1)[:, None]
        assert (np.abs(c - u) <= 0.5 + 127 * 10 * 2.0 ** -24).all()


# rows of every kernel: one wave, one to four vectors a thread, the long
# rows; lengths that end inside a vector, a wave or a row's threads
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("n,d", [(1, 1), (3, 7), (5, 8), (9, 63), (6, 512), (7, 513), (2, 1000), (4, 2048),
                                 (3, 2049), (5, 4096), (2, 4104), (3, 8192), (2, 8201), (2, 14336),
                                 (2, 16392), (1, 32768), (2, 32769), (2, 40000), (257, 1024)])
def test_int8(n, d, residual, dtype):
    _check(n, d, dtype, dtype, residual, False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("n,d", [(1, 32), (9, 64), (6, 512), (7, 544), (4, 2048), (3, 2080), (5, 4096),
                                 (2, 4128), (3, 8192), (2, 14336), (1, 32768), (2, 32800), (1, 131072),
                                 (1003, 1024)])
def test_mx4(n, d, residual, dtype):
    _check(n, d, dtype, dtype, residual, True)


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("dtype,wdtype", [("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("d", [64, 4096, 36864])
def test_weight_of_the_other_type(d, dtype, wdtype, mx4):
    _check(5, d, dtype, wdtype, True, mx4)


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("inplace", ["residual", "x"])
@pytest.mark.parametrize("d", [96, 4096, 14336, 40960])
def test_in_place_residual(d, inplace, mx4):
    _check(3, d, "bf16", "bf16", True, mx4, inplace=inplace)


def test_in_place_residual_odd_rows():
    for d in (37, 5001, 33001):
        _check(3, d, "bf16", "bf16", True, False, inplace="residual")


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("d", [64, 4096, 33024])
def test_zero_rows_and_extremes(d, mx4):
    x = _rows(6, d, 1)
    x[0] = 0                                     # r from eps alone
    x[1] = 0
    x[1, 5] = 1e-20
    x[2] *= np.float32(1e30)                     # the sum of squares exceeds fp32
    x[3] *= np.float32(1e-18)
    w = np.float32(1 + 0.1 * np.random.default_rng(2).standard_normal(d))
    w[3] = 0
    _check(6, d, "f32", "f32", False, mx4, x=x, w=w)


@pytest.mark.parametrize("d", [64, 4096, 33024])
def test_zero_eps(d):
    x = _rows(3, d, 1)
    x[1] = 0                                     # mean 0 and eps 0: y = 0
    for mx4 in (False, True):
        _check(3, d, "f32", "f32", False, mx4, x=x, eps=0.0)


@pytest.mark.parametrize("d", [64, 4096, 4097, 33024])
def test_int8_non_finite_rows(d):
    x = _rows(5, d, 1)
    x[1, 3], x[3, d - 1], x[4, 0] = np.nan, np.inf, -np.inf
    (_, w, _), c, s, _ = _run(5, d, "bf16", "bf16", False, False, x=x)
    assert np.isnan(s[[1, 3, 4]]).all() and (c[[1, 3, 4]] == 0).all()
    ok = [0, 2]
    q, so = mo.quantize_int8(mo.rmsnorm_f32(mo.round_bf16(x[ok]), w, eps=1e-5)[1])
    assert np.array_equal(s[ok], so) and np.array_equal(c[ok], q)


@pytest.mark.parametrize("d", [64, 4096, 33024])
def test_mx4_non_finite_rows(d):
    # the whole row's norm is not finite; other rows are untouched
    x = _rows(4, d, 1)
    x[1, 3], x[2, d - 1] = np.nan, np.inf
    (_, w, _), c, s, _ = _run(4, d, "bf16", "bf16", False, True, x=x)
    assert (s[1:3] == 255).all() and (c[1:3] == 0).all()
    ok = [0, 3]
    co, so = mo.quantize(mo.rmsnorm_f32(mo.round_bf16(x[ok]), w, eps=1e-5)[1])
    assert np.array_equal(s[ok], so) and np.array_equal(c[ok], co)


def test_capture_and_replay():
    torch = torch_mod()
    cat = _cat()
    n, d = 33, 4096
    x, res = (torch.empty(n, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    c = torch.empty(n, d, dtype=torch.int8, device="cuda")
    s = torch.empty(n, device="cuda")
    ro = torch.empty_like(res)

    def step():
        cat.cat_rmsnorm_quant(x, w, c, s, residual=res, residual_out=ro)
    x.normal_(), res.normal_()
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        x.normal_(), res.normal_()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (c, s, ro)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (c, s, ro)))


def test_binding_refusals():
    torch = torch_mod()
    cat = _cat()
    x, w = torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    c, s = torch.zeros(4, 64, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    for bad in (dict(residual=x), dict(residual_out=x), dict(residual=x[:3], residual_out=x[:3])):
        with pytest.raises(ValueError):
            cat.cat_rmsnorm_quant(x, w, c, s, **bad)
    with pytest.raises(TypeError):
        cat.cat_rmsnorm_quant(x, w, c, s, residual=x.bfloat16(), residual_out=x.bfloat16())
    with pytest.raises(ValueError):
        cat.cat_rmsnorm_quant(x, w[:63].contiguous(), c, s)
    with pytest.raises(ValueError):
        cat.cat_rmsnorm_quant(x, w, c[:3], s)
    with pytest.raises(cat.CatError):
        cat.cat_rmsnorm_quant(x, w, c, s, eps=-1.0)
    with pytest.raises(ValueError):
        cat.cat_rmsnorm_mx4(x, w, torch.zeros(4, 32, dtype=torch.uint8, device="cuda"),
                            torch.zeros(4, 1, dtype=torch.uint8, device="cuda"))


def test_layer_of_experts_as_used():
    # residual + norm + MXFP4 codes, gathered up-projections of the routed
    # experts, their quantized outputs through the down-projections: every
    # step against the oracle on the codes the previous one left
    torch = torch_mod()
    cat = _cat()
    n, d, f, groups, topk = 37, 256, 416, 6, 2
    rng = np.random.default_rng(0)
    (xd, x), (rd, res), (wd, w) = (_to(_rows(n, d, 1), "bf16"), _to(_rows(n, d, 2), "bf16"),
                                   _to(np.ones(d, np.float32), "bf16"))
    up, down = (np.float32(rng.standard_normal((groups, o, i)) / np.sqrt(i)) for o, i in ((f, d), (d, f)))
    expert = np.argsort(rng.standard_normal((n, groups)), 1)[:, :topk].reshape(-1)
    order = np.argsort(expert, kind="stable")
    offsets = np.concatenate([[0], np.cumsum(np.bincount(expert, minlength=groups))]).astype(np.int32)
    ids, m = (order // topk).astype(np.int32), n * topk

    def codes(rows, cols):
        return (torch.empty(rows, cols // 2, dtype=torch.uint8, device="cuda"),
                torch.empty(rows, cols // 32, dtype=torch.uint8, device="cuda"))

    def weights(v):
        c, s = codes(v.shape[0] * v.shape[1], v.shape[2])
        cat.cat_mx4_quant(_dev(v.reshape(-1, v.shape[2])), c, s)
        return c.view(groups, v.shape[1], -1), s.view(groups, v.shape[1], -1)
    cu, su = weights(up)
    cd, sd = weights(down)
    cx, sx = codes(n, d)
    cat.cat_rmsnorm_mx4(xd, wd, cx, sx, residual=rd, residual_out=rd, eps=1e-5)
    a = torch.empty(m, f, dtype=torch.bfloat16, device="cuda")
    cat.cat_mx4_linear_grouped(cx, sx, _dev(offsets), cu, su, a, row_ids=_dev(ids))
    ca, sa = codes(m, f)
    cat.cat_mx4_quant(a, ca, sa)
    y = torch.empty(m, d, device="cuda")
    cat.cat_mx4_linear_grouped(ca, sa, _dev(offsets), cd, sd, y)
    torch.cuda.synchronize()

    h, yn = mo.rmsnorm_f32(x, w, res, 1e-5)
    co, so = mo.quantize(yn)
    assert np.array_equal(cx.cpu().numpy(), co) and np.array_equal(sx.cpu().numpy(), so)
    assert np.array_equal(rd.float().cpu().numpy(), mo.round_bf16(h))
    cuo, suo = (t.cpu().numpy() for t in (cu, su))
    ref, absum = mo.linear_grouped(co, so, offsets, cuo, suo, m, ids)
    got = a.double().cpu().numpy()
    tol = (d / 32 + 16) * 2.0 ** -23 * absum
    assert (np.abs(got - ref) <= tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)).all()
    co2, so2 = mo.quantize(got)
    assert np.array_equal(ca.cpu().numpy(), co2) and np.array_equal(sa.cpu().numpy(), so2)
    ref, absum = mo.linear_grouped(co2, so2, offsets, cd.cpu().numpy(), sd.cpu().numpy(), m)
    assert (np.abs(y.double().cpu().numpy() - ref) <= (f / 32 + 16) * 2.0 ** -23 * absum).all()


@pytest.mark.parametrize("d", [32, 63, 4096, 33024])
def test_int8_rows_below_the_quantizer_are_zero(d):
    # 127 / amax overflows for amax below 127 * 2^-128 = 3.73e-37: such a
    # token has a zero scale and zero codes; the next larger one is quantized
    x = np.ones((4, d), np.float32)
    x[:, 0] = -1
    x[1] *= 0.5
    x[2] = 0
    w = np.zeros(d, np.float32)
    w[:2] = np.float32(3e-37)                    # |y| 3e-37 (1 - 2^-24 or so)
    (_, _, _), c, s, _ = _run(4, d, "f32", "f32", False, False, x=x, w=w, eps=0.0)
    assert (c == 0).all() and (s == 0).all()
    w[1] = np.float32(-4e-37)
    (_, _, _), c, s, _ = _run(4, d, "f32", "f32", False, False, x=x, w=w, eps=0.0)
    q, so = mo.quantize_int8(mo.rmsnorm_f32(x, w, eps=0.0)[1])
    assert np.array_equal(c, q) and np.array_equal(s, so) and (c[[0, 1, 3], 1] == -127).all()
