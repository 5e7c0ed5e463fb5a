"""MXFP4 products at the ends of the scales' range, on rows shorter than 512
elements, a few rows and large tiles, whole and general.

Subnormal sums are kept, so the bound of test_gpu_mx4.py holds down to fp32's
smallest number: a step of 2^-149 more covers its rounding.  A bf16 result adds
half a step, 2^-8 |y|, or of the smallest normal number, 2^-126 2^-8."""
import numpy as np
import pytest

from oracle import mx4_oracle as mo
from tests.gpu_common import say, torch_mod
from tests.test_gpu_mx4 import _cat, _codes, _dev

pytestmark = pytest.mark.gpu

# short rows; few rows, whole and general; large tiles, whole and general
SIZES = [(5, 256, 48), (70, 352, 200), (3, 512, 40), (7, 544, 90), (714, 512, 2699), (694, 640, 3425)]
TYPES = ["f32", "bf16"]


def _product(cx, sx, cw, sw, dtype):
    torch = torch_mod()
    y = torch.full((cx.shape[0], cw.shape[0]), 7.0, device="cuda",
                   dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
    _cat().cat_mx4_linear(_dev(cx), _dev(sx), _dev(cw), _dev(sw), y)
    return y.double().cpu().numpy()


def _bytes(rows, d_in, value):
    return np.full((rows, d_in // 32), value, np.uint8)


# products of 2^(bx + bw - 254): 1, large, small, and into fp32's subnormals
@pytest.mark.parametrize("bx,bw", [(0, 254), (254, 0), (1, 253), (254, 100), (90, 254), (254, 1), (0, 200), (60, 90),
                                   (0, 128), (127, 0), (58, 58), (20, 90)])
@pytest.mark.parametrize("n,d_in,d_out", SIZES)
def test_sums_in_range(n, d_in, d_out, bx, bw):
    cx, cw = _codes(n, d_in, 1)[0], _codes(d_out, d_in, 2)[0]
    sx, sw = _bytes(n, d_in, bx), _bytes(d_out, d_in, bw)
    ref, absum = mo.linear(cx, sx, cw, sw)
    tol = (d_in / 32 + 16) * 2.0 ** -23 * absum + 2.0 ** -149
    for dtype in TYPES:
        got = _product(cx, sx, cw, sw, dtype)
        bound = tol if dtype == "f32" else tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.maximum(np.abs(ref), 2.0 ** -126)
        err = np.abs(got - ref)
        say(f"  {n}x{d_in}->{d_out} {bx}+{bw} {dtype}: worst {float((err / bound).max()):.3g} of the bound,"
            f" zeros {int((got == 0).sum())} of {int((ref == 0).sum())}")
        assert np.isfinite(got).all() and (err <= bound).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d_in,d_out", SIZES)
def test_sums_beyond_the_range(n, d_in, d_out, dtype):
    # ones, with a sign a row and a sign an output: every product is 2^254
    cx, cw = np.full((n, d_in // 2), 0x22, np.uint8), np.full((d_out, d_in // 2), 0x22, np.uint8)
    cx[1::2] |= 0x88
    cw[::3] |= 0x88
    sign = np.where(np.arange(n) % 2 == 1, -1.0, 1.0)[:, None] * np.where(np.arange(d_out) % 3 == 0, -1.0, 1.0)
    got = _product(cx, _bytes(n, d_in, 254), cw, _bytes(d_out, d_in, 254), dtype)
    assert np.array_equal(got, sign * np.inf)
    # the smallest that are beyond it: 2^(254 + 127 - 254) (1 + 1) = 2^128
    cx[:] = 0
    cx[:, 0] = 0x22
    got = _product(cx, _bytes(n, d_in, 254), cw, _bytes(d_out, d_in, 127), dtype)
    assert np.array_equal(got, np.where(np.arange(d_out) % 3 == 0, -np.inf, np.inf)[None].repeat(n, 0))
    # 2^(254 + 127 - 254) alone is not
    cx[:, 0] = 0x02
    got = _product(cx, _bytes(n, d_in, 254), cw, _bytes(d_out, d_in, 127), dtype)
    assert np.array_equal(got, np.where(np.arange(d_out) % 3 == 0, -1.0, 1.0)[None].repeat(n, 0) * 2.0 ** 127)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d_in,d_out", SIZES)
def test_infinities_of_both_signs(n, d_in, d_out, dtype):
    # the second half of a row has the other sign, in parts of the sum that no
    # matrix step takes together.  Parts added in one accumulator, infinite by
    # then, leave it so (products are finite); parts of two waves meet as NaN
    cx, cw = np.full((n, d_in // 2), 0x22, np.uint8), np.full((d_out, d_in // 2), 0x22, np.uint8)
    cx[1:, d_in // 4:] |= 0x88
    got = _product(cx, _bytes(n, d_in, 254), cw, _bytes(d_out, d_in, 254), dtype)
    assert (got[0] == np.inf).all() and not np.isfinite(got[1:]).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d_in,d_out", SIZES)
@pytest.mark.parametrize("bx,bw", [(0, 0), (0, 40), (80, 1)])
def test_sums_below_the_range_are_zero(n, d_in, d_out, bx, bw, dtype):
    # |y| <= 36 d_in 2^(81 - 254) < 2^-150, half the smallest subnormal number
    cx, cw = _codes(n, d_in, 1)[0], _codes(d_out, d_in, 2)[0]
    got = _product(cx, _bytes(n, d_in, bx), cw, _bytes(d_out, d_in, bw), dtype)
    assert (got == 0).all()


@pytest.mark.parametrize("n,d_in,d_out", SIZES)
def test_nan_scale_beside_every_scale(n, d_in, d_out):
    # a NaN byte in a row of x reaches its row of y whatever it meets, and no
    # other: but beside 2^127 products, up to 36, go beyond the range on both
    # sides (4 2^127 2^0 does), so that rows may be NaN by themselves
    cx, cw = _codes(n, d_in, 1)[0], _codes(d_out, d_in, 2)[0]
    for bw in (0, 127, 254):
        sx, sw = _bytes(n, d_in, 127), _bytes(d_out, d_in, bw)
        sx[1, d_in // 32 - 1] = 255
        got = np.isnan(_product(cx, sx, cw, sw, "f32"))
        assert got[1].all() and (bw == 254 or not (got[0].any() or got[2:].any()))


@pytest.mark.parametrize("d_in", [32, 96, 160, 288, 352, 480, 544, 672])
@pytest.mark.parametrize("n,d_out", [(1, 1), (3, 5), (37, 43), (601, 507)])
def test_bytes_behind_a_scale_buffer_reach_no_result(n, d_out, d_in):
    # the scales' last word may be read past the buffer's end: NaN bytes there
    torch = torch_mod()
    cx, sx = _codes(n, d_in, 1, 118, 136)
    cw, sw = _codes(d_out, d_in, 2, 118, 136)
    views = []
    for a in (sx, sw):
        pad = torch.full((a.size + 64,), 255, dtype=torch.uint8, device="cuda")
        pad[:a.size] = _dev(a.reshape(-1))
        views.append(pad[:a.size].view(a.shape))
    y = torch.full((n, d_out), 7.0, device="cuda")
    _cat().cat_mx4_linear(_dev(cx), views[0], _dev(cw), views[1], y)
    ref, absum = mo.linear(cx, sx, cw, sw)
    assert (np.abs(y.double().cpu().numpy() - ref) <= (d_in / 32 + 16) * 2.0 ** -23 * absum).all()
