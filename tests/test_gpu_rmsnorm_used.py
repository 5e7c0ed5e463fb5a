"""The norm's 8-bit codes as cat_int8_linear reads them, and the norm at every
number of threads a row takes.  Bounds and equalities as in
test_gpu_rmsnorm.py; the integer product is exact and its two products with the
scales are rounded as stated, so it is compared for equality."""
import numpy as np
import pytest

from oracle import cat_oracle as o
from oracle import mx4_oracle as mo
from tests.gpu_common import torch_mod
from tests.test_gpu_mx4 import _cat, _dev, _rows, _to
from tests.test_gpu_rmsnorm import _check

pytestmark = pytest.mark.gpu


# the first and last length of 4, 8, 16, 32 and 64 threads a row, of two and
# four vectors of 64 and 256 threads, and of 1024
@pytest.mark.parametrize("dtype,wdtype", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("d", [32, 33, 64, 65, 128, 129, 256, 257, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097,
                               8192, 8193, 16384, 16385, 32768, 32769])
def test_int8_first_and_last_length_of_every_shape(d, dtype, wdtype):
    _check(67 if d < 1024 else 3, d, dtype, wdtype, True, False)


@pytest.mark.parametrize("dtype,wdtype", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 256, 288, 512, 544, 1024, 1056, 2048, 2080, 4096, 4128, 8192,
                               8224, 16384, 16416, 32768, 32800])
def test_mx4_first_and_last_length_of_every_shape(d, dtype, wdtype):
    _check(67 if d < 1024 else 3, d, dtype, wdtype, True, True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d,d_out", [(1, 4096, 640), (5, 96, 33), (48, 1024, 515), (300, 2080, 700)])
def test_norm_codes_through_the_8_bit_product(n, d, d_out, dtype):
    # residual + norm + codes, times 8-bit weights: rows of zeros give zeros,
    # rows with a NaN or an infinity NaN, the others what the oracle gives
    torch = torch_mod()
    cat = _cat()
    x, res = _rows(n, d, 1), _rows(n, d, 2)
    bad, zero = [], []
    if n > 4:
        x[1, d - 1], res[3, 2] = np.nan, np.inf
        x[4], res[4] = 0, 0
        bad, zero = [1, 3], [4]
    (xd, x), (rd, res), (wd, w) = (_to(x, dtype), _to(res, dtype),
                                   _to(1 + 0.1 * np.random.default_rng(3).standard_normal(d), dtype))
    cw, sw = cat.cat_quantize_weights(np.random.default_rng(4).standard_normal((d_out, d)) / np.sqrt(d), 8)
    codes = torch.empty(n, d, dtype=torch.int8, device="cuda")
    s = torch.empty(n, device="cuda")
    y = torch.full((n, d_out), 7.0, device="cuda")
    cat.cat_rmsnorm_quant(xd, wd, codes, s, residual=rd, residual_out=rd, eps=1e-5)
    cat.cat_int8_linear(codes, s, _dev(cw), _dev(sw), y)
    got = y.cpu().numpy()
    ok = [i for i in range(n) if i not in bad]
    h, yn = mo.rmsnorm_f32(x[ok], w, res[ok], 1e-5)
    q, so = mo.quantize_int8(yn)
    assert np.array_equal(codes.cpu().numpy()[ok], q) and np.array_equal(s.cpu().numpy()[ok], so)
    assert np.array_equal(got[ok], o.w4a4_linear(q, so, cw, sw)[1])
    assert np.isnan(got[bad]).all() and (got[zero] == 0).all()
    assert np.array_equal(rd.float().cpu().numpy()[ok], mo.round_bf16(h) if dtype == "bf16" else h)


@pytest.mark.parametrize("d", [64, 4096, 33024])
def test_infinite_products_with_the_weight(d):
    # fl(h w) or y beyond fp32 with finite h: an 8-bit token is NaN, an MXFP4
    # token in that block only
    torch = torch_mod()
    cat = _cat()
    x = np.ones((3, d), np.float32)
    x[0, 40] = 4                                 # fl(4 * 3e38) is infinite, 3e38 is not
    x[1, 40] = 0.5
    x[2, 40] = 0
    w = np.ones(d, np.float32)
    w[40] = 3e38
    xd, wd = _dev(x), _dev(w)
    c8, s8 = torch.full((3, d), 7, dtype=torch.int8, device="cuda"), torch.zeros(3, device="cuda")
    cat.cat_rmsnorm_quant(xd, wd, c8, s8, eps=0.0)
    assert np.array_equal(torch.isnan(s8).cpu().numpy(), [True, False, False]) and (c8[0] == 0).all()
    q, so = mo.quantize_int8(mo.rmsnorm_f32(x[1:], w, eps=0.0)[1])
    assert np.array_equal(c8[1:].cpu().numpy(), q) and np.array_equal(s8[1:].cpu().numpy(), so)
    c4 = torch.empty(3, d // 2, dtype=torch.uint8, device="cuda")
    s4 = torch.empty(3, d // 32, dtype=torch.uint8, device="cuda")
    cat.cat_rmsnorm_mx4(xd, wd, c4, s4, eps=0.0)
    with np.errstate(over="ignore"):
        co, so = mo.quantize(mo.rmsnorm_f32(x, w, eps=0.0)[1])
    assert (so[0] == 255).sum() == 1 and so[0, 1] == 255
    assert np.array_equal(c4.cpu().numpy(), co) and np.array_equal(s4.cpu().numpy(), so)


def test_streams():
    # two streams at once, by argument and as the current one, on buffers of
    # their own: each result is the one stream's
    torch = torch_mod()
    cat = _cat()
    n, d, d_out = 200, 2048, 512
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    wf = torch.randn(d_out, d, device="cuda")
    cw = torch.empty(d_out, d // 2, dtype=torch.uint8, device="cuda")
    sw = torch.empty(d_out, d // 32, dtype=torch.uint8, device="cuda")
    cat.cat_mx4_quant(wf, cw, sw)
    xs = [torch.randn(n, d, device="cuda").bfloat16() for _ in range(2)]

    def step(x, out, stream):
        c, s, v, y, c8, s8 = out
        cat.cat_rmsnorm_mx4(x, w, c, s, stream=stream)
        cat.cat_mx4_dequant(c, s, v, stream=stream)
        cat.cat_mx4_quant(v, c, s, stream=stream)
        cat.cat_mx4_linear(c, s, cw, sw, y, stream=stream)
        cat.cat_rmsnorm_quant(x, w, c8, s8, stream=stream)

    def buffers():
        return (torch.zeros(n, d // 2, dtype=torch.uint8, device="cuda"),
                torch.zeros(n, d // 32, dtype=torch.uint8, device="cuda"),
                torch.zeros(n, d, device="cuda"), torch.zeros(n, d_out, device="cuda"),
                torch.zeros(n, d, dtype=torch.int8, device="cuda"), torch.zeros(n, device="cuda"))
    want, got = [buffers() for _ in range(2)], [buffers() for _ in range(2)]
    for x, out in zip(xs, want):
        step(x, out, None)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        step(xs[0], got[0], streams[0])
        with torch.cuda.stream(streams[1]):
            step(xs[1], got[1], None)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
