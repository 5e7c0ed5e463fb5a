"""The MXFP4 product over drawn shapes at every alignment of its rows, and the
MXFP4 and norm calls at buffers beyond 32-bit offsets.  Tolerance as in
test_gpu_mx4.py; results beyond 32-bit offsets are compared at sampled rows."""
import math
import random

import numpy as np
import pytest

from oracle import mx4_oracle as mo
from tests.gpu_common import say, torch_mod
from tests.test_gpu_mx4 import _assert_close, _cat, _codes, _dev

pytestmark = pytest.mark.gpu


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# 512: scale rows of whole 16 bytes; 128: of whole dwords; 32: at any byte.
# Below 512 elements the rows are too short for whole lines.
@pytest.mark.parametrize("unit,lo,hi", [(512, 512, 4096), (256, 512, 4096), (128, 512, 4096), (32, 512, 4096),
                                        (128, 128, 500), (32, 32, 500)])
@pytest.mark.parametrize("rows", [(1, 30), (30, 300), (300, 1500)])
def test_drawn_shapes(unit, lo, hi, rows):
    torch = torch_mod()
    rng = random.Random(unit * 7 + lo + rows[1])
    for it in range(4):
        d_in = max(lo, _log_int(rng, lo, hi) // unit * unit)
        d_out, m = _log_int(rng, 1, 900), _log_int(rng, *rows)
        grouped, seed = it % 2 == 1, rng.randrange(1 << 30)
        dt = rng.choice([torch.float32, torch.bfloat16])
        label = f"{'by expert ' if grouped else ''}{m}x{d_in}->{d_out} {dt}"
        say("  case", label)
        if grouped:
            groups = rng.choice([1, 3, 8])
            n = _log_int(rng, 1, 400)
            cuts = sorted(rng.randint(0, m) for _ in range(groups - 1))
            off = np.array([0] + cuts + [m], np.int32)
            ids = np.random.default_rng(seed).integers(0, n, m).astype(np.int32)
        else:
            groups, n, off, ids = 1, m, None, None
        cx, sx = _codes(n, d_in, seed, 118, 136)
        cw, sw = _codes(groups * d_out, d_in, seed + 1, 118, 136)
        y = torch.full((m, d_out), float("nan"), dtype=dt, device="cuda")
        if grouped:
            cw, sw = cw.reshape(groups, d_out, -1), sw.reshape(groups, d_out, -1)
            _cat().cat_mx4_linear_grouped(_dev(cx), _dev(sx), _dev(off), _dev(cw), _dev(sw), y, row_ids=_dev(ids))
            ref, absum = mo.linear_grouped(cx, sx, off, cw, sw, m, ids)
        else:
            _cat().cat_mx4_linear(_dev(cx), _dev(sx), _dev(cw), _dev(sw), y)
            ref, absum = mo.linear(cx, sx, cw, sw)
        _assert_close(y, ref, absum, d_in, label)


@pytest.mark.parametrize("d_in,d_out,m", [(544, 300, 700), (1056, 520, 260), (4128, 40, 20), (8160, 700, 300)])
def test_scales_at_the_end_of_their_buffer(d_in, d_out, m):
    # scale bytes that end a buffer at every remainder modulo 4, with NaN
    # bytes behind them: none may reach a result
    torch = torch_mod()
    for extra in range(4):
        cx, sx = _codes(m + extra, d_in, extra)
        cw, sw = _codes(d_out + extra, d_in, 7 + extra)
        pads = [torch.full((a.size + 64,), 255, dtype=torch.uint8, device="cuda") for a in (sx, sw)]
        views = []
        for pad, a in zip(pads, (sx, sw)):
            pad[:a.size] = _dev(a.reshape(-1))
            views.append(pad[:a.size].view(a.shape))
        y = torch.empty(m + extra, d_out + extra, device="cuda")
        _cat().cat_mx4_linear(_dev(cx), views[0], _dev(cw), views[1], y)
        _assert_close(y, *mo.linear(cx, sx, cw, sw), d_in, f"{m + extra}x{d_in}->{d_out + extra}")


# Sizes at which the products take 128 x 128, 128 x 256 and 256 x 256 outputs a
# workgroup: whole and general rows, last row and output tiles partly filled,
# outputs at 2-byte addresses; by expert with gathered rows, experts without
# rows, and rows before the first and behind the last expert left alone.
@pytest.mark.parametrize("n,d_in,d_out", [(700, 544, 3001), (600, 1024, 2047), (1300, 2080, 3003),
                                          (1300, 2048, 3002), (2000, 544, 5001), (2000, 1024, 4999)])
@pytest.mark.parametrize("grouped", [False, True])
def test_large_tiles(n, d_in, d_out, grouped):
    torch = torch_mod()
    cw, sw = _codes(d_out, d_in, 3, 118, 136)
    if not grouped:
        cx, sx = _codes(n, d_in, 2, 118, 136)
        ref, absum = mo.linear(cx, sx, cw, sw)
        for dt in (torch.float32, torch.bfloat16):
            y = torch.full((n, d_out), float("nan"), dtype=dt, device="cuda")
            _cat().cat_mx4_linear(_dev(cx), _dev(sx), _dev(cw), _dev(sw), y)
            _assert_close(y, ref, absum, d_in, f"{n}x{d_in}->{d_out} {dt}")
        return
    # the experts' weights are the same rows, rotated, so that one product
    # holds every reference value
    groups, shift, tokens = 4, 37, 150
    cx, sx = _codes(tokens, d_in, 2, 118, 136)
    full, full_abs = mo.linear(cx, sx, cw, sw)
    cws, sws = (np.stack([np.roll(v, g * shift, 0) for g in range(groups)]) for v in (cw, sw))
    off = np.array([5, n // 3, n // 3, n - 140, n - 3], np.int32)
    ids = np.random.default_rng(n).integers(0, tokens, n).astype(np.int32)
    of = np.searchsorted(off, np.arange(5, n - 3), side="right") - 1
    ref = np.stack([np.roll(full[ids[i]], of[i - 5] * shift) for i in range(5, n - 3)])
    absum = np.stack([np.roll(full_abs[ids[i]], of[i - 5] * shift) for i in range(5, n - 3)])
    for dt in (torch.float32, torch.bfloat16):
        y = torch.full((n, d_out), 7.0, dtype=dt, device="cuda")
        _cat().cat_mx4_linear_grouped(_dev(cx), _dev(sx), _dev(off), _dev(cws), _dev(sws), y, row_ids=_dev(ids))
        assert (y[:5] == 7).all() and (y[n - 3:] == 7).all()
        _assert_close(y[5:n - 3], ref, absum, d_in, f"by expert {n}x{d_in}->{d_out} {dt}")


# --------------------------------------------------------- beyond 32-bit offsets
def _random_codes(torch, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(sum(shape))
    codes = torch.randint(0, 256, shape, dtype=torch.uint8, device="cuda", generator=g)
    scales = torch.randint(115, 135, (*shape[:-1], shape[-1] // 16), dtype=torch.uint8, device="cuda", generator=g)
    return codes, scales


def _sampled(y, rows, cx, sx, src, cw, sw, d_in, label):
    ref, absum = mo.linear(cx[src].cpu().numpy(), sx[src].cpu().numpy(), cw.cpu().numpy(), sw.cpu().numpy())
    _assert_close(y[rows], ref, absum, d_in, label)


@pytest.mark.parametrize("d_in", [8192, 8224])
def test_linear_tokens_beyond_4_gib(d_in):
    torch = torch_mod()
    n, d_out = 2 ** 32 // (d_in // 2) + 1111, 72
    cx, sx = _random_codes(torch, n, d_in // 2)
    cw, sw = _random_codes(torch, d_out, d_in // 2)
    y = torch.empty(n, d_out, dtype=torch.bfloat16, device="cuda")
    _cat().cat_mx4_linear(cx, sx, cw, sw, y)
    rows = [0, 255, 256, n // 2, n - 1200, n - 257, n - 2, n - 1]
    _sampled(y, rows, cx, sx, rows, cw, sw, d_in, f"{n}x{d_in}->{d_out}")
    # the same rows gathered from both ends of the buffer, by expert
    ids = torch.tensor([n - 1, 0, n - 1, n - 1113, 5, n // 2] * 60, dtype=torch.int32, device="cuda")
    m = ids.numel()
    off = torch.tensor([0, 7, m], dtype=torch.int32, device="cuda")
    yg = torch.empty(m, d_out // 2, device="cuda")
    _cat().cat_mx4_linear_grouped(cx, sx, off, cw.view(2, d_out // 2, -1), sw.view(2, d_out // 2, -1), yg, row_ids=ids)
    src = [int(i) for i in ids[:16].tolist()]
    _sampled(yg, list(range(7)), cx, sx, src[:7], cw[:d_out // 2], sw[:d_out // 2], d_in, "gathered, first expert")
    _sampled(yg, list(range(7, 16)), cx, sx, src[7:], cw[d_out // 2:], sw[d_out // 2:], d_in, "gathered, second")


def test_grouped_weights_beyond_4_gib():
    torch = torch_mod()
    groups, d_out, d_in, m = 70, 16384, 8192, 333
    cw, sw = _random_codes(torch, groups, d_out, d_in // 2)
    assert cw.numel() > 2 ** 32
    cx, sx = _random_codes(torch, m, d_in // 2)
    off = torch.zeros(groups + 1, dtype=torch.int32, device="cuda")
    off[1:3], off[3:groups], off[groups:] = 3, 300, m      # experts 0, 2 and the last one
    y = torch.empty(m, d_out, dtype=torch.bfloat16, device="cuda")
    _cat().cat_mx4_linear_grouped(cx, sx, off, cw, sw, y)
    for rows, g in (([0, 2], 0), ([3, 299], 2), ([300, m - 1], groups - 1)):
        for cols in (slice(0, 64), slice(d_out - 64, d_out)):
            _sampled(y[:, cols], rows, cx, sx, rows, cw[g, cols], sw[g, cols], d_in, f"expert {g}")


@pytest.mark.parametrize("d_in", [512, 64])
def test_linear_outputs_beyond_4_gib(d_in):
    torch = torch_mod()
    n, d_out = 70001, 16400
    cx, sx = _random_codes(torch, n, d_in // 2)
    cw, sw = _random_codes(torch, d_out, d_in // 2)
    y = torch.empty(n, d_out, device="cuda")
    assert y.numel() * 4 > 2 ** 32
    _cat().cat_mx4_linear(cx, sx, cw, sw, y)
    rows = [0, 255, n // 2, n - 1]
    for cols in (slice(0, 70), slice(d_out - 70, d_out)):
        _sampled(y[:, cols], rows, cx, sx, rows, cw[cols], sw[cols], d_in, f"{n}x{d_in}->{d_out}")


def test_linear_more_tiles_than_one_launch_of_workgroups():
    # rows of 32 elements: more small tiles than a launch has workgroups
    torch = torch_mod()
    n, d_out, d_in = 36_000_001, 520, 32
    cx, sx = _random_codes(torch, n, d_in // 2)
    cw, sw = _random_codes(torch, d_out, d_in // 2)
    y = torch.empty(n, d_out, dtype=torch.bfloat16, device="cuda")
    _cat().cat_mx4_linear(cx, sx, cw, sw, y)
    rows = [0, 63, 64, n // 3, n // 2 + 5, n - 65, n - 1]
    _sampled(y, rows, cx, sx, rows, cw, sw, d_in, f"{n}x{d_in}->{d_out}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quant_and_norm_beyond_4_gib(dtype):
    torch = torch_mod()
    cat = _cat()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    n, d = 2 ** 32 // 8192 + 333, 8192
    x = torch.randn(n, d, device="cuda", dtype=dt)
    w = torch.ones(d, device="cuda", dtype=dt)
    c4 = torch.empty(n, d // 2, dtype=torch.uint8, device="cuda")
    s4 = torch.empty(n, d // 32, dtype=torch.uint8, device="cuda")
    rows = [0, 1, n // 2, n - 334, n - 1]
    xs = x[rows].float().cpu().numpy()
    cat.cat_mx4_quant(x, c4, s4)
    co, so = mo.quantize(xs)
    assert np.array_equal(c4[rows].cpu().numpy(), co) and np.array_equal(s4[rows].cpu().numpy(), so)
    out = torch.empty(n, d, device="cuda", dtype=torch.bfloat16)
    cat.cat_mx4_dequant(c4, s4, out)
    assert np.array_equal(out[rows].double().cpu().numpy(), mo.dequantize(co, so))
    del out
    ro = torch.empty_like(x)
    cat.cat_rmsnorm_mx4(x, w, c4, s4, residual=x, residual_out=ro, eps=1e-5)
    h, y = mo.rmsnorm_f32(xs, np.ones(d), xs, 1e-5)
    co, so = mo.quantize(y)
    assert np.array_equal(c4[rows].cpu().numpy(), co) and np.array_equal(s4[rows].cpu().numpy(), so)
    assert np.array_equal(ro[rows].float().cpu().numpy(), mo.round_bf16(h) if dtype == "bf16" else h)
    del c4, s4, ro
    c8 = torch.empty(n, d, dtype=torch.int8, device="cuda")
    s8 = torch.empty(n, device="cuda")
    cat.cat_rmsnorm_quant(x, w, c8, s8, eps=1e-5)
    q, s = mo.quantize_int8(mo.rmsnorm_f32(xs, np.ones(d), None, 1e-5)[1])
    assert np.array_equal(c8[rows].cpu().numpy(), q) and np.array_equal(s8[rows].cpu().numpy(), s)


def test_norm_of_more_rows_than_one_launch():
    # four lanes a row of 8 elements, 64 rows a workgroup: more than 2^31 threads
    torch = torch_mod()
    n, d = 2 ** 29 + 77, 8
    x = torch.randn(n, d, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(d, device="cuda", dtype=torch.bfloat16)
    c = torch.empty(n, d, dtype=torch.int8, device="cuda")
    s = torch.empty(n, device="cuda")
    _cat().cat_rmsnorm_quant(x, w, c, s, eps=1e-5)
    rows = [0, 63, 2 ** 28, 2 ** 29 - 1, 2 ** 29, 2 ** 29 + 13, n - 1]
    q, so = mo.quantize_int8(mo.rmsnorm_f32(x[rows].float().cpu().numpy(), np.ones(d), None, 1e-5)[1])
    assert np.array_equal(c[rows].cpu().numpy(), q) and np.array_equal(s[rows].cpu().numpy(), so)
