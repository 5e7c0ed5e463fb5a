"""MXFP4 quantization, its inverse and the product, dense and grouped,
against the fp64 oracle.

Codes, scale bytes and dequantized values are defined exactly (the division
by the scale is exact), so they are compared for equality.

Product tolerance: E2M1 products are multiples of 1/4 up to 36, so the 32
products of a block sum exactly in fp32 (13 bits); d_in / 32 block sums, and
at most 16 partial sums of them, are then added with an error of at most one
unit in the last place (2^-23) of a partial sum, itself at most S = sum
|products|: |y - y64| <= (d_in / 32 + 16) 2^-23 S, plus half a bf16 step
(2^-8 |y|) where y is bf16."""
import numpy as np
import pytest

from oracle import mx4_oracle as mo
from tests.gpu_common import say, torch_mod

pytestmark = pytest.mark.gpu


def _cat():
    import paper_2603_04359_amd as cat
    return cat


def _dev(a):
    return torch_mod().from_numpy(np.ascontiguousarray(a)).cuda()


def _to(x, dtype):
    """Device tensor in `dtype` and the host values it holds."""
    torch = torch_mod()
    if dtype == "bf16":
        x = mo.round_bf16(x)
        return _dev(np.float32(x)).to(torch.bfloat16), x
    return _dev(np.float32(x)), np.float32(x)


def _rows(n, d, seed, spread=1.0):
    rng = np.random.default_rng(seed)
    scale = np.exp(spread * rng.standard_normal(d))
    scale[rng.integers(0, d, 4)] *= 30
    return np.float32(rng.standard_normal((n, d)) * scale)


def _codes(n, d, seed, lo=115, hi=135):
    rng = np.random.default_rng(seed)
    return (rng.integers(0, 256, (n, d // 2), dtype=np.uint8),
            rng.integers(lo, hi, (n, d // 32), dtype=np.uint8))


# ------------------------------------------------------- quantize, dequantize
def _quantize(x_dev):
    torch = torch_mod()
    n, d = x_dev.shape
    c = torch.full((n, d // 2), 0xAB, dtype=torch.uint8, device="cuda")
    s = torch.full((n, d // 32), 0xCD, dtype=torch.uint8, device="cuda")
    _cat().cat_mx4_quant(x_dev, c, s)
    torch.cuda.synchronize()
    return c, s


def _check_quant(x_dev, x):
    c, s = _quantize(x_dev)
    co, so = mo.quantize(x)
    assert np.array_equal(s.cpu().numpy(), so)
    assert np.array_equal(c.cpu().numpy(), co)
    return c, s, co, so


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d", [(1, 32), (1, 4096), (3, 160), (33, 96), (257, 14336), (1000, 4128)])
def test_quant_and_dequant(n, d, dtype):
    torch = torch_mod()
    xd, x = _to(_rows(n, d, n + d), dtype)
    c, s, co, so = _check_quant(xd, x)
    want = mo.dequantize(co, so)
    for t in (torch.float32, torch.bfloat16):
        out = torch.empty(n, d, dtype=t, device="cuda")
        _cat().cat_mx4_dequant(c, s, out)
        assert np.array_equal(out.double().cpu().numpy(), want)


def test_quant_every_bf16_value():
    # all 65536 bit patterns, each once as the largest of its block and once
    # next to a larger element, NaN and infinity among them
    torch = torch_mod()
    bits = np.arange(65536, dtype=np.uint32) << 16
    v = bits.view(np.float32)
    x = np.zeros((65536, 64), np.float32)
    x[:, 3] = v
    x[:, 32:] = np.roll(v, 1)[:, None] * np.float32(0.7)
    x[:, 40] = v
    with np.errstate(invalid="ignore", over="ignore"):
        # NaN payloads: keep the pattern through the conversion
        xd = _dev(x).to(torch.bfloat16)
        _check_quant(xd, xd.float().cpu().numpy())


def test_quant_ties_and_levels_at_every_scale():
    # every multiple of 1/8 up to 8 next to an element that fixes the scale,
    # and one unit in the last place beside it on both sides
    grid = np.arange(-64, 65, dtype=np.float32) / 8
    u = np.concatenate([grid, np.nextafter(grid, np.float32(100)), np.nextafter(grid, np.float32(-100))])
    u = u[np.abs(u) < 8]
    u = np.concatenate([u, np.zeros(-len(u) % 31, np.float32)]).reshape(-1, 31)
    blk = np.concatenate([np.full((len(u), 1), 4, np.float32), u], 1)      # 4 <= amax < 8: scale 1
    x = np.concatenate([blk * np.float32(2.0 ** e) for e in (-124, -100, -20, -1, 0, 1, 20, 100, 124)])
    xd, xh = _to(x, "f32")
    _check_quant(xd, xh)


def test_quant_subnormal_and_zero():
    rng = np.random.default_rng(3)
    x = np.float32(rng.standard_normal((64, 64)))
    tiny = (x.astype(np.float64) * 2.0 ** -rng.integers(120, 152, (64, 1))).astype(np.float32)
    tiny[5] = 0
    tiny[6, ::2] = -0.0
    xd, xh = _to(tiny, "f32")
    _check_quant(xd, xh)


def test_dequant_every_code_and_scale():
    torch = torch_mod()
    codes = np.tile(np.arange(256, dtype=np.uint8), 256).reshape(256, 256)
    scales = np.repeat(np.arange(256, dtype=np.uint8), 16).reshape(256, 16)
    want = mo.dequantize(codes, scales)
    for t in (torch.float32, torch.bfloat16):
        out = torch.empty(256, 512, dtype=t, device="cuda")
        _cat().cat_mx4_dequant(_dev(codes), _dev(scales), out)
        got = out.double().cpu().numpy()
        with np.errstate(over="ignore"):
            # 2^127 times 2 or more exceeds both types' range
            assert np.array_equal(got, np.float32(want).astype(np.float64), equal_nan=True)


# ------------------------------------------------------------------- product
def _assert_close(y, ref, absum, d_in, label=""):
    got = y.double().cpu().numpy()
    tol = (d_in / 32 + 16) * 2.0 ** -23 * absum
    if "bfloat16" in str(y.dtype):
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref)
    err = np.abs(got - ref)
    worst = float((err / np.maximum(tol, 1e-300)).max())
    say(f"  {label}: worst error {worst:.3f} of the bound")
    assert np.isfinite(got).all() and worst <= 1.0


def _out(torch, m, d_out, dtype):
    # one guard row on each side
    buf = torch.full((m + 16, d_out), 7.0, dtype=dtype, device="cuda")
    return buf, buf[8:8 + m]


def _linear(n, d_in, d_out, dtype, seed=0, spread=(115, 135)):
    torch = torch_mod()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    cx, sx = _codes(n, d_in, seed, *spread)
    cw, sw = _codes(d_out, d_in, seed + 1, *spread)
    ref, absum = mo.linear(cx, sx, cw, sw)
    buf, y = _out(torch, n, d_out, dt)
    if y.data_ptr() % 16:
        buf = None
        y = torch.empty(n, d_out, dtype=dt, device="cuda")
    _cat().cat_mx4_linear(_dev(cx), _dev(sx), _dev(cw), _dev(sw), y)
    torch.cuda.synchronize()
    _assert_close(y, ref, absum, d_in, f"{n}x{d_in}->{d_out} {dtype}")
    if buf is not None:
        assert (buf[:8] == 7).all() and (buf[8 + n:] == 7).all()


# tokens from one to several tiles, outputs and reductions that end inside a tile
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d_in,d_out", [(32, 1), (64, 5), (96, 33), (256, 256), (1024, 100), (4128, 72),
                                        (4096, 512)])
@pytest.mark.parametrize("n", [1, 2, 7, 16, 17, 48, 130])
def test_linear_small(n, d_in, d_out, dtype):
    _linear(n, d_in, d_out, dtype)


@pytest.mark.parametrize("n,d_in,d_out", [(255, 512, 511), (256, 512, 512), (257, 544, 513),
                                          (300, 4096, 1030), (1025, 1056, 2050), (513, 8192, 520),
                                          (64, 14336, 4096), (2048, 256, 3000), (9, 131072, 40)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear_tiles(n, d_in, d_out, dtype):
    _linear(n, d_in, d_out, dtype, seed=5)


def test_linear_more_tiles_than_workgroups():
    # each workgroup then walks several tiles, the last round not full
    _linear(2500, 512, 9000, "bf16", seed=6)
    _linear(4096, 1024, 4500, "f32", seed=7)


@pytest.mark.parametrize("n,d_in,d_out", [(4, 512, 64), (300, 512, 512)])
def test_linear_wide_scale_range(n, d_in, d_out):
    # scales over 2^+-60: a block then dominates its row
    _linear(n, d_in, d_out, "f32", seed=9, spread=(67, 187))


@pytest.mark.parametrize("n,d_out", [(3, 40), (300, 600)])
def test_linear_extreme_scales(n, d_out):
    # scale bytes 0 against 254: products 2^(127 - 127) in the end
    torch = torch_mod()
    d_in = 512
    cx, sx = _codes(n, d_in, 1)
    cw, sw = _codes(d_out, d_in, 2)
    sx[:] = 0
    sw[:] = 252
    ref, absum = mo.linear(cx, sx, cw, sw)
    y = torch.empty(n, d_out, device="cuda")
    _cat().cat_mx4_linear(_dev(cx), _dev(sx), _dev(cw), _dev(sw), y)
    _assert_close(y, ref, absum, d_in, "bytes 0 x 252")


@pytest.mark.parametrize("n,d_in,d_out", [(5, 512, 48), (300, 1024, 520)])
def test_linear_nan_scale_reaches_its_row_and_column_only(n, d_in, d_out):
    torch = torch_mod()
    cx, sx = _codes(n, d_in, 1)
    cw, sw = _codes(d_out, d_in, 2)
    sx[n - 2, 3] = 255
    sw[7, d_in // 32 - 1] = 255
    cw[7, -16:] = 0                    # as the quantizer leaves them
    cx[n - 2, 48:64] = 0
    y = torch.empty(n, d_out, device="cuda")
    _cat().cat_mx4_linear(_dev(cx), _dev(sx), _dev(cw), _dev(sw), y)
    got = np.isnan(y.cpu().numpy())
    want = np.zeros((n, d_out), bool)
    want[n - 2] = True
    want[:, 7] = True
    assert np.array_equal(got, want)


def test_linear_repeats_bit_for_bit_and_permutes():
    torch = torch_mod()
    n, d_in, d_out = 300, 2048, 700
    cx, sx = _codes(n, d_in, 1)
    cw, sw = _codes(d_out, d_in, 2)
    args = [_dev(a) for a in (cx, sx, cw, sw)]
    y1, y2 = (torch.empty(n, d_out, device="cuda") for _ in range(2))
    _cat().cat_mx4_linear(*args, y1)
    _cat().cat_mx4_linear(*args, y2)
    assert torch.equal(y1, y2)
    p = np.random.default_rng(0).permutation(n)
    _cat().cat_mx4_linear(_dev(cx[p]), _dev(sx[p]), args[2], args[3], y2)
    assert torch.equal(y1[torch.from_numpy(p).cuda()], y2)


# ------------------------------------------------------------------- grouped
def _grouped(counts, d_in, d_out, dtype, gather, n=None, first=0, tail=0, seed=0):
    torch = torch_mod()
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    rng = np.random.default_rng(seed)
    groups = len(counts)
    offsets = np.concatenate([[first], first + np.cumsum(counts)]).astype(np.int32)
    m = int(offsets[-1]) + tail
    n = n or m
    cx, sx = _codes(n, d_in, seed)
    cw, sw = _codes(groups * d_out, d_in, seed + 1)
    cw, sw = cw.reshape(groups, d_out, -1), sw.reshape(groups, d_out, -1)
    ids = rng.integers(0, n, m).astype(np.int32) if gather else None
    ref, absum = mo.linear_grouped(cx, sx, offsets, cw, sw, m, ids)
    y = torch.full((m, d_out), 7.0, dtype=dt, device="cuda")
    _cat().cat_mx4_linear_grouped(_dev(cx), _dev(sx), _dev(offsets), _dev(cw), _dev(sw), y,
                                  row_ids=None if ids is None else _dev(ids))
    torch.cuda.synchronize()
    inside = slice(first, int(offsets[-1]))
    assert (y[:first] == 7).all() and (y[int(offsets[-1]):] == 7).all()
    if offsets[-1] > first:
        _assert_close(y[inside], ref[inside], absum[inside], d_in, f"{counts} {d_in}->{d_out}")


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("counts,d_in,d_out", [
    ([1], 32, 1), ([0, 1, 0], 64, 17), ([3, 0, 5, 1], 96, 40), ([16, 17, 15], 512, 64),
    ([0, 0, 0, 130], 1024, 100), ([1] * 70, 256, 33), ([200, 0, 63, 64, 65], 544, 260),
    ([300, 513, 1, 0, 256], 512, 520)])
def test_grouped(counts, d_in, d_out, dtype, gather):
    _grouped(counts, d_in, d_out, dtype, gather)


@pytest.mark.parametrize("counts", [[3, 0, 5], [300, 257]])
def test_grouped_leaves_rows_outside_the_experts(counts):
    _grouped(counts, 256, 264, "f32", False, first=3, tail=9)
    _grouped(counts, 256, 264, "bf16", True, first=3, tail=300, n=50)


def test_grouped_all_empty():
    _grouped([0, 0, 0], 256, 64, "f32", False, first=2, tail=3)


@pytest.mark.parametrize("groups", [64, 65, 1000])
def test_grouped_many_experts(groups):
    rng = np.random.default_rng(groups)
    _grouped(list(rng.integers(0, 4, groups)), 64, 24, "f32", True, n=37)
    c = [0] * groups
    c[groups // 2] = 40
    _grouped(c, 64, 24, "f32", False)


def test_grouped_same_row_for_every_expert():
    # one token routed to all experts, and each expert's rows equal the dense product
    torch = torch_mod()
    cat = _cat()
    groups, d_in, d_out = 5, 256, 48
    cx, sx = _codes(4, d_in, 1)
    cw, sw = _codes(groups * d_out, d_in, 2)
    ids = np.full(10, 2, np.int32)
    off = np.arange(0, 11, 2).astype(np.int32)
    y = torch.empty(10, d_out, device="cuda")
    cat.cat_mx4_linear_grouped(_dev(cx), _dev(sx), _dev(off), _dev(cw.reshape(groups, d_out, -1)),
                               _dev(sw.reshape(groups, d_out, -1)), y, row_ids=_dev(ids))
    dense = torch.empty(4, groups * d_out, device="cuda")
    cat.cat_mx4_linear(_dev(cx), _dev(sx), _dev(cw), _dev(sw), dense)
    want = dense[2].view(groups, d_out).repeat_interleave(2, 0)
    # sums may be taken in another order: each is within the product's bound
    ref, absum = mo.linear(cx[2:3], sx[2:3], cw, sw)
    tol = torch.from_numpy(2 * (d_in / 32 + 16) * 2.0 ** -23 * absum.reshape(groups, d_out)).cuda()
    assert ((y - want).abs() <= tol.repeat_interleave(2, 0)).all()


def test_grouped_bad_offsets_and_ids_stay_in_bounds():
    # values outside the documented ranges: rows undefined, buffers intact
    torch = torch_mod()
    groups, d_in, d_out, m = 3, 128, 40, 20
    cx, sx = _codes(m, d_in, 1)
    cw, sw = _codes(groups * d_out, d_in, 2)
    cw, sw = cw.reshape(groups, d_out, -1), sw.reshape(groups, d_out, -1)
    for off in ([0, 5, 3, 50], [-7, 4, 30, 10], [2 ** 31 - 1] * 4, [20, 15, 10, 0], [0, 20, 0, 20]):
        buf = torch.full((m + 64, d_out), 7.0, device="cuda")
        y = buf[32:32 + m]
        ids = _dev(np.array([-1, 2 ** 31 - 1, 0, 400] * 5, np.int32))
        _cat().cat_mx4_linear_grouped(_dev(cx), _dev(sx), _dev(np.array(off, np.int64).astype(np.int32)),
                                      _dev(cw), _dev(sw), y, row_ids=ids)
        torch.cuda.synchronize()
        assert (buf[:32] == 7).all() and (buf[32 + m:] == 7).all()


def test_grouped_bad_offsets_on_large_tiles():
    torch = torch_mod()
    groups, d_in, d_out, m = 8, 512, 600, 4000
    cx, sx = _codes(m, d_in, 1)
    cw, sw = _codes(groups * d_out, d_in, 2)
    cw, sw = _dev(cw.reshape(groups, d_out, -1)), _dev(sw.reshape(groups, d_out, -1))
    cx, sx = _dev(cx), _dev(sx)
    for off in ([0, 4000] * 4 + [0], [9, 5000, 3, -4, 4000, 10, 2 ** 31 - 1, 0, 77], [-2 ** 31] * 9):
        buf = torch.full((m + 64, d_out), 7.0, device="cuda")
        _cat().cat_mx4_linear_grouped(cx, sx, _dev(np.array(off, np.int64).astype(np.int32)), cw, sw,
                                      buf[32:32 + m])
        torch.cuda.synchronize()
        assert (buf[:32] == 7).all() and (buf[32 + m:] == 7).all()


# --------------------------------------------------------- streams and graphs
def test_capture_and_replay_with_other_routing():
    torch = torch_mod()
    cat = _cat()
    groups, d_in, d_out, m = 4, 256, 96, 64
    x = torch.empty(32, d_in, dtype=torch.bfloat16, device="cuda")
    cx = torch.empty(32, d_in // 2, dtype=torch.uint8, device="cuda")
    sx = torch.empty(32, d_in // 32, dtype=torch.uint8, device="cuda")
    cw, sw = (_dev(a.reshape(groups, d_out, -1)) for a in _codes(groups * d_out, d_in, 3))
    off = torch.zeros(groups + 1, dtype=torch.int32, device="cuda")
    ids = torch.zeros(m, dtype=torch.int32, device="cuda")
    y = torch.zeros(m, d_out, device="cuda")

    def step():
        cat.cat_mx4_quant(x, cx, sx)
        cat.cat_mx4_linear_grouped(cx, sx, off, cw, sw, y, row_ids=ids)
    x.copy_(torch.randn(32, d_in, device="cuda"))
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    rng = np.random.default_rng(0)
    for i in range(4):
        cuts = np.sort(rng.integers(0, m + 1, groups - 1))
        off.copy_(_dev(np.concatenate([[0], cuts, [m - i]]).clip(0, m - i).astype(np.int32)))
        ids.copy_(_dev(rng.integers(0, 32, m).astype(np.int32)))
        x.copy_(torch.randn(32, d_in, device="cuda"))
        y.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        got = y.clone()
        y.fill_(7.0)
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, y)
        assert (y[m - i:] == 7).all()


def test_another_stream():
    torch = torch_mod()
    cat = _cat()
    cx, sx, cw, sw = (_dev(a) for a in _codes(40, 512, 1) + _codes(72, 512, 2))
    want = torch.empty(40, 72, device="cuda")
    cat.cat_mx4_linear(cx, sx, cw, sw, want)
    torch.cuda.synchronize()
    for by_arg in (False, True):
        st = torch.cuda.Stream()
        y = torch.zeros(40, 72, device="cuda")
        st.wait_stream(torch.cuda.current_stream())
        if by_arg:
            cat.cat_mx4_linear(cx, sx, cw, sw, y, stream=st)
        else:
            with torch.cuda.stream(st):
                cat.cat_mx4_linear(cx, sx, cw, sw, y)
        st.synchronize()
        assert torch.equal(y, want)


# ---------------------------------------------------------------- refusals
def test_binding_refusals():
    torch = torch_mod()
    cat = _cat()

    def u8(*s):
        return torch.zeros(*s, dtype=torch.uint8, device="cuda")
    x = torch.zeros(4, 64, device="cuda")
    with pytest.raises(ValueError):
        cat.cat_mx4_quant(x, u8(4, 32), u8(4, 3))
    with pytest.raises(ValueError):
        cat.cat_mx4_quant(x.t(), u8(64, 2), u8(64, 1))
    with pytest.raises(TypeError):
        cat.cat_mx4_quant(x.double(), u8(4, 32), u8(4, 2))
    with pytest.raises(ValueError):
        cat.cat_mx4_quant(x[:, :48].contiguous(), u8(4, 24), u8(4, 1))
    with pytest.raises(ValueError):
        cat.cat_mx4_dequant(u8(4, 32), u8(5, 2), x)
    y = torch.zeros(4, 8, device="cuda")
    with pytest.raises(ValueError):
        cat.cat_mx4_linear(u8(4, 32), u8(4, 2), u8(8, 16), u8(8, 1), y)
    with pytest.raises(ValueError):
        cat.cat_mx4_linear(u8(4, 32), u8(4, 2), u8(8, 32), u8(8, 2), y[:3])
    with pytest.raises(TypeError):
        cat.cat_mx4_linear(u8(4, 32), u8(4, 2), u8(8, 32), u8(8, 2), y.half())
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        cat.cat_mx4_linear_grouped(u8(4, 32), u8(4, 2), off.long(), u8(2, 8, 32), u8(2, 8, 2), y)
    with pytest.raises(ValueError):
        cat.cat_mx4_linear_grouped(u8(4, 32), u8(4, 2), off[:2], u8(2, 8, 32), u8(2, 8, 2), y)
    with pytest.raises(ValueError):
        cat.cat_mx4_linear_grouped(u8(3, 32), u8(3, 2), off, u8(2, 8, 32), u8(2, 8, 2), y)
    with pytest.raises(ValueError):
        cat.cat_mx4_linear_grouped(u8(3, 32), u8(3, 2), off, u8(2, 8, 32), u8(2, 8, 2), y, row_ids=off)
    with pytest.raises(ValueError, match="GPU"):
        cat.cat_mx4_linear(u8(4, 32), u8(4, 2), u8(8, 32).cpu(), u8(8, 2), y)
