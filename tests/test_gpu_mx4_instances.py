"""Every kernel instance of the MXFP4 product, at rows, outputs and rows of x
that end inside its tiles, dense and by expert, in both output types.  Weights
repeat 131 rows, so that one product of those holds every reference value.
Tolerance as in test_gpu_mx4.py."""
import numpy as np
import pytest

from oracle import mx4_oracle as mo
from tests.gpu_common import torch_mod
from tests.mx4_cases import CASES
from tests.test_gpu_mx4 import _assert_close, _cat, _codes, _dev

pytestmark = pytest.mark.gpu
BASE = 131


@pytest.mark.parametrize("key,case", CASES, ids=lambda v: "-".join(map(str, v)))
def test_instance(key, case):
    torch = torch_mod()
    groups, n, m, d_in, d_out, gathered = case
    rng = np.random.default_rng(n + m + d_in + d_out)
    cx, sx = _codes(n, d_in, 2, 118, 136)
    cb, sb = _codes(BASE, d_in, 3, 118, 136)
    full, full_abs = mo.linear(cx, sx, cb, sb)
    base = [_dev(v) for v in (cb, sb)]
    dx = [_dev(v) for v in (cx, sx)]
    at = np.arange(max(groups, 1))[:, None] * 37 + np.arange(d_out)[None, :]
    of = torch.from_numpy(at % BASE).cuda()
    cw, sw = (v[of.view(-1)].view(*of.shape, -1) for v in base)
    if groups:
        # ragged experts, the second without rows, rows outside all of them
        first, tail = min(2, m - 1), 1 if m > 3 else 0
        cuts = np.sort(rng.integers(first, m - tail + 1, groups - 1))
        off = np.concatenate([[first], cuts, [m - tail]]).astype(np.int32)
        if groups > 2:
            off[2] = off[1]
        ids = rng.integers(0, n, m).astype(np.int32) if gathered else None
        inside = np.arange(first, m - tail)
        expert = np.searchsorted(off, inside, side="right") - 1
        src = ids[inside] if gathered else inside
    else:
        inside, expert, src = np.arange(m), np.zeros(m, int), np.arange(m)
    cols = at[expert] % BASE
    ref, absum = full[src[:, None], cols], full_abs[src[:, None], cols]
    for dt in (torch.float32, torch.bfloat16):
        y = torch.full((m, d_out), 7.0, dtype=dt, device="cuda")
        if groups:
            _cat().cat_mx4_linear_grouped(*dx, _dev(off), cw, sw, y, row_ids=None if ids is None else _dev(ids))
            assert (y[:first] == 7).all() and (y[m - tail:] == 7).all()
        else:
            _cat().cat_mx4_linear(*dx, cw[0], sw[0], y)
        _assert_close(y[int(inside[0]):int(inside[-1]) + 1], ref, absum, d_in, f"{key} {case} {dt}")
