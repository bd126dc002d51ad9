"""Layer of experts: both sides of the rule by which shares are added up, and rows beside one that is not finite.  Bounds as in
test_gpu_moe.py."""
import numpy as np
import pytest
import torch

from hgsynth import bf16_round
from tests.gpu_util import dev, lib, need_gpu, tdtype
from tests.test_gpu_moe import call, check, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,E,top,d,f", [(1, 9, 8, 256, 264), (1, 16, 2, 256, 1032), (1, 16, 3, 256, 136), (1, 5, 4, 128, 520),
                                         (1, 9, 5, 128, 40), (1, 8, 8, 64, 2056), (2, 2, 1, 256, 520), (2, 3, 2, 128, 264),
                                         (2, 4, 4, 64, 136), (2, 9, 5, 64, 24), (3, 1, 1, 64, 4104), (1, 2, 2, 128, 16384)])
def test_shares_added_by_the_last_cta_or_by_a_launch(dt, n, E, top, d, f):
    need_gpu()
    hg = lib()
    td = tdtype(dt)
    x, *ws = problem(dt, n, E, d, f, E + f)
    p, X = hg.MoeParams(*(dev(w, td) for w in ws), top, residual=True), dev(x, td)
    got = call(hg, p, X)
    check(dt, got, x, ws, top, "silu", True, True)
    again = call(hg, p, X)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_a_row_that_is_not_finite_leaves_the_others_bits(dt, bad):
    """Row 9 chooses experts 0 and 1 with and without its bad value (an infinity's logits go by the signs of its row of
    W_router, a NaN's are all NaN), so every list and every sum of the other rows is the same."""
    need_gpu()
    hg = lib()
    td, n, E, d, f = tdtype(dt), 50, 4, 128, 40
    x, wr, *ws = problem(dt, n, E, d, f, 6)
    wr[:, 0] += 30 * x[9] / (x[9] @ x[9])
    wr[:, 1] += 20 * x[9] / (x[9] @ x[9])
    wr[77] = 0.25, 0.25, -0.25, -0.25
    wr = bf16_round(wr.astype(np.float32)) if dt == "bf16" else wr.astype(np.float32)
    p = hg.MoeParams(*(dev(w, td) for w in (wr, *ws)), 2, residual=True)
    ref = call(hg, p, dev(x, td))
    check(dt, ref, x, (wr, *ws), 2, "silu", True, True)
    y = x.copy()
    y[9, 77] = bad
    got = call(hg, p, dev(y, td))
    assert ref[1][9].sort()[0].tolist() == got[1][9].sort()[0].tolist() == [0, 1]
    keep = torch.arange(n, device="cuda") != 9
    assert all(torch.equal(a[keep], b[keep]) for a, b in zip(got, ref))
    assert torch.isnan(got[0][9]).all() and torch.isnan(got[2][9]).all()
