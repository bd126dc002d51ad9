"""Layer of experts: both sides of the rule by which shares are added up.  Bounds as in
test_gpu_moe.py."""
import pytest
import torch

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
