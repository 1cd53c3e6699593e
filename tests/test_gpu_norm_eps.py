"""The norms' gradients without an eps: rows that are not zero have a finite gradient, whatever the slots of a workgroup that have no row make of
theirs (1 / sqrt(0 + 0)).

Tolerances are test_gpu_norms's, whose bounds do not ask how large eps is: they are relative to r, and r only grows by leaving eps out."""
import pytest
import torch

import paper_2511_09323_amd as moc
from tests import test_gpu_norms as N

pytestmark = pytest.mark.gpu


# fewer rows than a workgroup takes at once, one more than a multiple of them, one less; rows that are narrow, odd, whole and wider than a wavefront's
@pytest.mark.parametrize("T", [1, 9, 255, 257])
@pytest.mark.parametrize("d", [3, 7, 96, 768, 1001, 2048, 4095, 4096])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_eps(T, d, dtype, monkeypatch):
    monkeypatch.setattr(N, "EPS", 0.0)
    a = N.make(T, d, dtype, 31 * T + d)
    N.check_forward(a, dtype, True, moc.moc_layernorm(a["h"], a["gain"], a["bias"], 0.0))
    N.check_backward(a, dtype, False, True, moc.moc_layernorm_bwd(a["h"], a["gain"], 0.0, a["dy"], dres=a["dres"]))
    N.check_backward(a, dtype, True, False, moc.moc_rmsnorm_bwd(a["h"], a["gain"], 0.0, a["dy"]))


def test_a_row_of_zeros_without_eps_is_nan_by_itself():
    """0 / 0 in its own row of dh, and in dgain, which sums over the rows; not in the other rows."""
    a = N.make(9, 512, "f32", 5)
    clean = moc.moc_rmsnorm_bwd(a["h"], a["gain"], 0.0, a["dy"])[0]
    a["h"][4] = 0
    dh, dgain = moc.moc_rmsnorm_bwd(a["h"], a["gain"], 0.0, a["dy"])
    keep = torch.arange(9, device="cuda") != 4
    assert dh[4].isnan().all() and dgain.isnan().all() and torch.equal(dh[keep], clean[keep])
