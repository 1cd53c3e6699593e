"""The router where a token's logits hold +inf or NaN: what is chosen, what becomes NaN, and that it stays in that token but for the loss."""
import pytest
import torch

import paper_2511_09323_amd as moc
from tests import test_gpu_route as RT

pytestmark = pytest.mark.gpu


# one lane a token and several, one workgroup and several
@pytest.mark.parametrize("T,E", [(40, 8), (600, 8), (40, 60), (600, 256)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("renorm", [False, True])
def test_infinities_and_nan(T, E, dtype, renorm):
    k, inf, nan = 3, float("inf"), float("nan")
    logits = RT.logits_of(T, E, dtype, T + E)
    odd = torch.zeros(T, dtype=torch.bool, device="cuda")
    odd[[3, 5, 7, 9, 11]] = True
    clean = moc.moc_route(logits, k, renorm=renorm)
    dw, dl = torch.randn(T, k, device="cuda"), torch.ones(1, device="cuda")
    logits[3, 2] = inf                                        # with other experts left
    logits[5], logits[5, 1] = -inf, inf                       # with none: two empty slots
    logits[7, 2] = nan
    logits[9], logits[9, 4], logits[9, 0] = -inf, 1.0, nan    # one expert, two empty slots
    logits[11], logits[11, 2] = -inf, 1.0                     # the same without a NaN
    r = moc.moc_route(logits, k, renorm=renorm)
    d = moc.moc_route_bwd(logits, r.ids, r.coef, dw, dl, renorm=renorm)
    ids, w = r.ids.tolist(), r.weights
    assert ids[3][0] == 2 and ids[5] == [1, -1, -1] and 2 not in ids[7] and -1 not in ids[7] and ids[9] == [4, -1, -1] and ids[11] == [2, -1, -1]
    # empty slots weigh nothing, whatever the token's softmax is
    assert not w[r.ids < 0].any() and not w[r.ids < 0].isnan().any()
    assert w[3].isnan().all() and w[5, 0].isnan()
    assert w[7].isnan().all() if not renorm else abs(float(w[7].sum()) - 1) < 1e-6
    assert w[9, 0].isnan() if not renorm else float(w[9, 0]) == 1.0
    assert float(w[11, 0]) == 1.0 and r.loss.isnan().all()
    assert d[[3, 5, 7, 9]].isnan().all() and not d[11].isnan().any()
    # the other tokens, and every count
    assert torch.equal(r.ids[~odd], clean.ids[~odd]) and torch.equal(r.weights[~odd], clean.weights[~odd]) and not d[~odd].isnan().any()
    assert int(r.counts.sum()) == int((r.ids >= 0).sum()) == 3 * T - 6 and not r.coef.isnan().any()
    live = r.order[r.order >= 0].long()
    assert live.numel() == 3 * T - 6 and (r.ids.view(-1)[live] >= 0).all()
