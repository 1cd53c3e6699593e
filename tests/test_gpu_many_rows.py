"""More rows than one launch has work-items for (2^32): a block of rows over and over gives what it gives on its own, over and over."""
import pytest
import torch

import paper_2511_09323_amd as moc
from tests import test_gpu_act8 as A8
from tests import test_gpu_norms as N
from tests import test_gpu_route as RT

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def repeated(block, times):
    return block.unsqueeze(0).expand(times, *block.shape).reshape(times * block.shape[0], *block.shape[1:])


def same(got, block, times):
    got = got.view(times, *block.shape)
    for part in got.split(64):
        assert torch.equal(part, block.unsqueeze(0).expand_as(part))


N_ROWS, TIMES = 1000003, 68      # 68 million rows; 64 lanes a row from 2^26 = 67.1 million on


def test_layernorm():
    a = N.make(N_ROWS, 8, "bf16", 1)
    h = repeated(a["h"], TIMES)
    same(moc.moc_layernorm(h, a["gain"], a["bias"], N.EPS, out=h), moc.moc_layernorm(a["h"], a["gain"], a["bias"], N.EPS), TIMES)


def test_act8_save_and_load():
    d, F, K = 8, 32, 1
    x, idx, g, u = A8.stored(N_ROWS, d, F, K, "bf16", 2)
    saved = moc.moc_act8_save(x, idx, g, u, F)
    many = tuple(repeated(t, TIMES) for t in (x, idx, g, u))
    all_saved = moc.moc_act8_save(*many, F)
    for a, b in zip(all_saved, saved):
        same(a, b, TIMES)
    for a, b in zip(moc.moc_act8_load(all_saved, F, torch.bfloat16, out=many), moc.moc_act8_load(saved, F, torch.bfloat16)):
        same(a, b, TIMES)


def test_route_bwd():
    """32 lanes a token from 129 experts on, 134 million tokens, 35 GB."""
    n, times, E = 131101, 1024, 129
    block = RT.logits_of(n, E, "bf16", 3)
    r = moc.moc_route(block, 1, renorm=False)
    dw, dl = torch.randn(n, 1, device="cuda"), torch.ones(1, device="cuda")
    want = moc.moc_route_bwd(block, r.ids, r.coef, dw, dl, renorm=False)
    logits = repeated(block, times)
    assert logits.shape[0] * 32 > 2 ** 32
    got = moc.moc_route_bwd(logits, repeated(r.ids, times), r.coef, repeated(dw, times), dl, renorm=False, out=logits)
    same(got, want, times)
