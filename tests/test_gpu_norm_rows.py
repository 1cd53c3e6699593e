"""Layer norm of a row does not depend on how many rows go with it: bit for bit."""
import pytest
import torch

import paper_2511_09323_amd as moc
from tests import test_gpu_norms as N

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [5, 128, 768, 1001, 1024, 1032, 2048, 2049, 4096, 8200, 16384])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_alone_and_among_others(d, dtype):
    a = N.make(1500, d, dtype, d)
    out = moc.moc_layernorm(a["h"], a["gain"], a["bias"], N.EPS)
    for rows in (slice(0, 1), slice(700, 703), slice(400, 1423), slice(476, 1500)):
        assert torch.equal(moc.moc_layernorm(a["h"][rows].clone(), a["gain"], a["bias"], N.EPS), out[rows]), rows
