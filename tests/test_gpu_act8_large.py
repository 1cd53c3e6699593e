"""The backward from 8 bits on layers whose dense rows are too long for the expansion kernel of moc_ffn_bwd (three of them in 160 KB of LDS: up to 27264 channels in
bf16, 13632 in fp32): bit for bit moc_ffn_bwd from the restored set, as below that."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2511_09323_amd as moc
from tests import parity as P
from tests import test_gpu_act8 as A8

pytestmark = pytest.mark.gpu


def same(saved, w, dy, F, dtype):
    T, d = saved.xq.shape
    need = moc.workspace_bytes(T, d, F, saved.gq.shape[1], A8.DT[dtype], moc.OP_BWD_ACT8)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    got = moc.moc_ffn_bwd_act8(saved, *w, dy, ws=ws, out=(torch.empty_like(dy),) + tuple(torch.empty_like(v) for v in w))
    x, idx, g, u = moc.moc_act8_load(saved, F, A8.DT[dtype])
    want = moc.moc_ffn_bwd(x, *w, idx, g, u, dy)
    for n, a, b in zip(("dx", "dwg", "dwu", "dwd"), got, want):
        assert torch.equal(a, b), n
    return got, (x, idx, g, u)


# the last F of the expansion kernel and the first past it, rows below and over a k-slice, F inside a padded slice, few and all channels
@pytest.mark.parametrize("T,d,F,K,dtype", [(33, 64, 27264, 3408, "bf16"), (33, 64, 27265, 3408, "bf16"), (50, 64, 30000, 600, "bf16"), (5, 72, 28672, 28672, "bf16"),
                                           (129, 64, 32768, 1, "bf16"), (9, 64, 13632, 1704, "f32"), (9, 64, 13633, 1704, "f32"), (40, 33, 20000, 2500, "f32")])
def test_wide_layers(T, d, F, K, dtype):
    x, idx, g, u, w, dy = A8.layer(T, d, F, K, dtype, T + F)
    got, back = same(moc.moc_act8_save(x, idx, g, u, F), w, dy, F, dtype)
    for n, a, b in zip(("dx", "dwg", "dwu", "dwd"), got, A8.oracle_grads(back, w, dy, F)):
        P.assert_close(n, P.to_np(a), b, P.TOL[dtype])


def test_wide_layers_with_masks_that_were_not_saved():
    """Fewer or more bits than slots: what moc_act8_load makes of them."""
    T, d, F, K = 4, 64, 28000, 300
    x, idx, g, u, w, dy = A8.layer(T, d, F, K, "bf16", 3)
    saved = moc.moc_act8_save(x, idx, g, u, F)
    saved.sel[0] = 0
    saved.sel[1] = -1
    got, _ = same(saved, w, dy, F, "bf16")
    assert not got[0][0].any() and all(bool(torch.isfinite(t).all()) for t in got)


def test_wide_layers_captured_and_replayed():
    T, d, F, K = 40, 64, 28000, 300
    parts = A8.layer(T, d, F, K, "bf16", 1)
    x, idx, g, u, w, dy = parts
    saved = moc.act8_empty(T, d, F, K)
    ws = torch.empty(moc.workspace_bytes(T, d, F, K, torch.bfloat16, moc.OP_BWD_ACT8), dtype=torch.uint8, device="cuda")
    out = (torch.empty_like(dy),) + tuple(torch.empty_like(v) for v in w)

    def step():
        moc.moc_act8_save(x, idx, g, u, F, out=saved)
        moc.moc_ffn_bwd_act8(saved, *w, dy, ws=ws, out=out)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        other = A8.layer(T, d, F, K, "bf16", 60 + i)
        for a, b in zip((x, idx, g, u, dy), other[:4] + other[5:]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, out)), i


def test_with_the_step_in_the_epilogue_everywhere():
    """MOC_BWD_EPILOGUE=1 puts moc_ffn_bwd's pointwise step into the product at every F; the library reads it when it is loaded."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = ("import paper_2511_09323_amd as moc\nfrom tests import test_gpu_act8 as A8, test_gpu_act8_large as L\n"
            "for T, d, F, K, dtype in ((130, 128, 515, 64, 'bf16'), (45, 96, 200, 25, 'f32')):\n"
            "    x, idx, g, u, w, dy = A8.layer(T, d, F, K, dtype, T)\n"
            "    L.same(moc.moc_act8_save(x, idx, g, u, F), w, dy, F, dtype)\nprint('same')\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=root, env=dict(os.environ, MOC_BWD_EPILOGUE="1"), capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and r.stdout.strip().endswith("same"), r.stdout[-1000:] + r.stderr[-2000:]
