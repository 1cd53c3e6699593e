"""The operators together, as a training step of one pre-norm block of MoC experts uses them: layer norm, router, rows by expert, the experts'
forward, the stored set in 8 bits, and the way back -- against the same block in float64 from the library's own choices (experts, channels) and
8-bit values.  bf16 roundings between the steps: P.TOL, as for the layer alone."""
import numpy as np
import pytest
import torch

import paper_2511_09323_amd as moc
from oracle import moc_oracle as O
from oracle import training_oracle as R
from tests import parity as P

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.mark.parametrize("dtype,padded", [("bf16", True), ("f32", False)])
def test_training_step_of_a_block(dtype, padded):
    T, d, F, K, E, k = 300, 128, 344, 43, 8, 2
    rng = np.random.default_rng(12)
    dt = P.TORCH_DTYPE[dtype]
    dev = lambda s, std: torch.from_numpy((rng.standard_normal(s) * std).astype(np.float32)).cuda().to(dt)
    h, gain, bias = dev((T, d), 1.0), 1 + dev((d,), 0.1), dev((d,), 0.1)
    wr = dev((d, E), 0.1)
    w = [dev((E, F, d), 0.05) for _ in range(3)]
    dnext = dev((T, d), 1.0)
    alpha = torch.full((1,), 0.5, device="cuda")
    valid = None
    if padded:
        valid = torch.ones(T, dtype=torch.uint8, device="cuda")
        valid[-40:] = 0
    # forward
    x = moc.moc_layernorm(h, gain, bias, EPS)
    logits = x @ wr
    r = moc.moc_route(logits, k, valid=valid)
    counts = r.counts.tolist()
    A = sum(counts)
    off = [0] + np.cumsum(counts).tolist()
    order = r.order[:A].long()
    token = order // k
    rows = x[token].contiguous()
    y, idx, g, u = moc.moc_ffn_fwd_experts(rows, off, *w, K)
    saved = moc.moc_act8_save(rows, idx, g, u, F)
    back = moc.moc_act8_load(saved, F, dt)
    wt = r.weights.view(-1)[order]
    out = h.float().index_add(0, token, y.float() * wt[:, None]).to(dt)
    # backward of sum(out * dnext) + alpha * loss
    drow = dnext.float()[token]
    dweights = torch.zeros(T * k, device="cuda").index_put_((order,), (drow * y.float()).sum(1)).view(T, k)
    drows, *dw = moc.moc_ffn_bwd_experts_act8(saved, off, *w, (drow * wt[:, None]).to(dt))
    dlogits = moc.moc_route_bwd(logits, r.ids, r.coef, dweights, alpha)
    dx = torch.zeros(T, d, device="cuda").index_add(0, token, drows.float()) + dlogits.float() @ wr.float().t()
    dwr = x.float().t() @ dlogits.float()
    dh, dgain, dbias = moc.moc_layernorm_bwd(h, gain, EPS, dx.to(dt), dres=dnext)
    torch.cuda.synchronize()

    # the same in float64
    n64 = lambda t: t.detach().double().cpu().numpy()
    H, GN, BI, WR, DN = n64(h), n64(gain), n64(bias), n64(wr), n64(dnext)
    X = R.norm_forward(H, GN, BI, EPS, False)[0]
    tol = P.TOL[dtype]
    P.assert_close("x", n64(x), X, tol)
    route = R.route(n64(logits), k, None if valid is None else valid.cpu().numpy())
    assert np.array_equal(route["ids"], r.ids.cpu().numpy()) and np.array_equal(route["order"], r.order.cpu().numpy())
    P.assert_close("logits", n64(logits), X @ WR, tol)
    tok, om = token.cpu().numpy(), order.cpu().numpy()
    WT = route["weights"].reshape(-1)[om]
    Y, DR, DW = np.zeros((A, d)), np.zeros((A, d)), [np.zeros((E, F, d)) for _ in range(3)]
    BX, BG, BU = n64(back[0]), n64(back[2]), n64(back[3])
    idx_np = idx.cpu().numpy()
    dyr = DN[tok] * WT[:, None]
    M = O.mask_from_idx(idx_np, F)
    for e in range(E):
        s = slice(off[e], off[e + 1])
        if counts[e] == 0:
            continue
        We = [n64(v[e]) for v in w]
        Y[s] = O.moc_forward_given_mask(X[tok[s]], We[0].T, We[1].T, We[2], M[s])[0]
        Ms, GM, UM = O.expand_saved(idx_np[s], BG[s], BU[s], F)
        DR[s], a, b, c = O.moc_backward(BX[s], We[0].T, We[1].T, We[2], Ms, GM, UM, dyr[s])
        DW[0][e], DW[1][e], DW[2][e] = a.T, b.T, c
    P.assert_close("y", n64(y), Y, tol)
    OUT = H.copy()
    np.add.at(OUT, tok, Y * WT[:, None])
    P.assert_close("out", n64(out), OUT, tol)
    DWT = np.zeros(T * k)
    DWT[om] = (DN[tok] * Y).sum(axis=1)
    DL = R.route_backward(route, DWT.reshape(T, k), 0.5, True)
    P.assert_close("dlogits", n64(dlogits), DL, tol)
    DX = DL @ WR.T
    np.add.at(DX, tok, DR)
    P.assert_close("dwr", n64(dwr), X.T @ DL, tol)
    for n, a, b in zip(("dwg", "dwu", "dwd"), dw, DW):
        P.assert_close(n, n64(a), b, tol)
    for n, a, b in zip(("dh", "dgain", "dbias"), (dh, dgain, dbias), R.norm_backward(H, GN, EPS, DX, DN, False)):
        P.assert_close(n, n64(a), b, tol)
    if padded:
        assert not dlogits[-40:].any() and torch.equal(out[-40:], h[-40:])


def test_two_graphs_share_a_workspace():
    """Nothing in a workspace lasts from one call to the next: two captured steps of other sizes over one workspace, replayed in turn, are the eager ones."""
    sizes = ((700, 640, 8, 2), (3000, 200, 64, 3))
    need = max(max(moc.norm_bwd_workspace_bytes(T, d, torch.bfloat16), moc.route_workspace_bytes(T, E, k)) for T, d, E, k in sizes)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    parts = []
    for T, d, E, k in sizes:
        h, dy, gain = (torch.randn(*s, device="cuda").bfloat16() for s in ((T, d), (T, d), (d,)))
        logits = torch.randn(T, E, device="cuda")
        grads = (torch.empty_like(h), torch.empty_like(gain), torch.empty_like(gain))
        out = tuple(torch.empty_like(t) for t in moc.moc_route(logits, k))

        def step(h=h, dy=dy, gain=gain, logits=logits, grads=grads, out=out, k=k):
            moc.moc_layernorm_bwd(h, gain, EPS, dy, ws=ws, out=grads)
            moc.moc_route(logits, k, ws=ws, out=out)
        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        parts.append((g, step, grads + out, (h, dy, logits)))
    for i in range(3):
        for g, step, results, inputs in parts:
            for t in inputs:
                t.normal_()
            g.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in results]
            step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, results)), i
