"""The stored set in 8 bits: packed bytes and restored values exactly as the definition says, and the backward pass from it bit for bit that of
moc_ffn_bwd from the restored set (whose own parity with the oracle is tested elsewhere) as well as near the oracle's."""
import numpy as np
import pytest
import torch

import paper_2511_09323_amd as moc
from oracle import moc_oracle as O
from oracle import training_oracle as R
from paper_2511_09323_amd import inputs
from tests import parity as P

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def stored(T, d, F, K, dtype, seed):
    """x, idx, gvals, uvals as a forward call leaves them, values of very different sizes."""
    rng = np.random.default_rng(seed)
    idx = np.sort(np.argsort(rng.random((T, F)), axis=1)[:, :K], axis=1).astype(np.int32)
    val = lambda n: (rng.standard_normal((T, n)) * 10.0 ** rng.integers(-3, 3, (T, n))).astype(np.float32)
    dev = lambda v: torch.from_numpy(v).cuda().to(DT[dtype])
    return dev(val(d)), torch.from_numpy(idx).cuda(), dev(val(K)), dev(val(K))


def f32(t):
    return t.float().cpu().numpy()


def check_set(saved, x, idx, g, u, F):
    for q, e, v in ((saved.xq, saved.xe, x), (saved.gq, saved.ge, g), (saved.uq, saved.ue, u)):
        wq, we = R.pack8(f32(v))
        assert np.array_equal(e.cpu().numpy(), we) and np.array_equal(q.cpu().numpy(), wq)
    assert np.array_equal(saved.sel.cpu().numpy().view(np.uint32), R.pack_mask(idx.cpu().numpy(), F))


def check_load(saved, F, dtype, back):
    x, idx, g, u = back
    for q, e, v in ((saved.xq, saved.xe, x), (saved.gq, saved.ge, g), (saved.uq, saved.ue, u)):
        want = R.unpack8(q.cpu().numpy(), e.cpu().numpy())
        assert np.array_equal(f32(v).astype(np.float64), want, equal_nan=True)
    assert idx.cpu().numpy().tolist() == R.unpack_mask(saved.sel.cpu().numpy().view(np.uint32), F)


# T, d, F, K: one of everything, blocks that end inside, F inside a word, d aligned and not, K = F, rows of more than one pass
SHAPES = [(1, 8, 1, 1), (1, 8, 33, 33), (3, 32, 100, 31), (5, 40, 96, 32), (2, 72, 1376, 172), (7, 128, 171, 21), (4, 2056, 2048, 257), (2, 520, 9000, 5000),
          (2, 4104, 32768, 4100), (33, 64, 2736, 342)]


@pytest.mark.parametrize("T,d,F,K", SHAPES + [(3, 33, 50, 7), (2, 1, 5, 2), (2, 1028, 70, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_save_and_load(T, d, F, K, dtype):
    if dtype == "bf16" and d % 8:
        d += 8 - d % 8                                       # a rule of the library
    x, idx, g, u = stored(T, d, F, K, dtype, T + d + F)
    saved = moc.moc_act8_save(x, idx, g, u, F)
    check_set(saved, x, idx, g, u, F)
    back = moc.moc_act8_load(saved, F, DT[dtype])
    check_load(saved, F, dtype, back)
    assert torch.equal(back[1], idx)
    # again from what was restored, into arrays of the caller's: the same bytes
    out = moc.act8_empty(T, d, F, K)
    for t in out:
        t.fill_(77)
    again = moc.moc_act8_save(*back, F, out=out)
    assert all(torch.equal(a, b) for a, b in zip(saved, again))
    out = tuple(torch.full_like(t, 7) for t in back)
    assert all(torch.equal(a, b) for a, b in zip(back, moc.moc_act8_load(saved, F, DT[dtype], out=out)))


@pytest.mark.parametrize("T,d,F,K,dtype", [(5000, 136, 9000, 1100, "bf16"), (4097, 72, 171, 21, "f32"), (4099, 2056, 2048, 2048, "bf16")])
def test_many_tokens(T, d, F, K, dtype):
    """Tokens do not know of each other: all at once is a part after the other."""
    x, idx, g, u = stored(T, d, F, K, dtype, T)
    saved = moc.moc_act8_save(x, idx, g, u, F)
    back = moc.moc_act8_load(saved, F, DT[dtype])
    assert torch.equal(back[1], idx)
    for r in (slice(0, 8), slice(1000, 3500), slice(T - 3, T)):
        part = moc.moc_act8_save(*(t[r].clone() for t in (x, idx, g, u)), F)
        assert all(torch.equal(a[r], b) for a, b in zip(saved, part))
        assert all(torch.equal(a[r], b) for a, b in zip(back, moc.moc_act8_load(part, F, DT[dtype])))
    r = slice(T - 3, T)
    check_load(moc.Act8Set(*(t[r].clone() for t in saved)), F, dtype, [t[r] for t in back])


def test_values_at_the_edges():
    """Zeros of both signs, blocks of subnormals and just above 2^-119, the largest values, values that round to 128, ties, infinities and NaN."""
    v = np.zeros((11, 64), dtype=np.float32)
    v[1, ::2] = -0.0
    v[2, 5] = 1e-40
    v[3, 5] = 2.0 ** -119
    v[3, 6] = 2.0 ** -121
    v[4, :] = np.float32(3.4e38)
    v[5, :4] = (127.75, -127.75, 0.5, 1.5)
    v[6, :6] = (64, 0.5, 1.5, 2.5, -0.5, -2.5)
    v[7, 40] = np.inf
    v[8, 0] = -np.inf
    v[9, 63] = np.nan
    v[10, :3] = (np.float32(2.0 ** -120), 0, 1e-38)
    x = torch.from_numpy(v).cuda()
    idx = torch.arange(64, dtype=torch.int32, device="cuda").repeat(11, 1).contiguous()
    saved = moc.moc_act8_save(x, idx, x, x, 64)
    check_set(saved, x, idx, x, x, 64)
    check_load(saved, 64, "f32", moc.moc_act8_load(saved, 64, torch.float32))
    assert (saved.xe[7, 1], saved.xe[8, 0], saved.xe[9, 1], saved.xe[7, 0]) == (255, 255, 255, 0)
    h = x.bfloat16()
    saved = moc.moc_act8_save(h, idx, h, h, 64)
    check_set(saved, h, idx, h, h, 64)


def test_masks_that_were_not_saved():
    """Fewer or more bits than slots, bits behind the last channel: nothing out of bounds, the missing slots are -1."""
    T, d, F, K = 4, 32, 70, 10
    x, idx, g, u = stored(T, d, F, K, "f32", 1)
    saved = moc.moc_act8_save(x, idx, g, u, F)
    saved.sel[0] = 0
    saved.sel[1] = -1
    saved.sel[2, 2] |= -64                                    # channels 70 ..
    back = moc.moc_act8_load(saved, F, torch.float32)
    assert (back[1][0] == -1).all()
    assert back[1][1].tolist() == list(range(10))
    assert torch.equal(back[1][2:], idx[2:])
    w = torch.randn(F, d, device="cuda")
    dy = torch.randn(T, d, device="cuda")
    grads = moc.moc_ffn_bwd_act8(saved, w, w, w, dy)
    assert all(bool(torch.isfinite(t).all()) for t in grads)
    assert not grads[0][0].any()                             # no channel, no gradient


def layer(T, d, F, K, dtype, seed, E=0):
    rng = np.random.default_rng(seed)
    x, idx, g, u = stored(T, d, F, K, dtype, seed)
    dev = lambda s, std: torch.from_numpy((rng.standard_normal(s) * std).astype(np.float32)).cuda().to(DT[dtype])
    g, u = dev((T, K), 1.0), dev((T, K), 1.0)
    shape = (E, F, d) if E else (F, d)
    return (x / 100).to(DT[dtype]), idx, g, u, [dev(shape, 0.02) for _ in range(3)], dev((T, d), 1.0)


def oracle_grads(back, w, dy, F):
    x, idx, g, u = back
    Wg, Wu, Wd = (P.to_np(v) for v in w)
    M, GM, UM = O.expand_saved(idx.cpu().numpy(), P.to_np(g), P.to_np(u), F)
    dX, dWg, dWu, dWd = O.moc_backward(P.to_np(x), Wg.T, Wu.T, Wd, M, GM, UM, P.to_np(dy))
    return dX, dWg.T, dWu.T, dWd


# rows below and over a k-slice, F inside a padded slice, K = F, channels past one wavefront's span, more than 8192 of them
@pytest.mark.parametrize("T,d,F,K,dtype", [
    (1, 64, 96, 12, "bf16"), (31, 64, 171, 21, "bf16"), (33, 128, 515, 64, "bf16"), (200, 256, 1376, 172, "bf16"), (64, 64, 128, 128, "bf16"),
    (257, 128, 5461, 683, "bf16"), (40, 64, 11008, 1376, "bf16"), (1, 12, 20, 3, "f32"), (45, 96, 200, 25, "f32"), (70, 33, 1030, 129, "f32"),
    (32, 64, 2048, 2048, "f32"), (9, 64, 20000, 2500, "f32"), (50, 64, 30000, 600, "bf16")])
def test_backward(T, d, F, K, dtype):
    x, idx, g, u, w, dy = layer(T, d, F, K, dtype, T + F)
    saved = moc.moc_act8_save(x, idx, g, u, F)
    got = moc.moc_ffn_bwd_act8(saved, *w, dy)
    ws = torch.full((moc.workspace_bytes(T, d, F, K, DT[dtype], moc.OP_BWD_ACT8),), 255, dtype=torch.uint8, device="cuda")
    out = tuple(torch.empty_like(t) for t in got)
    again = moc.moc_ffn_bwd_act8(saved, *w, dy, ws=ws, out=out)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    back = moc.moc_act8_load(saved, F, DT[dtype])
    if 3 * 64 * -(-F // 64) * x.element_size() <= 160 * 1024 - 64:      # (beyond, moc_ffn_bwd takes the step in the product's epilogue)
        want = moc.moc_ffn_bwd(*(back[0], *w, back[1], back[2], back[3], dy))
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    for n, a, b in zip(("dx", "dwg", "dwu", "dwd"), got, oracle_grads(back, w, dy, F)):
        P.assert_close(n, P.to_np(a), b, P.TOL[dtype])


@pytest.mark.parametrize("counts,d,F,K,dtype", [((40, 0, 33, 200, 7, 64, 90, 50), 128, 520, 65, "bf16"), ((64, 96, 160), 96, 200, 25, "f32"), ((0, 1), 64, 96, 12, "bf16"),
                                                ((35,), 64, 2096, 262, "bf16")])
def test_experts_backward(counts, d, F, K, dtype):
    E, off = len(counts), [0] + np.cumsum(counts).tolist()
    x, idx, g, u, w, dy = layer(off[-1], d, F, K, dtype, 77, E)
    saved = moc.moc_act8_save(x, idx, g, u, F)
    got = moc.moc_ffn_bwd_experts_act8(saved, off, *w, dy)
    back = moc.moc_act8_load(saved, F, DT[dtype])
    want = moc.moc_ffn_bwd_experts(back[0], off, *w, back[1], back[2], back[3], dy)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ws = torch.full((moc.workspace_bytes(off[-1], d, F, K, DT[dtype], moc.OP_BWD_ACT8),), 255, dtype=torch.uint8, device="cuda")
    again = moc.moc_ffn_bwd_experts_act8(saved, tuple(off), *w, dy, ws=ws, out=tuple(torch.empty_like(t) for t in got))
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    for e in range(E):
        r = slice(off[e], off[e + 1])
        if counts[e]:
            for n, a, b in zip(("dx", "dwg", "dwu", "dwd"), (got[0][r], got[1][e], got[2][e], got[3][e]),
                               oracle_grads([t[r] for t in back], [v[e] for v in w], dy[r], F)):
                P.assert_close("%s[%d]" % (n, e), P.to_np(a), b, P.TOL[dtype])
        else:
            assert not any(bool(t[e].any()) for t in got[1:])


def test_every_forward_leaves_a_set_that_can_be_saved():
    T, d, F, K = 96, 128, 520, 130
    L = {k: P.to_dev(v, "bf16") for k, v in inputs.make_layer(31, T, d, F, "bf16", with_dy=True).items()}
    w = (L["wg"], L["wu"], L["wd"])
    for call in (lambda: moc.moc_ffn_fwd(L["x"], *w, K), lambda: moc.moc_ffn_fwd_grouped(L["x"], *w, 2, 8), lambda: moc.moc_ffn_fwd_keyed(L["x"], *w, K, "abs_silu")):
        _, idx, g, u = call()
        saved = moc.moc_act8_save(L["x"], idx, g, u, F)
        back = moc.moc_act8_load(saved, F, torch.bfloat16)
        assert torch.equal(back[1], idx)
        got = moc.moc_ffn_bwd_act8(saved, *w, L["dy"])
        assert all(torch.equal(a, b) for a, b in zip(got, moc.moc_ffn_bwd(back[0], *w, back[1], back[2], back[3], L["dy"])))
        # 8 bits against 16: a rounding to half a step, 2^-7 of a block's largest value, spread over the block: about 1 % of a value; gradients are
        # linear or nearly so in each of x, g and u: 2 % of their norm
        full = moc.moc_ffn_bwd(L["x"], *w, idx, g, u, L["dy"])
        for a, b in zip(got, full):
            assert float((a.double() - b.double()).norm() / b.double().norm()) <= 2e-2


def test_captured_and_replayed():
    T, d, F, K = 130, 128, 515, 64
    parts = layer(T, d, F, K, "bf16", 1)
    x, idx, g, u, w, dy = parts
    saved = moc.act8_empty(T, d, F, K)
    ws = torch.empty(moc.workspace_bytes(T, d, F, K, torch.bfloat16, moc.OP_BWD_ACT8), dtype=torch.uint8, device="cuda")
    out = (torch.empty_like(dy),) + tuple(torch.empty_like(v) for v in w)
    back = tuple(torch.empty_like(t) for t in (x, idx, g, u))

    def step():
        moc.moc_act8_save(x, idx, g, u, F, out=saved)
        moc.moc_act8_load(saved, F, torch.bfloat16, out=back)
        moc.moc_ffn_bwd_act8(saved, *w, dy, ws=ws, out=out)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        other = layer(T, d, F, K, "bf16", 50 + i)
        for a, b in zip((x, idx, g, u, dy), other[:4] + other[5:]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out + back + tuple(saved)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, out + back + tuple(saved))), i


def test_refusals_with_tensors():
    T, d, F, K = 6, 32, 70, 10
    x, idx, g, u, w, dy = layer(T, d, F, K, "f32", 1)
    saved = moc.moc_act8_save(x, idx, g, u, F)
    with pytest.raises(moc.MocError, match="sel has shape"):
        moc.moc_act8_load(saved, 200, torch.float32)
    with pytest.raises(moc.MocError, match="sel has shape"):
        moc.moc_act8_load(saved, 9, torch.float32)
    with pytest.raises(moc.MocError, match="idx has dtype"):
        moc.moc_act8_save(x, idx.long(), g, u, F)
    with pytest.raises(moc.MocError, match="gvals has dtype"):
        moc.moc_act8_save(x, idx, g.bfloat16(), u, F)
    with pytest.raises(moc.MocError, match="wu has shape"):
        moc.moc_ffn_bwd_act8(saved, w[0], w[1][:-1].contiguous(), w[2], dy)
    with pytest.raises(moc.MocError, match="MOC_ERR_WORKSPACE"):
        moc.moc_ffn_bwd_act8(saved, *w, dy, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(moc.MocError, match="n_experts"):
        moc.moc_ffn_bwd_experts_act8(saved, [0, 3, 6], *[v[None] for v in w], dy)
    with pytest.raises(moc.MocError, match="xe"):
        moc.moc_ffn_bwd_act8(saved._replace(xe=None), *w, dy)


def test_offsets_past_32_bits():
    """262149 rows of 8192: the last rows are what they are on their own."""
    T, d, F, K = (1 << 18) + 5, 8192, 64, 9
    x, idx, g, u = stored(32, d, F, K, "bf16", 5)
    alone = moc.moc_act8_save(x, idx, g, u, F)
    big = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    big[-32:] = x
    rest = [torch.cat([t[:1].expand(T - 32, -1), t]).contiguous() for t in (idx, g, u)]
    saved = moc.moc_act8_save(big, *rest, F)
    assert all(torch.equal(a[-32:], b) for a, b in zip(saved, alone))
    back = moc.moc_act8_load(saved, F, torch.bfloat16, out=(big, *rest))
    assert all(torch.equal(a[-32:], b) for a, b in zip(back, moc.moc_act8_load(alone, F, torch.bfloat16)))
    assert not back[0][:-32].any()


def test_one_workspace_for_call_after_call():
    """A workspace of a larger layer, used before, serves a smaller one on the same stream."""
    ws = torch.empty(moc.workspace_bytes(257, 128, 5461, 683, torch.bfloat16, moc.OP_BWD_ACT8), dtype=torch.uint8, device="cuda")
    for T, d, F, K in ((257, 128, 5461, 683), (40, 64, 171, 21), (257, 128, 5461, 683)):
        x, idx, g, u, w, dy = layer(T, d, F, K, "bf16", T)
        saved = moc.moc_act8_save(x, idx, g, u, F)
        want = moc.moc_ffn_bwd_act8(saved, *w, dy)
        got = moc.moc_ffn_bwd_act8(saved, *w, dy, ws=ws, out=tuple(torch.empty_like(t) for t in want))
        assert all(torch.equal(a, b) for a, b in zip(got, want))
