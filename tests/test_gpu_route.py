"""The router and its gradient against the token-by-token oracle.

Experts, counts and order are equal.  Tolerances of the rest, fp32: exp is good to 2 steps of 2^-23 and its argument (a difference of logits, at most 60
in magnitude here) to 60 * 2^-24 absolute, so an exponential is off by 64 * 2^-24 relative and sums of positive ones by as much and their own
roundings (8 + 5 additions in a row, T / 256 over tokens): 128 * 2^-24 for a weight or probability.  loss and coef: sums of positives, the
same.  dlogits: 4 products of such factors, relative to the magnitudes that are subtracted, and one rounding to the type."""
import numpy as np
import pytest
import torch

import paper_2511_09323_amd as moc
from oracle import training_oracle as R

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def check(logits, k, valid=None, renorm=True, seed=0, check_grad=True, outputs=True):
    T, E = logits.shape
    out = ws = None
    if outputs:          # outputs and workspace of the caller's, full of something else
        out = tuple(torch.full(s, 7, dtype=d, device="cuda") for d, s in ((torch.int32, (T, k)), (torch.float32, (T, k)), (torch.int32, (E,)), (torch.int32, (T * k,)),
                                                                        (torch.float32, (1,)), (torch.float32, (E,))))
        ws = torch.full((moc.route_workspace_bytes(T, E, k),), 255, dtype=torch.uint8, device="cuda")
    got = moc.moc_route(logits, k, valid=valid, renorm=renorm, ws=ws, out=out)
    want = R.route(logits.double().cpu().numpy(), k, None if valid is None else valid.cpu().numpy(), renorm)
    for n in ("ids", "counts", "order"):
        assert np.array_equal(getattr(got, n).cpu().numpy(), want[n]), n
    near = lambda a, b, tol: np.all(np.abs(a.double().cpu().numpy() - b) <= tol)
    depth = 128 + T / 256
    assert near(got.weights, want["weights"], depth * U * want["weights"] + 1e-38)
    assert near(got.coef, want["coef"], 4 * U * want["coef"])
    assert near(got.loss, want["loss"], depth * U * want["loss"])
    if not check_grad:
        return got
    g = torch.Generator().manual_seed(seed)
    dw, dl = torch.randn(T, k, generator=g).cuda(), torch.randn(1, generator=g).cuda() * T
    half = torch.finfo(logits.dtype).eps / 2
    for use_w, use_l in ((True, True), (True, False), (False, True)):
        d = moc.moc_route_bwd(logits, got.ids, got.coef, dw if use_w else None, dl if use_l else None, renorm=renorm)
        dwn = dw.double().cpu().numpy() if use_w else None
        scale = float(dl) if use_l else 0.0
        ref = R.route_backward(want, dwn, scale, renorm)
        # magnitudes: every difference's terms added instead
        size = abs(scale) * want["p"] * (want["coef"] + (want["p"] * want["coef"]).sum(axis=1, keepdims=True))
        if use_w:
            part = want["weights"] * np.abs(dwn)
            base = want["p"].copy()
            for t in range(T):
                live = want["ids"][t] >= 0
                if renorm:
                    base[t] = 0
                    base[t, want["ids"][t, live]] = want["weights"][t, live]
                size[t, want["ids"][t, live]] += part[t, live]
            size += base * part.sum(axis=1, keepdims=True)
        assert near(d, ref, half * np.abs(ref) + 4 * depth * U * size + 1e-37), (use_w, use_l)
    d = moc.moc_route_bwd(logits, got.ids, got.coef, renorm=renorm)
    assert not d.any()
    return got


def logits_of(T, E, dtype, seed, std=2.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, E, generator=g) * std).to(DT[dtype]).cuda()


# one token, one expert, widths of every kernel, aligned and not, every k, workgroups of one and many passes
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (3, 8, 8), (37, 8, 2), (256, 4, 1), (257, 8, 2), (300, 5, 5), (511, 12, 3), (700, 16, 16), (260, 60, 4), (130, 64, 6),
                                   (90, 100, 9), (70, 128, 16), (600, 130, 2), (40, 256, 16), (515, 255, 3), (70001, 4, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_router(T, E, k, dtype):
    check(logits_of(T, E, dtype, T + E), k, renorm=True, outputs=T != 37)
    if T < 1000:
        check(logits_of(T, E, dtype, T + E + 1), k, renorm=False)


@pytest.mark.parametrize("renorm", [False, True])
def test_padding(renorm):
    logits = logits_of(600, 8, "f32", 3)
    valid = (torch.rand(600, generator=torch.Generator().manual_seed(1)) < 0.7).to(torch.uint8).cuda()
    valid[256:512] = 0                                       # a whole workgroup without a token
    logits[valid == 0] = float("nan")                        # not looked at
    got = check(logits.nan_to_num(0.0), 2, valid, renorm)
    same = moc.moc_route(logits, 2, valid=valid, renorm=renorm)
    assert all(torch.equal(a, b) for a, b in zip(got, same))
    d = moc.moc_route_bwd(logits, same.ids, same.coef, torch.ones(600, 2, device="cuda"), torch.ones(1, device="cuda"), renorm=renorm)
    assert not d[valid == 0].any() and not d.isnan().any()


def test_no_token_at_all():
    for T in (5, 700):
        got = check(logits_of(T, 8, "f32", 4), 2, torch.zeros(T, dtype=torch.uint8, device="cuda"))
        assert float(got.loss) == 0.0 and not got.coef.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("renorm", [False, True])
def test_masked_experts(dtype, renorm):
    """Experts at -inf are never chosen, also where too few are left; the type's lowest value is a logit like others."""
    logits = logits_of(300, 8, dtype, 5)
    logits[:100, 2:] = -float("inf")
    logits[100:150, 1:] = -float("inf")
    logits[150:160] = -float("inf")
    logits[160:200, 4:] = torch.finfo(DT[dtype]).min
    logits[200:210] = torch.finfo(DT[dtype]).min
    check(logits, 3, renorm=renorm)


@pytest.mark.parametrize("E,k", [(8, 2), (64, 6), (100, 10)])
def test_ties_go_to_the_lower_expert(E, k):
    g = torch.Generator().manual_seed(E)
    logits = torch.randint(-2, 3, (400, E), generator=g).float()
    logits[::3] *= 0.0                                        # zeros of both signs
    check(logits.cuda(), k)
    check(torch.zeros(300, E, device="cuda"), k)


def test_far_logits():
    """Differences past the range of exp: weights of 0 and 1, no NaN."""
    logits = logits_of(64, 8, "f32", 6)
    logits[:, 3] += 50.0
    check(logits, 2, renorm=False)
    logits[:, 3] += 3e38
    got = moc.moc_route(logits, 2)
    assert (got.ids[:, 0] == 3).all() and torch.equal(got.weights, torch.tensor([[1.0, 0.0]], device="cuda").repeat(64, 1))


def test_nan_is_not_chosen_and_shows():
    logits = logits_of(300, 8, "f32", 7)
    logits[17, 3] = float("nan")
    logits[18] = float("nan")
    got = moc.moc_route(logits, 2)
    assert ((got.ids >= -1) & (got.ids < 8)).all() and 3 not in got.ids[17].tolist() and (got.ids[18] == -1).all()
    assert got.loss.isnan().all() and int(got.counts.sum()) == 2 * 299


def test_same_bits_in_place_and_on_another_stream():
    logits = logits_of(5000, 8, "bf16", 8)
    dw, dl = torch.randn(5000, 2, device="cuda"), torch.ones(1, device="cuda")
    a = moc.moc_route(logits, 2)
    da = moc.moc_route_bwd(logits, a.ids, a.coef, dw, dl)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = moc.moc_route(logits, 2)
        db = moc.moc_route_bwd(logits, b.ids, b.coef, dw, dl)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and torch.equal(da, db)
    own = logits.clone()
    assert moc.moc_route_bwd(own, a.ids, a.coef, dw, dl, out=own) is own and torch.equal(own, da)


def test_captured_and_replayed():
    logits, dw, dl = logits_of(3000, 8, "f32", 9), torch.randn(3000, 2, device="cuda"), torch.ones(1, device="cuda")
    r = moc.moc_route(logits, 2)
    ws = torch.empty(moc.route_workspace_bytes(3000, 8, 2), dtype=torch.uint8, device="cuda")
    d = torch.empty_like(logits)

    def step():
        moc.moc_route(logits, 2, ws=ws, out=r)
        moc.moc_route_bwd(logits, r.ids, r.coef, dw, dl, out=d)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        logits.copy_(logits_of(3000, 8, "f32", 40 + i))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in tuple(r) + (d,)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, tuple(r) + (d,))), i


def test_refusals_with_tensors():
    logits = logits_of(10, 8, "f32", 10)
    with pytest.raises(moc.MocError, match="k must"):
        moc.moc_route(logits, 9)
    with pytest.raises(moc.MocError, match="valid has dtype"):
        moc.moc_route(logits, 2, valid=torch.ones(10, dtype=torch.bool, device="cuda"))
    with pytest.raises(moc.MocError, match="contiguous"):
        moc.moc_route(logits.t().contiguous().t(), 2)
    with pytest.raises(moc.MocError, match="256"):
        moc.moc_route(torch.zeros(2, 300, device="cuda"), 2)
    r = moc.moc_route(logits, 2)
    with pytest.raises(moc.MocError, match="dweights has shape"):
        moc.moc_route_bwd(logits, r.ids, r.coef, torch.zeros(10, 3, device="cuda"))
    with pytest.raises(moc.MocError, match="MOC_ERR_WORKSPACE"):
        moc.moc_route(logits, 2, ws=torch.empty(16, dtype=torch.uint8, device="cuda"), out=r)


def test_offsets_past_32_bits():
    """36 million tokens of 64 logits, the same 8192 over and over: what they give on their own, over and over."""
    n, times, E, k = 8192, 4400, 64, 2
    block = logits_of(n, E, "bf16", 12)
    logits = block.repeat(times, 1)
    T = n * times
    assert T * E > 2 ** 31
    one, r = moc.moc_route(block, k), moc.moc_route(logits, np.int64(k))
    assert torch.equal(r.counts, one.counts * times)
    for name in ("ids", "weights"):
        a, b = getattr(r, name).view(times, n, k), getattr(one, name)
        assert all(torch.equal(a[i], b) for i in (0, 1, times // 2, times - 1)), name
    assert torch.equal(r.ids.view(times, n, k).sum(0), one.ids * times)
    # the mean over tokens is the block's; sums of 2200 numbers of one size in a row: 2200 * 2^-24, twice
    assert abs(float(r.loss) - float(one.loss)) <= 2.0 ** -11 * float(one.loss)
    # order: slots ascend within an expert, and a slot's expert is the one its place says
    at = torch.repeat_interleave(torch.arange(E, device="cuda"), r.counts.long())
    assert torch.equal(r.ids.view(-1)[r.order.long()].long(), at)
    assert bool(((r.order[1:] > r.order[:-1]) | (at[1:] != at[:-1])).all())
    dw = torch.randn(n, k, device="cuda")
    d = moc.moc_route_bwd(logits, r.ids, r.coef, dw.repeat(times, 1), None)
    d1 = moc.moc_route_bwd(block, one.ids, one.coef, dw, None)
    assert torch.equal(d[-n:], d1) and torch.equal(d[:n], d1)
