"""Layer norm and the gradients of layer norm and RMSNorm against float64.

Tolerances.  An output is rounded once: half a step, finfo.eps / 2 relative.  What fp32 adds before that is bounded by DEPTH * 2^-24 times the sum of
the magnitudes that went into the value: n is at most nb = r (|h| + mean |h|) in magnitude even where h and its mean cancel, a sum over a row
is a chain of at most 64 + 6 + 8 additions, a sum over T rows of at most T / 8 + 8 + 256 / 16 + 16 (one row's share of a workgroup, then of the
workgroups), and a handful of operations follow each; a squared error counts twice in r.  DEPTH = 256 covers rows, 256 + T / 8 the sums over rows."""
import numpy as np
import pytest
import torch

import paper_2511_09323_amd as moc
from oracle import training_oracle as R

pytestmark = pytest.mark.gpu

EPS = 1e-5
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
DEPTH = 256


def host(t):
    return t.detach().double().cpu().numpy()


def make(T, d, dtype, seed, offset=0.3):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)
    h = n(T, d) * (0.5 + n(d).abs()) + offset * n(d)
    t = dict(h=h, gain=1 + 0.1 * n(d), bias=0.1 * n(d), dy=n(T, d), dres=n(T, d))
    return {k: v.to(DT[dtype]).cuda() for k, v in t.items()}


def close(name, got, want, magnitude, dtype, depth):
    half = torch.finfo(DT[dtype]).eps / 2
    room = half * np.abs(want) + depth * 2.0 ** -24 * (1 + half) * magnitude + 1e-37
    worst = float(np.max(np.abs(host(got) - want) / room))
    print("[norm] %-6s uses %.3f of its tolerance" % (name, worst), flush=True)
    assert worst <= 1.0, "%s: %.3f times the tolerance" % (name, worst)


def check_forward(a, dtype, bias, got):
    h, gain, b = host(a["h"]), host(a["gain"]), host(a["bias"]) if bias else None
    want, _, r = R.norm_forward(h, gain, b, EPS, False)
    nb = r * (np.abs(h) + np.abs(h).mean(axis=1, keepdims=True))
    close("out", got, want, nb * np.abs(gain) + (0 if b is None else np.abs(b)), dtype, DEPTH)


def check_backward(a, dtype, rms, dres, got):
    h, gain, dy = host(a["h"]), host(a["gain"]), host(a["dy"])
    res = host(a["dres"]) if dres else None
    dh, dgain, dbias = R.norm_backward(h, gain, EPS, dy, res, rms)
    _, _, r = R.norm_forward(h, gain, None, EPS, rms)
    nb = r * (np.abs(h) + (0 if rms else np.abs(h).mean(axis=1, keepdims=True)))
    p = np.abs(dy * gain)
    size = r * (p + p.mean(axis=1, keepdims=True) + nb * (p * nb).mean(axis=1, keepdims=True)) + (0 if res is None else np.abs(res))
    T = h.shape[0]
    close("dh", got[0], dh, size, dtype, DEPTH)
    close("dgain", got[1], dgain, (np.abs(dy) * nb).sum(axis=0), dtype, DEPTH + T / 8)
    if not rms and got[2] is not None:
        close("dbias", got[2], dbias, np.abs(dy).sum(axis=0), dtype, DEPTH + T / 8)


# one row and few, rows past a workgroup's and a launch's, widths of every kernel: aligned and not, one element, just over each limit
SHAPES = [(1, 1), (1, 4096), (2, 8), (3, 7), (5, 1023), (7, 1024), (8, 1032), (9, 2047), (64, 2048), (33, 2056), (257, 4095), (65, 4096), (6, 4104), (3, 8191),
          (5, 8192), (2, 8200), (2, 16384), (2, 16383), (4099, 17), (2500, 520), (2311, 1001), (2049, 2048)]


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layernorm(T, d, dtype):
    a = make(T, d, dtype, T * 10007 + d)
    for bias in (True, False):
        check_forward(a, dtype, bias, moc.moc_layernorm(a["h"], a["gain"], a["bias"] if bias else None, EPS))
    check_backward(a, dtype, False, False, moc.moc_layernorm_bwd(a["h"], a["gain"], EPS, a["dy"]))
    ws = torch.full((moc.norm_bwd_workspace_bytes(T, d, DT[dtype]),), 255, dtype=torch.uint8, device="cuda")      # NaN
    out = (torch.empty_like(a["h"]), torch.empty_like(a["gain"]), None)
    check_backward(a, dtype, False, True, moc.moc_layernorm_bwd(a["h"], a["gain"], EPS, a["dy"], dres=a["dres"], ws=ws, out=out))


@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rmsnorm_bwd(T, d, dtype):
    a = make(T, d, dtype, T * 20011 + d)
    check_backward(a, dtype, True, False, moc.moc_rmsnorm_bwd(a["h"], a["gain"], EPS, a["dy"]))
    ws = torch.full((moc.norm_bwd_workspace_bytes(T, d, DT[dtype]),), 255, dtype=torch.uint8, device="cuda")
    out = (torch.empty_like(a["h"]), torch.empty_like(a["gain"]))
    check_backward(a, dtype, True, True, moc.moc_rmsnorm_bwd(a["h"], a["gain"], EPS, a["dy"], dres=a["dres"], ws=ws, out=out))


def test_a_mean_large_against_the_spread():
    """Offsets of 1000 and a spread of 1: the variance comes from differences, not from squares (2^-24 * 1000^2 is 6 %)."""
    a = make(37, 1536, "f32", 3, offset=0.0)
    a["h"] += 1000.0
    check_forward(a, "f32", True, moc.moc_layernorm(a["h"], a["gain"], a["bias"], EPS))
    check_backward(a, "f32", False, False, moc.moc_layernorm_bwd(a["h"], a["gain"], EPS, a["dy"]))


def test_constant_rows_and_rows_of_zeros():
    a = make(6, 256, "f32", 4)
    a["h"][1] = 0
    a["h"][4] = 2.5
    check_forward(a, "f32", True, moc.moc_layernorm(a["h"], a["gain"], a["bias"], EPS))
    check_backward(a, "f32", False, True, moc.moc_layernorm_bwd(a["h"], a["gain"], EPS, a["dy"], dres=a["dres"]))
    check_backward(a, "f32", True, True, moc.moc_rmsnorm_bwd(a["h"], a["gain"], EPS, a["dy"], dres=a["dres"]))


def test_nan_stays_in_its_row():
    a = make(9, 512, "bf16", 5)
    clean = moc.moc_layernorm(a["h"], a["gain"], a["bias"], EPS), moc.moc_layernorm_bwd(a["h"], a["gain"], EPS, a["dy"])[0]
    a["h"][3, 100] = float("nan")
    for was, now in zip(clean, (moc.moc_layernorm(a["h"], a["gain"], a["bias"], EPS), moc.moc_layernorm_bwd(a["h"], a["gain"], EPS, a["dy"])[0])):
        assert now[3].isnan().all()
        keep = torch.arange(9, device="cuda") != 3
        assert torch.equal(now[keep], was[keep])


@pytest.mark.parametrize("T,d", [(700, 768), (40, 8192), (3, 33)])
def test_in_place(T, d):
    a = make(T, d, "bf16", 6)
    out = moc.moc_layernorm(a["h"], a["gain"], a["bias"], EPS)
    h = a["h"].clone()
    assert moc.moc_layernorm(h, a["gain"], a["bias"], EPS, out=h) is h and torch.equal(h, out)
    for f, rest in ((moc.moc_layernorm_bwd, 2), (moc.moc_rmsnorm_bwd, 1)):
        want = f(a["h"], a["gain"], EPS, a["dy"], dres=a["dres"])
        for which in ("dy", "dres"):
            b = {k: v.clone() for k, v in a.items()}
            got = f(b["h"], b["gain"], EPS, b["dy"], dres=b["dres"], out=(b[which],) + tuple(torch.empty_like(a["gain"]) for _ in range(rest)))
            assert got[0] is b[which] and all(torch.equal(x, y) for x, y in zip(got, want)), which


def test_gradient_is_a_difference():
    """Along a random direction, fp32: (L(h + s v) - L(h - s v)) / 2 s, L summed in float64 from the fp32 output.  With s = 2^-6 the third-order term is
    about s^2 = 2e-4 of the slope's size and fp32's rounding 6e-8 * sqrt(T d) / s = 1e-3 of 1, against slopes of size sqrt(T d) = 160: 2e-3 of that."""
    a = make(50, 512, "f32", 7)
    dh, dgain, dbias = moc.moc_layernorm_bwd(a["h"], a["gain"], EPS, a["dy"])
    L = lambda h, gain, bias: float((moc.moc_layernorm(h, gain, bias, EPS).double() * a["dy"].double()).sum())
    s = 2.0 ** -6
    for grad, at in ((dh, 0), (dgain, 1), (dbias, 2)):
        args = [a["h"], a["gain"], a["bias"]]
        v = torch.randn_like(args[at])
        plus, minus = list(args), list(args)
        plus[at], minus[at] = args[at] + s * v, args[at] - s * v
        want = (L(*plus) - L(*minus)) / (2 * s)
        assert abs(float((grad.double() * v.double()).sum()) - want) <= 2e-3 * (50 * 512) ** 0.5 * 2


def test_same_bits_every_time_and_other_streams():
    a = make(3000, 1024, "bf16", 8)
    first = moc.moc_layernorm_bwd(a["h"], a["gain"], EPS, a["dy"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = moc.moc_layernorm_bwd(a["h"], a["gain"], EPS, a["dy"])
    torch.cuda.current_stream().wait_stream(side)
    again = moc.moc_layernorm_bwd(a["h"], a["gain"], EPS, a["dy"])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) and torch.equal(x, z) for x, y, z in zip(first, other, again))


def test_captured_and_replayed():
    a = make(300, 640, "bf16", 9)
    ws = torch.empty(moc.norm_bwd_workspace_bytes(300, 640, torch.bfloat16), dtype=torch.uint8, device="cuda")
    out, grads = torch.empty_like(a["h"]), (torch.empty_like(a["h"]), torch.empty_like(a["gain"]), torch.empty_like(a["gain"]))

    def step():
        moc.moc_layernorm(a["h"], a["gain"], a["bias"], EPS, out=out)
        moc.moc_layernorm_bwd(a["h"], a["gain"], EPS, a["dy"], dres=out, ws=ws, out=grads)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(3):
        b = make(300, 640, "bf16", 20 + i)
        for k in a:
            a[k].copy_(b[k])
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out,) + grads]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, (out,) + grads)), i


def test_refusals_with_tensors():
    a = make(4, 64, "bf16", 10)
    with pytest.raises(moc.MocError, match="gain has shape"):
        moc.moc_layernorm(a["h"], a["gain"][:-1].contiguous(), None, EPS)
    with pytest.raises(moc.MocError, match="contiguous"):
        moc.moc_layernorm(a["h"][:, ::2], a["gain"][:32], None, EPS)
    with pytest.raises(moc.MocError, match="dy has dtype"):
        moc.moc_rmsnorm_bwd(a["h"], a["gain"], EPS, a["dy"].float())
    with pytest.raises(moc.MocError, match="aligned"):
        moc.moc_layernorm(a["h"].view(-1)[4:4 + 64].view(1, 64), a["gain"], None, EPS)
    with pytest.raises(moc.MocError, match="MOC_ERR_WORKSPACE"):
        moc.moc_layernorm_bwd(a["h"], a["gain"], EPS, a["dy"], ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(moc.MocError, match="16384"):
        moc.moc_layernorm(torch.zeros(1, 16385, device="cuda"), torch.zeros(16385, device="cuda"), None, EPS)


def test_offsets_past_32_bits():
    """262149 rows of 8192: the last rows are what they are on their own."""
    T, d = (1 << 18) + 5, 8192
    block = make(64, d, "bf16", 11)
    tail = slice(T - 64, T)
    h, dy = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    h[tail], dy[tail] = block["h"], block["dy"]
    out = moc.moc_layernorm(h, block["gain"], block["bias"], EPS)
    assert torch.equal(out[tail], moc.moc_layernorm(block["h"], block["gain"], block["bias"], EPS))
    assert torch.equal(out[0], block["bias"])
    del out
    dh, dgain, dbias = moc.moc_layernorm_bwd(h, block["gain"], EPS, dy)
    for got in (dh, moc.moc_rmsnorm_bwd(h, block["gain"], EPS, dy)[0]):
        assert not got[:-64].any()
    # (rows of zeros add nothing to the sums; their number is not in the bound of the others' sum)
    check_backward(block, "bf16", False, False, (dh[tail], dgain, dbias))
