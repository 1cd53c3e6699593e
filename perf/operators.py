"""Cases for the operators around the MoC layer in training: the norms and their gradients, the layer's stored set in
8 bits, and the router before the experts.

  norm    layer norm (or RMSNorm's gradient) of T rows of d: forward, or forward and backward, in one pass;
  saved   a layer's stored set (x, the Top-K mask, the gate and up values there) packed to 8 bits and restored;
  bwd     the layer's backward pass from such a set, plain or with the tokens sorted by expert;
  route   softmax router: chosen experts, weights, counts, the copies in expert order, balance loss, and its gradient.

`own` false: the operators in elementary torch operations, 32 bits, rounded once at the end.  `own` true: the library's calls.
The (d, F) pairs are those of paper_2511_09323_amd/configs.py and its neighbours (F = 8/3 d, K about F/8); experts and their
shares are those of perf/cases.py.

The 8-bit form: 32 consecutive values of a row share one byte e, the fp32 exponent field of the largest magnitude among them;
a value is q * 2^(e - 133) with q = round(v * 2^(133 - e)), halves to even, at most 127 in magnitude.  e below 8 is stored as 0
and means zeros, 255 means NaN (a block with an infinity or a NaN).  The Top-K mask is one bit per channel.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
WEIGHT_STD = 0.02
EXPERTS = 8
LARGEST = {"norm": 8192 * 4096, "saved": 8192 * 2048, "bwd": 8192 * 2048 * 5461, "bwd_f32": 512 * 768 * 2048, "route": 32768 * 64}


def _norm(T, d, dtype="bf16", rms=False, bias=True, dres=False, bwd=True, **name):
    return dict(kind="norm", T=T, d=d, dtype=dtype, rms=rms, bias=bias and not rms, dres=dres, bwd=bwd, **name)


def _set(kind, T, d, F, K, dtype="bf16", experts=0, **name):
    return dict(kind=kind, T=T, d=d, F=F, K=K, dtype=dtype, experts=experts, **name)


def _route(T, E, k, dtype="bf16", renorm=True, padded=False, **name):
    return dict(kind="route", T=T, E=E, k=k, dtype=dtype, renorm=renorm, padded=padded, **name)


def listed():
    return [
        # the norm of one token in a decode step: latency
        _norm(1, 4096, bwd=False, name="layernorm_token"),
        # gradient check of a small model in fp32: odd rows, odd width, no 16-byte alignment
        _norm(2047, 1001, "f32", name="layernorm_odd_f32"),
        # the largest: a block's norm on the 7B width, 4 x 2048 tokens
        _norm(8192, 4096, name="layernorm_7b"),
        # the norm that the prefill stack uses, with the residual's gradient added
        _norm(8192, 2048, rms=True, dres=True, name="rmsnorm_1b"),
        # the fp32 layer of the smallest shape
        _set("saved", 256, 512, 1376, 172, "f32", name="saved_60m_f32"),
        # the headline training shape
        _set("saved", 8192, 2048, 5461, 683, name="saved_1b"),
        # a short ragged batch of a small model: launches count
        _set("bwd", 333, 768, 2048, 256, name="bwd_130m_t333"),
        # the headline training shape: large products
        _set("bwd", 8192, 2048, 5461, 683, name="bwd_1b"),
        # the experts of an MoE layer: 8192 tokens, two of eight experts each, uneven
        _set("bwd", 16384, 768, 2048, 384, experts=EXPERTS, name="bwd_moe"),
        # a handful of tokens: latency
        _route(37, 8, 2, name="route_t37"),
        # the router of that MoE layer, fp32 logits
        _route(16384, 8, 2, "f32", name="route_moe"),
        # many small experts, padded sequences, weights as the softmax gives them
        _route(32768, 64, 6, renorm=False, padded=True, name="route_64_padded"),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(("norm", "norm", "saved", "bwd", "bwd_f32", "route", "route"))
    if kind == "norm":
        d = rng.choice((512, 768, 1024, 1536, 2048, 4096)) if rng.random() < 0.5 else _log_int(rng, 17, 6000)
        rms = rng.random() < 0.4
        bwd = rms or rng.random() < 0.8
        return _norm(_log_int(rng, 1, min(16384, LARGEST[kind] // d)), d, rng.choice(("bf16", "bf16", "f32")), rms=rms, bias=rng.random() < 0.7,
                     dres=bwd and rng.random() < 0.5, bwd=bwd)
    if kind == "route":
        E = rng.choice((4, 8, 8, 16, 60, 64))
        return _route(_log_int(rng, 1, LARGEST[kind] // E if E >= 16 else 65536), E, rng.randint(1, min(E, 6)), rng.choice(("bf16", "f32")),
                      rng.random() < 0.5, rng.random() < 0.5)
    f32 = kind == "bwd_f32"
    d = rng.choice((512, 768) if f32 else (512, 768, 1024, 1536, 2048))
    step = rng.choice((1, 8, 32))
    F = -(-(8 * d // 3) // step) * step
    K = int(F * rng.choice((0.125, 0.1875, 0.2)))
    if kind == "saved":
        return _set(kind, _log_int(rng, 1, LARGEST[kind] // d), d, F, K, rng.choice(("bf16", "bf16", "f32")))
    experts = EXPERTS if not f32 and d < 1024 and rng.random() < 0.4 else 0
    top = min(512 if f32 else 16384 if experts else 8192, LARGEST[kind] // (d * F))
    return _set("bwd", _log_int(rng, 64, top), d, F, K, "f32" if f32 else "bf16", experts)


# ---------------------------------------------------------------------------------------------------------- inputs
def _power(n):
    """2^n of whole numbers n, exactly (float32; n from -126 to 127)."""
    return ((n + 127) << 23).to(torch.int32).view(torch.float32)


def _blocks(v):
    n = v.shape[1]
    return torch.nn.functional.pad(v, (0, -n % 32)).view(v.shape[0], -1, 32)


def _pack(v):
    """(q int8 [T, n], e uint8 [T, ceil(n / 32)]) of v [T, n]."""
    b = _blocks(v.float())
    amax = b.abs().amax(2)
    e = (amax.view(torch.int32) >> 23).to(torch.int32)      # NaN and infinity: 255
    e = torch.where(e < 8, 0, e)
    live = ((e > 0) & (e < 255)).unsqueeze(2)
    q = torch.where(live, torch.round(b * _power(torch.where(live, 133 - e.unsqueeze(2), 0))).clamp(-127, 127), 0.0)
    return q.to(torch.int8).view(v.shape[0], -1)[:, :v.shape[1]].contiguous(), e.to(torch.uint8)


def _unpack(q, e):
    """float32 values of an 8-bit array."""
    e = e.int()
    step = torch.where(e == 255, math.nan, torch.where(e == 0, 0.0, _power((e - 133).clamp(min=-126))))
    return (_blocks(q.float()) * step.unsqueeze(2)).view(q.shape[0], -1)[:, :q.shape[1]]


def _mask_words(idx, F):
    """One bit per channel: int32 [T, ceil(F / 32)]."""
    bits = torch.zeros((idx.shape[0], -(-F // 32) * 32), dtype=torch.int64, device=idx.device).scatter_(1, idx.long(), 1)
    w = (bits.view(idx.shape[0], -1, 32) << torch.arange(32, device=idx.device)).sum(2)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)


def _mask_idx(sel, K):
    """The channels of the set bits, ascending: int32 [T, K]."""
    bits = ((sel.unsqueeze(2) >> torch.arange(32, dtype=torch.int32, device=sel.device)) & 1).view(sel.shape[0], -1)
    slot = torch.where(bits > 0, bits.cumsum(1) - 1, K)
    idx = torch.empty((sel.shape[0], K + 1), dtype=torch.int32, device=sel.device)
    idx.scatter_(1, slot, torch.arange(bits.shape[1], dtype=torch.int32, device=sel.device).expand(sel.shape[0], -1))
    return idx[:, :K]


def _stored(case, normal):
    """x and the stored set of a layer as its forward pass leaves them: idx ascending, gate values above the row's threshold."""
    T, d, F, K = case["T"], case["d"], case["F"], case["K"]
    g = normal((T, F), WEIGHT_STD * math.sqrt(d), torch.float32)
    idx = torch.topk(g, K, dim=1, sorted=False)[1].sort(dim=1)[0]
    dt = DTYPES[case["dtype"]]
    return normal((T, d)), idx.to(torch.int32), g.gather(1, idx).to(dt), normal((T, K), WEIGHT_STD * math.sqrt(d))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]

    def normal(shape, std=1.0, dtype=dt):
        return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * std).to(dtype)

    s = dict(case, kept={})
    T = case["T"]
    if case["kind"] == "norm":
        d = case["d"]
        # a residual stream: channels of different sizes and offsets
        s["h"] = (normal((T, d), 1.0, torch.float32) * (0.5 + normal((d,), 1.0, torch.float32).abs()) + normal((d,), 0.3, torch.float32)).to(dt)
        s["gain"] = 1 + normal((d,), 0.1)
        s["shift"] = normal((d,), 0.1) if case["bias"] else None
        s["dy"] = normal((T, d)) if case["bwd"] else None
        s["res"] = normal((T, d)) if case["dres"] else None
    elif case["kind"] == "saved":
        s["x"], s["idx"], s["g"], s["u"] = _stored(case, normal)
    elif case["kind"] == "bwd":
        x, idx, g, u = _stored(case, normal)
        (s["xq"], s["xe"]), (s["gq"], s["ge"]), (s["uq"], s["ue"]) = _pack(x), _pack(g), _pack(u)
        s["sel"] = _mask_words(idx, case["F"])
        E = case["experts"]
        s["w"] = [normal(((E,) if E else ()) + (case["F"], case["d"]), WEIGHT_STD) for _ in range(3)]      # W_gate, W_up, W_down
        s["dy"] = normal((T, case["d"]))
        # host row offsets of uneven experts, as the caller of the expert entry points has them
        share = (torch.rand(max(1, E), generator=gen, device="cuda") + 0.5).double()
        s["offsets"] = [0] + (share.cumsum(0) / share.sum() * T).round().long().tolist()
        s["offsets"][-1] = T
    else:
        E = case["E"]
        s["logits"] = normal((T, E), 1.5) + normal((E,), 0.5)
        s["valid"] = None
        if case["padded"]:                                     # sequences of up to 512 tokens, padded to 512
            length = torch.randint(1, 513, (-(-T // 512), 1), generator=gen, device="cuda")
            s["valid"] = (torch.arange(512, device="cuda") < length).view(-1)[:T].to(torch.uint8)
        s["dweights"] = normal((T, case["k"]), 1.0, torch.float32)
        s["dloss"] = torch.full((1,), 0.01 * T, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------------ plain forms
def _plain_norm(s):
    dt, h, gain = s["h"].dtype, s["h"].float(), s["gain"].float()
    c = h if s["rms"] else h - h.mean(1, keepdim=True)
    r = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
    n = c * r
    out = {}
    if not s["rms"]:
        out["out"] = (n * gain + s["shift"].float() if s["bias"] else n * gain).to(dt)
    if s["bwd"]:
        dy = s["dy"].float()
        p = dy * gain
        dh = p - n * (p * n).mean(1, keepdim=True)
        dh = r * (dh if s["rms"] else dh - p.mean(1, keepdim=True))
        out["dh"] = (dh + s["res"].float() if s["dres"] else dh).to(dt)
        out["dgain"] = (dy * n).sum(0).to(dt)
        if s["bias"]:
            out["dbias"] = dy.sum(0).to(dt)
    return out


def _plain_saved(s):
    dt, K = s["x"].dtype, s["K"]
    sel = _mask_words(s["idx"], s["F"])
    x, g, u = (_unpack(*_pack(v)).to(dt) for v in (s["x"], s["g"], s["u"]))
    return {"sel": sel, "x": x, "idx": _mask_idx(sel, K), "g": g, "u": u}


def _plain_bwd(s):
    dt, F = s["dy"].dtype, s["F"]
    idx = _mask_idx(s["sel"], s["K"]).long()
    x, g, u, dy = _unpack(s["xq"], s["xe"]), _unpack(s["gq"], s["ge"]), _unpack(s["uq"], s["ue"]), s["dy"].float()
    wg, wu, wd = (w.float().view(-1, F, s["d"]) for w in s["w"])
    E, at = wg.shape[0], s["offsets"]
    rows = [slice(at[e], at[e + 1]) for e in range(E)]
    dz = torch.cat([dy[r] @ wd[e].t() for e, r in enumerate(rows)]).gather(1, idx)
    sig = 1 / (1 + torch.exp(-g))

    def dense(v):
        return torch.zeros((v.shape[0], F), device=v.device).scatter_(1, idx, v)

    z, dg, du = dense(g * sig * u), dense(u * dz * (sig * (1 + g * (1 - sig)))), dense(g * sig * dz)
    dx = torch.cat([dg[r] @ wg[e] + du[r] @ wu[e] for e, r in enumerate(rows)])
    grads = [torch.stack([a[r].t() @ b[r] for r in rows]).view(s["w"][0].shape) for a, b in ((dg, x), (du, x), (z, dy))]
    return {n: v.to(dt) for n, v in zip(("dx", "dwg", "dwu", "dwd"), [dx] + grads)}


def _plain_route(s):
    E, k = s["E"], s["k"]
    lo = s["logits"].float()
    top, ids = lo.sort(dim=1, descending=True, stable=True)           # equal values: the lower expert first
    top, ids = top[:, :k], ids[:, :k]
    live = top > -math.inf
    if s["padded"]:
        live = live & (s["valid"] > 0).unsqueeze(1)
    used = live[:, :1].float()
    p = torch.exp(lo - lo.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True) * used
    w = p.gather(1, ids) * live
    if s["renorm"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-30)
    here = (ids.unsqueeze(2) == torch.arange(E, device=ids.device)) & live.unsqueeze(2)          # [T, k, E]
    counts = here.sum((0, 1))
    A, N = counts.sum(), used.double().sum()
    coef = (E * counts.double() / (A * N).clamp(min=1)).float()
    loss = (coef.double() * p.double().sum(0)).sum().float().view(1)
    ids = torch.where(live, ids, -1).to(torch.int32)
    key, order = torch.where(live, ids, E).view(-1).sort(stable=True)
    order = torch.where(key < E, order, -1).to(torch.int32)
    # gradient: of the weights through the softmax (over the chosen experts alone where they are renormalised), of the loss through p
    dw = s["dweights"] * live
    own_part = (here * (w * dw).unsqueeze(2)).sum(1)                                             # w_j dw_j at the chosen expert
    base = (here * w.unsqueeze(2)).sum(1) if s["renorm"] else p
    dl = own_part - base * (w * dw).sum(1, keepdim=True)
    dl = dl + s["dloss"] * p * (coef - (p * coef).sum(1, keepdim=True))
    return {"ids": ids, "weights": w, "counts": counts.to(torch.int32), "order": order, "loss": loss, "coef": coef, "dlogits": dl.to(s["logits"].dtype)}


# ------------------------------------------------------------------------------------------------- the library's calls
def _own(s):
    import paper_2511_09323_amd as moc
    kept = s["kept"]                     # outputs and workspaces, made once, as a training program keeps them

    def empty(*shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def scratch(n):
        return empty(max(256, n), dtype=torch.uint8)

    if s["kind"] == "norm":
        T, d, dt = s["T"], s["d"], s["h"].dtype
        if not kept:
            kept["out"] = empty(T, d, dtype=dt)
            if s["bwd"]:
                kept["ws"] = scratch(moc.norm_bwd_workspace_bytes(T, d, dt))
                kept["grads"] = (empty(T, d, dtype=dt), empty(d, dtype=dt)) + (() if s["rms"] else (empty(d, dtype=dt) if s["bias"] else None,))
        out = {}
        if not s["rms"]:
            out["out"] = moc.moc_layernorm(s["h"], s["gain"], s["shift"], EPS, out=kept["out"])
        if s["bwd"]:
            f = moc.moc_rmsnorm_bwd if s["rms"] else moc.moc_layernorm_bwd
            grads = f(s["h"], s["gain"], EPS, s["dy"], dres=s["res"], ws=kept["ws"], out=kept["grads"])
            out.update((n, v) for n, v in zip(("dh", "dgain", "dbias"), grads) if v is not None)
        return out
    if s["kind"] == "saved":
        T, K, dt = s["T"], s["K"], s["x"].dtype
        if not kept:
            kept["set"] = moc.act8_empty(T, s["d"], s["F"], K)
            kept["out"] = (empty(T, s["d"], dtype=dt), empty(T, K, dtype=torch.int32), empty(T, K, dtype=dt), empty(T, K, dtype=dt))
        saved = moc.moc_act8_save(s["x"], s["idx"], s["g"], s["u"], s["F"], out=kept["set"])
        x, idx, g, u = moc.moc_act8_load(saved, s["F"], dt, out=kept["out"])
        return {"sel": saved.sel, "x": x, "idx": idx, "g": g, "u": u}
    if s["kind"] == "bwd":
        saved = moc.Act8Set(s["xq"], s["xe"], s["sel"], s["gq"], s["ge"], s["uq"], s["ue"])
        if not kept:
            kept["ws"] = scratch(moc.workspace_bytes(s["T"], s["d"], s["F"], s["K"], s["dy"].dtype, moc.OP_BWD_ACT8))
            kept["out"] = (torch.empty_like(s["dy"]),) + tuple(torch.empty_like(w) for w in s["w"])
        if s["experts"]:
            grads = moc.moc_ffn_bwd_experts_act8(saved, s["offsets"], *s["w"], s["dy"], ws=kept["ws"], out=kept["out"])
        else:
            grads = moc.moc_ffn_bwd_act8(saved, *s["w"], s["dy"], ws=kept["ws"], out=kept["out"])
        return dict(zip(("dx", "dwg", "dwu", "dwd"), grads))
    T, E, k = s["T"], s["E"], s["k"]
    if not kept:
        kept["out"] = (empty(T, k, dtype=torch.int32), empty(T, k, dtype=torch.float32), empty(E, dtype=torch.int32), empty(T * k, dtype=torch.int32),
                       empty(1, dtype=torch.float32), empty(E, dtype=torch.float32))
        kept["ws"] = scratch(moc.route_workspace_bytes(T, E, k))
        kept["grad"] = torch.empty_like(s["logits"])
    ids, w, counts, order, loss, coef = moc.moc_route(s["logits"], k, valid=s["valid"], renorm=s["renorm"], ws=kept["ws"], out=kept["out"])
    dl = moc.moc_route_bwd(s["logits"], ids, coef, s["dweights"], s["dloss"], renorm=s["renorm"], out=kept["grad"])
    return {"ids": ids, "weights": w, "counts": counts, "order": order, "loss": loss, "coef": coef, "dlogits": dl}


def run(s):
    if own:
        return _own(s)
    return {"norm": _plain_norm, "saved": _plain_saved, "bwd": _plain_bwd, "route": _plain_route}[s["kind"]](s)


def work(case):
    """Bytes: every input and every output once.  Operations: those of the products on the selected channels; a few per element otherwise."""
    T, es = case["T"], 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "norm":
        d = case["d"]
        rows = 1 + (not case["rms"]) + (2 + case["dres"] if case["bwd"] else 0)        # h, out; dy, dres, dh
        return {"bytes": rows * T * d * es + (2 + 2 * case["bias"]) * d * es, "flops": (8.0 + 14.0 * case["bwd"]) * T * d}
    if case["kind"] == "route":
        E, k = case["E"], case["k"]
        return {"bytes": 2 * T * E * es + T * k * 16 + T * case["padded"] + 8 * E, "flops": 20.0 * T * E}
    d, F, K = case["d"], case["F"], case["K"]
    stored = T * (d + 2 * K + (d + 2 * K) / 32 + F / 8)
    if case["kind"] == "saved":
        return {"bytes": 2 * T * (d * es + K * (4 + 2 * es)) + T * F / 8, "flops": 8.0 * T * (d + 2 * K)}
    return {"bytes": stored + 6 * max(1, case["experts"]) * F * d * es + 2 * T * d * es, "flops": 12.0 * T * d * K}


# ------------------------------------------------------------------------------------ the definitions in 64 bits
def _exact_norm(s):
    h, gain = s["h"].double().requires_grad_(), s["gain"].double().requires_grad_()
    shift = s["shift"].double().requires_grad_() if s["bias"] else None
    mean = 0.0 if s["rms"] else h.sum(1, keepdim=True) / s["d"]
    n = (h - mean) / torch.sqrt(((h - mean) ** 2).sum(1, keepdim=True) / s["d"] + EPS)
    y = n * gain if shift is None else n * gain + shift
    out = {} if s["rms"] else {"out": y.detach()}
    if s["bwd"]:
        leaves = [h, gain] + ([shift] if s["bias"] else [])
        out.update(zip(("dh", "dgain", "dbias"), torch.autograd.grad(y, leaves, s["dy"].double())))
        if s["dres"]:
            out["dh"] = out["dh"] + s["res"].double()
    return out


def _restored64(v):
    """What the 8-bit form keeps of v, from its definition in 64 bits."""
    T, n = v.shape
    b = torch.nn.functional.pad(v.double(), (0, -n % 32)).view(T, -1, 32)
    top = torch.frexp(b.abs().amax(2, keepdim=True))[1] - 1            # the largest magnitude is in [2^top, 2^(top + 1))
    step = ((top.long() - 6 + 1023) << 52).view(torch.float64)
    return (torch.round(b / step).clamp(-127, 127) * step).view(T, -1)[:, :n]


def _exact_saved(s):
    return {"sel": None, "x": _restored64(s["x"]), "idx": None, "g": _restored64(s["g"]), "u": _restored64(s["u"])}


def _values64(q, e):
    step = ((e.long() - 133 + 1023) << 52).view(torch.float64).repeat_interleave(32, dim=1)[:, :q.shape[1]]
    return q.double() * step


def _exact_bwd(s):
    """Expert by expert: dense g and u are leaves, the selected channels' z = SiLU(g) u goes through W_down."""
    T, F, at = s["T"], s["F"], s["offsets"]
    lane = torch.arange(32, device=s["sel"].device, dtype=torch.int32)
    bits = ((s["sel"].unsqueeze(2) >> lane) & 1).bool().view(T, -1)[:, :F]
    w = [v.double().view(-1, F, s["d"]) for v in s["w"]]
    parts = []
    for e in range(w[0].shape[0]):
        r = slice(at[e], at[e + 1])
        m = bits[r]
        g = torch.zeros(m.shape, dtype=torch.float64, device=m.device)
        u = torch.zeros_like(g)
        g[m], u[m] = _values64(s["gq"], s["ge"])[r].reshape(-1), _values64(s["uq"], s["ue"])[r].reshape(-1)
        g.requires_grad_(), u.requires_grad_()
        wd = w[2][e].clone().requires_grad_()
        z = g * torch.sigmoid(g) * u * m
        dg, du, dwd = torch.autograd.grad(z @ wd, (g, u, wd), s["dy"][r].double())
        x = _values64(s["xq"], s["xe"])[r]
        parts.append((dg @ w[0][e] + du @ w[1][e], dg.t() @ x, du.t() @ x, dwd))
    shape = s["w"][0].shape
    return {"dx": torch.cat([p[0] for p in parts]), **{n: torch.stack([p[i] for p in parts]).view(shape) for i, n in ((1, "dwg"), (2, "dwu"), (3, "dwd"))}}


def _exact_route(s):
    T, E, k = s["T"], s["E"], s["k"]
    lo = s["logits"].double().requires_grad_()
    # rank of every expert in its row: larger logits, and equal ones of lower experts, are before it
    v = lo.detach()
    before = (v.unsqueeze(1) > v.unsqueeze(2)) | ((v.unsqueeze(1) == v.unsqueeze(2)) & (torch.arange(E, device=v.device) < torch.arange(E, device=v.device).unsqueeze(1)))
    ids = torch.argsort(before.sum(2), dim=1)[:, :k]
    mask = torch.ones(T, dtype=torch.float64, device=v.device) if s["valid"] is None else (s["valid"] > 0).double()
    p = torch.softmax(lo, 1)
    w = p.gather(1, ids)
    w = (w / w.sum(1, keepdim=True) if s["renorm"] else w) * mask.unsqueeze(1)
    counts = torch.zeros(E, dtype=torch.float64, device=v.device).index_add_(0, ids.reshape(-1), mask.repeat_interleave(k))
    N = mask.sum()
    share = counts / counts.sum()
    loss = (E * (share * (p * mask.unsqueeze(1)).sum(0) / N).sum()).view(1)
    dl, = torch.autograd.grad((w * s["dweights"].double()).sum() + loss[0] * s["dloss"][0].double(), lo)
    return {"ids": None, "weights": w.detach(), "counts": None, "order": None, "loss": loss.detach(), "coef": E * share / N, "dlogits": dl}


def exact(case, seed):
    return {"norm": _exact_norm, "saved": _exact_saved, "bwd": _exact_bwd, "route": _exact_route}[case["kind"]](prepare(case, seed))
