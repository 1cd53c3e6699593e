"""Host-side checks of the norms, the 8-bit set and the router that need no GPU: sizes, refusals before anything is launched, and what the
native marshalling leaves to the ctypes path."""
import ctypes

import pytest
import torch

from paper_2511_09323_amd import binding as B

FAKE = ctypes.c_void_p(0x1000)      # aligned, never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1004)


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def _set(**other):
    return ctypes.byref(B.MocAct8Set(*(other.get(n, 0x1000) for n in B.Act8Set._fields)))


def test_norm_refusals(lib):
    ws = 1 << 30
    ln, lb, rb = lib.moc_layernorm, lib.moc_layernorm_bwd, lib.moc_rmsnorm_bwd
    for T, d, dt, rc in ((0, 16, 0, -1), (4, 0, 0, -1), (4, 16, 2, -1), (-1, 16, 1, -1), (4, 16385, 1, -3)):
        assert ln(T, d, dt, FAKE, FAKE, FAKE, 1e-5, FAKE, None) == rc
        assert lb(T, d, dt, FAKE, FAKE, 1e-5, FAKE, None, FAKE, FAKE, FAKE, FAKE, ws, None) == rc
        assert rb(T, d, dt, FAKE, FAKE, 1e-5, FAKE, None, FAKE, FAKE, FAKE, ws, None) == rc
        assert lib.moc_norm_bwd_workspace_bytes(T, d, dt) == 0
    assert ln(4, 16, 0, None, FAKE, FAKE, 1e-5, FAKE, None) == -1 and b"h is NULL" in lib.moc_last_error()
    assert ln(4, 16, 0, FAKE, FAKE, ODD, 1e-5, FAKE, None) == -1 and b"aligned" in lib.moc_last_error()
    assert lb(4, 16, 0, FAKE, FAKE, 1e-5, FAKE, ODD, FAKE, FAKE, None, FAKE, ws, None) == -1
    assert lb(4, 16, 0, FAKE, FAKE, 1e-5, FAKE, None, FAKE, FAKE, ODD, FAKE, ws, None) == -1
    assert rb(4, 16, 0, FAKE, FAKE, 1e-5, FAKE, None, FAKE, None, FAKE, ws, None) == -1
    need = lib.moc_norm_bwd_workspace_bytes(4, 16, 0)
    assert 0 < need <= lib.moc_norm_bwd_workspace_bytes(4096, 16, 0)
    assert lb(4, 16, 0, FAKE, FAKE, 1e-5, FAKE, None, FAKE, FAKE, FAKE, FAKE, need - 1, None) == -2
    assert rb(4, 16, 0, FAKE, FAKE, 1e-5, FAKE, None, FAKE, FAKE, FAKE, need - 1, None) == -2
    assert rb(4, 16, 0, FAKE, FAKE, 1e-5, FAKE, None, FAKE, FAKE, None, ws, None) == -1


def test_act8_refusals(lib):
    good, bad = B.MocShape(4, 64, 128, 16, B.MOC_BF16), B.MocShape(4, 64, 128, 129, B.MOC_BF16)
    w = [FAKE] * 4
    assert lib.moc_act8_save(ctypes.byref(bad), *w, _set(), None) == -1
    assert lib.moc_act8_load(ctypes.byref(bad), _set(), *w, None) == -1
    assert lib.moc_act8_save(ctypes.byref(good), *w, None, None) == -1 and b"set is NULL" in lib.moc_last_error()
    for n in B.Act8Set._fields:
        for p in (None, 0x1004):
            assert lib.moc_act8_save(ctypes.byref(good), *w, _set(**{n: p}), None) == -1 and n.encode() in lib.moc_last_error()
            assert lib.moc_act8_load(ctypes.byref(good), _set(**{n: p}), *w, None) == -1
            assert lib.moc_ffn_bwd_act8(ctypes.byref(good), _set(**{n: p}), *[FAKE] * 9, 1 << 30, None) == -1
    assert lib.moc_act8_save(ctypes.byref(good), FAKE, None, FAKE, FAKE, _set(), None) == -1
    assert lib.moc_act8_load(ctypes.byref(good), _set(), FAKE, FAKE, ODD, FAKE, None) == -1
    need = lib.moc_workspace_bytes(ctypes.byref(good), B.OP_BWD_ACT8)
    assert need >= lib.moc_workspace_bytes(ctypes.byref(good), B.OP_BWD) + 4 * 64 * 2
    assert lib.moc_ffn_bwd_act8(ctypes.byref(good), _set(), *[FAKE] * 9, need - 1, None) == -2
    off = (ctypes.c_int32 * 3)(0, 3, 4)
    assert lib.moc_ffn_bwd_experts_act8(ctypes.byref(good), 2, off, _set(), *[FAKE] * 9, need - 1, None) == -2
    assert lib.moc_ffn_bwd_experts_act8(ctypes.byref(good), 2, (ctypes.c_int32 * 3)(0, 5, 4), _set(), *[FAKE] * 9, 1 << 30, None) == -1
    assert lib.moc_ffn_bwd_experts_act8(ctypes.byref(good), 9, off, _set(), *[FAKE] * 9, 1 << 30, None) == -3
    assert lib.moc_ffn_bwd_act8(ctypes.byref(good), _set(), FAKE, FAKE, FAKE, FAKE, None, *[FAKE] * 4, 1 << 30, None) == -1


def test_route_refusals(lib):
    out = [FAKE] * 6
    for T, E, k, dt, rc in ((0, 8, 2, 0, -1), (4, 0, 1, 0, -1), (4, 8, 0, 0, -1), (4, 8, 9, 0, -1), (4, 8, 2, 3, -1), (4, 257, 2, 0, -3), (4, 64, 17, 0, -3),
                            (2147483647, 8, 2, 0, -3), (2147483647, 8, 1, 0, -3)):
        assert lib.moc_route(T, E, k, dt, 1, FAKE, None, *out, FAKE, 1 << 40, None) == rc, (T, E, k, dt)
        assert lib.moc_route_bwd(T, E, k, dt, 1, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None) == rc
    assert lib.moc_route_workspace_bytes(4, 8, 9) == 0 and lib.moc_route_workspace_bytes(0, 8, 2) == 0
    need = lib.moc_route_workspace_bytes(4096, 8, 2)
    assert lib.moc_route(4096, 8, 2, 0, 1, FAKE, None, *out, FAKE, need - 1, None) == -2
    assert lib.moc_route(4, 8, 2, 0, 1, FAKE, ODD, *out, FAKE, 1 << 20, None) == -1
    for i in range(6):
        assert lib.moc_route(4, 8, 2, 0, 1, FAKE, None, *(out[:i] + [None] + out[i + 1:]), FAKE, 1 << 20, None) == -1
    assert lib.moc_route_bwd(4, 8, 2, 0, 1, FAKE, FAKE, None, FAKE, FAKE, FAKE, None) == -1
    assert lib.moc_route_bwd(4, 8, 2, 0, 1, FAKE, FAKE, FAKE, ODD, FAKE, FAKE, None) == -1


def test_host_tensors_are_refused_by_name(lib):
    h, g = torch.zeros(4, 64), torch.zeros(64)
    ws, idx = torch.zeros(1 << 16, dtype=torch.uint8), torch.zeros(4, 16, dtype=torch.int32)
    v, w = torch.zeros(4, 16), torch.zeros(128, 64)
    saved = B.act8_empty(4, 64, 128, 16, "cpu")
    for call in (lambda: B.moc_layernorm(h, g, None, 1e-5), lambda: B.moc_layernorm(h, g, g, 1e-5, out=h),
                 lambda: B.moc_layernorm_bwd(h, g, 1e-5, h, ws=ws, out=(h, g, None)), lambda: B.moc_rmsnorm_bwd(h, g, 1e-5, h),
                 lambda: B.moc_act8_save(h, idx, v, v, 128), lambda: B.moc_act8_save(h, idx, v, v, 128, out=saved),
                 lambda: B.moc_act8_load(saved, 128, torch.float32), lambda: B.moc_ffn_bwd_act8(saved, w, w, w, h),
                 lambda: B.moc_ffn_bwd_experts_act8(saved, [0, 4], w[None], w[None], w[None], h, ws=ws, out=(h, w[None], w[None], w[None])),
                 lambda: B.moc_route(h, 2), lambda: B.moc_route_bwd(h, idx, g)):
        with pytest.raises(B.MocError, match="must be a GPU tensor"):
            call()
    for call in (lambda: B.moc_layernorm(g, g, None, 1e-5), lambda: B.moc_layernorm(h.half(), g, None, 1e-5), lambda: B.moc_act8_load(saved, 128, torch.float16),
                 lambda: B.moc_ffn_bwd_experts_act8(saved, [0, 4], w, w, w, h), lambda: B.moc_ffn_bwd_act8(saved[:6], w, w, w, h), lambda: B.moc_route(h.long(), 2)):
        with pytest.raises(B.MocError):
            call()


def test_marshalling_leaves_host_tensors_alone(lib):
    f = B._fast
    h, g, ws = torch.zeros(4, 64), torch.zeros(64), torch.zeros(1 << 16, dtype=torch.uint8)
    idx, v, w = torch.zeros(4, 16, dtype=torch.int32), torch.zeros(4, 16), torch.zeros(128, 64)
    s = tuple(B.act8_empty(4, 64, 128, 16, "cpu"))
    for status in (f.layernorm(h, g, None, 1e-5, h), f.layernorm(h, g, None, 1, h), f.layernorm_bwd(h, g, 1e-5, h, None, h, g, None, ws),
                   f.rmsnorm_bwd(h, g, 1e-5, h, None, h, g, ws), f.rmsnorm_bwd(h, g), f.act8_save(h, idx, v, v, 128, *s), f.act8_load(128, *s, h, idx, v, v),
                   f.bwd_act8(*s, w, w, w, h, h, w, w, w, ws), f.bwd_experts_act8([0, 4], *s, w[None], w[None], w[None], h, h, w[None], w[None], w[None], ws),
                   f.route(h, 2, None, True, idx, v, g, idx, g, g, ws), f.route(None, 2, None, True, idx, v, g, idx, g, g, ws),
                   f.route_bwd(h, idx, g, None, None, True, h), f.route_bwd(h, idx, g, None, None, 1, h)):
        assert status == B._NOT_TAKEN
