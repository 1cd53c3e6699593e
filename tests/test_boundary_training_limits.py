"""Host-side checks at the limits of the 8-bit sets, the norms and the router that need no GPU: sizes of workspaces and refusals before anything is launched."""
import ctypes

import pytest

from paper_2511_09323_amd import binding as B

FAKE = ctypes.c_void_p(0x1000)      # aligned, never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def _set():
    return ctypes.byref(B.MocAct8Set(*[0x1000] * 7))


@pytest.mark.parametrize("dtype,size,last", [(B.MOC_BF16, 2, 27264), (B.MOC_F32, 4, 13632)])
def test_workspaces_of_wide_layers_hold_the_whole_set(lib, dtype, size, last):
    """Up to `last` channels the backward from 8 bits restores x alone, past it idx, gvals and uvals, too (every piece 256-byte aligned)."""
    T, d, K = 40, 64, 300
    for F in (last, last + 1):
        shape = ctypes.byref(B.MocShape(T, d, F, K, dtype))
        more = lib.moc_workspace_bytes(shape, B.OP_BWD_ACT8) - lib.moc_workspace_bytes(shape, B.OP_BWD)
        assert 0 <= more - T * d * size - (T * K * (4 + 2 * size) if F > last else 0) < 4 * 256


def test_rows_past_a_launch_are_refused_by_the_backward_from_8_bits(lib):
    """Before anything is launched: -3, and what the next check finds (a workspace too small) up to the limit."""
    most = (1 << 24) - 8192
    for T, F, rc in ((most, 4096, -2), (most + 1, 4096, -3), (most // 2, 4097, -2), (most // 2 + 1, 4097, -3), (most // 2, 8192, -2), (most // 2, 8193, -3), (1 << 24, 32, -3),
                     (2147483647, 64, -3)):
        shape = ctypes.byref(B.MocShape(T, 8, F, 1, B.MOC_BF16))
        assert lib.moc_ffn_bwd_act8(shape, _set(), *[FAKE] * 9, 256, None) == rc, (T, F)
        assert lib.moc_ffn_bwd_experts_act8(shape, 1, (ctypes.c_int32 * 2)(0, T), _set(), *[FAKE] * 9, 256, None) == rc, (T, F)


def test_widths_that_no_set_has_are_refused_by_all(lib):
    for d, rc in (((1 << 24) + 8, -3), ((1 << 31) - 8, -3)):
        shape, w = ctypes.byref(B.MocShape(1, d, 64, 8, B.MOC_BF16)), [FAKE] * 4
        assert lib.moc_act8_save(shape, *w, _set(), None) == rc and lib.moc_act8_load(shape, _set(), *w, None) == rc
        assert lib.moc_ffn_bwd_act8(shape, _set(), *[FAKE] * 9, 256, None) == rc
        assert lib.moc_ffn_bwd_experts_act8(shape, 1, (ctypes.c_int32 * 2)(0, 1), _set(), *[FAKE] * 9, 256, None) == rc
    shape = ctypes.byref(B.MocShape(1, 1 << 24, 64, 8, B.MOC_BF16))
    assert lib.moc_ffn_bwd_act8(shape, _set(), *[FAKE] * 9, 256, None) == -2
