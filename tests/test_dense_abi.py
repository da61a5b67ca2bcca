"""Host-side checks of the dense operators' entry points, without a GPU: sizes of workspaces, and every argument error
before anything is enqueued (fake pointers, never dereferenced)."""
import ctypes as C

import pytest

OK, EINVAL, ENOSPC, EUNSUPPORTED = 0, -1, -2, -3


@pytest.fixture(scope="module")
def hire():
    from paper_2402_09360_amd import hire as H
    return H


def gated(hire, d=2048, ff=16384, wg=0x10000, wu=0x20000, w2=0x30000, act=1):
    return hire._GatedLayer(d, ff, wg, wu, w2, act)


BAD_GATED = [(dict(d=2052), EINVAL), (dict(d=0), EINVAL), (dict(ff=-8), EINVAL), (dict(ff=12), EINVAL), (dict(act=3), EINVAL),
             (dict(act=-1), EINVAL), (dict(d=(1 << 20) + 8), EUNSUPPORTED), (dict(ff=(1 << 20) + 8), EUNSUPPORTED)]


def test_gated_workspaces(hire):
    fwd, bwd = hire._lib.hire_gated_ffn_workspace_bytes, hire._lib.hire_gated_ffn_backward_workspace_bytes
    for T in (1, 16, 64, 65, 1000, 100000):
        assert 0 < fwd(C.byref(gated(hire)), T) and fwd(C.byref(gated(hire)), T) % 256 == 0
        assert bwd(C.byref(gated(hire)), T) >= 2 * T * 16384 * 2
    for size in (fwd, bwd):
        assert size(C.byref(gated(hire)), 0) == 0 and size(C.byref(gated(hire)), (1 << 20) + 1) == 0 and size(None, 1) == 0
        for bad, _ in BAD_GATED:
            assert size(C.byref(gated(hire, **bad)), 1) == 0


def test_gated_refusals(hire):
    def step(T=3, x=0x40000, y=0x50000, g=None, u=None, h=None, ws=0x60000, nbytes=256, **layer):
        return hire._lib.hire_gated_ffn_step(C.byref(gated(hire, **layer)), x, T, y, g, u, h, ws, nbytes, None)

    def back(T=3, x=0x40000, g=0x41000, u=0x42000, h=0x43000, dy=0x44000, outs=(0x45000,) * 4, ws=0x60000, nbytes=256, **layer):
        return hire._lib.hire_gated_ffn_backward(C.byref(gated(hire, **layer)), x, T, g, u, h, dy, *outs, ws, nbytes, None)

    for call in (step, back):
        assert call() == ENOSPC                       # all else is right
        for bad, code in BAD_GATED:
            assert call(**bad) == code, bad
        for name in ("wg", "wu", "w2"):
            assert call(**{name: None}) == EINVAL and call(**{name: 0x10080}) == EINVAL
        assert call(T=0) == EINVAL and call(T=-1) == EINVAL and call(T=(1 << 20) + 1) == EUNSUPPORTED
        assert call(x=None) == EINVAL and call(x=0x40008) == EINVAL and call(ws=None) == EINVAL and call(ws=0x60010) == EINVAL
    assert step(y=None) == EINVAL and step(y=0x50002) == EINVAL
    assert step(g=0x1000) == EINVAL and step(g=0x1000, u=0x2000) == EINVAL and step(u=0x1000, h=0x2000) == EINVAL
    assert step(g=0x1008, u=0x2000, h=0x3000) == EINVAL and step(g=0x1000, u=0x2000, h=0x3000) == ENOSPC
    for name in ("g", "u", "h", "dy"):
        assert back(**{name: None}) == EINVAL and back(**{name: 0x1008}) == EINVAL
    assert back(outs=(None,) * 4) == EINVAL and back(outs=(0x1008, None, None, None)) == EINVAL
    assert back(outs=(None, None, None, 0x1000)) == ENOSPC
    assert hire._lib.hire_gated_ffn_step(None, 0x40000, 1, 0x50000, None, None, None, 0x60000, 256, None) == EINVAL
