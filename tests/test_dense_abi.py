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
    saved = hire._lib.hire_gated_ffn_saved_bytes
    assert saved(C.byref(gated(hire)), 3) == 4 * 3 * 16384 * 2
    for size in (fwd, bwd, saved):
        assert size(C.byref(gated(hire)), 0) == 0 and size(C.byref(gated(hire)), (1 << 20) + 1) == 0 and size(None, 1) == 0
        for bad, _ in BAD_GATED:
            assert size(C.byref(gated(hire, **bad)), 1) == 0


def test_gated_refusals(hire):
    def step(T=3, x=0x40000, y=0x50000, saved=None, ws=0x60000, nbytes=256, **layer):
        return hire._lib.hire_gated_ffn_step(C.byref(gated(hire, **layer)), x, T, y, saved, ws, nbytes, None)

    def back(T=3, x=0x40000, saved=0x41000, dy=0x44000, outs=(0x45000,) * 4, ws=0x60000, nbytes=256, **layer):
        return hire._lib.hire_gated_ffn_backward(C.byref(gated(hire, **layer)), x, T, saved, dy, *outs, ws, nbytes, None)

    for call in (step, back):
        assert call() == ENOSPC                       # all else is right
        for bad, code in BAD_GATED:
            assert call(**bad) == code, bad
        for name in ("wg", "wu", "w2"):
            assert call(**{name: None}) == EINVAL and call(**{name: 0x10080}) == EINVAL
        assert call(T=0) == EINVAL and call(T=-1) == EINVAL and call(T=(1 << 20) + 1) == EUNSUPPORTED
        assert call(x=None) == EINVAL and call(x=0x40008) == EINVAL and call(ws=None) == EINVAL and call(ws=0x60010) == EINVAL
        assert call(saved=0x41080) == EINVAL and call(saved=0x41000) == ENOSPC
    assert step(y=None) == EINVAL and step(y=0x50002) == EINVAL
    assert back(saved=None) == EINVAL and back(dy=None) == EINVAL and back(dy=0x44008) == EINVAL
    assert back(outs=(None,) * 4) == EINVAL and back(outs=(0x1008, None, None, None)) == EINVAL
    assert back(outs=(None, None, None, 0x1000)) == ENOSPC
    assert hire._lib.hire_gated_ffn_step(None, 0x40000, 1, 0x50000, None, 0x60000, 256, None) == EINVAL


def test_mxfp4_refusals(hire):
    lib = hire._lib
    for f in (lambda rows, cols, w=0x1000, c=0x2000, s=0x3001: lib.hire_pack_mxfp4(w, rows, cols, c, s, None),
              lambda rows, cols, w=0x1000, c=0x2000, s=0x3001: lib.hire_unpack_mxfp4(c, s, rows, cols, w, None)):
        for rows, cols in ((0, 32), (-1, 32), (1, 0), (1, 16), (1, 40), (1, -32)):
            assert f(rows, cols) == EINVAL
        assert f(1, 32, w=None) == EINVAL and f(1, 32, c=None) == EINVAL and f(1, 32, s=None) == EINVAL
        assert f(1, 32, w=0x1008) == EINVAL and f(1, 32, c=0x2004) == EINVAL

    size = lib.hire_mxfp4_product_workspace_bytes
    assert size(1, 1, 32) > 0 and size(1 << 20, 1 << 24, 1 << 20) > 0
    limits = [((0, 5, 64), EINVAL), ((1, 0, 64), EINVAL), ((1, 5, 0), EINVAL), ((1, 5, 48), EINVAL),
              (((1 << 20) + 1, 5, 64), EUNSUPPORTED), ((1, (1 << 24) + 1, 64), EUNSUPPORTED), ((1, 5, (1 << 20) + 32), EUNSUPPORTED)]

    def packed(T=2, rows=5, cols=64, x=0x1000, xs=0x2000, w=0x3000, s=0x4000, y=0x5000, kind=0, ws=0x6000, nbytes=0):
        return lib.hire_mxfp4_product(x, xs, T, w, s, rows, cols, y, kind, ws, nbytes, None)

    def bf16(T=2, rows=5, cols=64, x=0x1000, w=0x3000, s=0x4000, y=0x5000, kind=0, ws=0x6000, nbytes=0):
        return lib.hire_mxfp4_product_bf16(x, T, w, s, rows, cols, y, kind, ws, nbytes, None)

    for call in (packed, bf16):
        assert call() == ENOSPC and call(kind=1) == ENOSPC
        assert call(kind=2) == EINVAL and call(kind=-1) == EINVAL
        for (T, rows, cols), code in limits:
            assert call(T=T, rows=rows, cols=cols) == code and size(T, rows, cols) == 0
        for name in ("x", "w", "y", "ws"):
            assert call(**{name: None}) == EINVAL and call(**{name: 0x1008}) == EINVAL
        assert call(s=None) == EINVAL
    assert packed(xs=None) == EINVAL
    assert bf16(T=65) == EUNSUPPORTED and packed(T=65) == ENOSPC


def test_draft_refusals(hire):
    lib = hire._lib
    base = dict(B=2, n=3, vocab=100, lengths=None, tokens=0x100, target_prob=0x200, target_idx=None, target_k=0,
                draft_prob=0x300, draft_idx=None, draft_k=0, accept_u=0x400, sample_u=0x500)

    def call(out=0x600, acc=0x700, ws=0x800, nbytes=0, **changes):
        d = hire._Drafts(**{**base, **changes})
        code = lib.hire_verify_draft(C.byref(d), out, acc, ws, nbytes, None)
        size = lib.hire_verify_draft_workspace_bytes(C.byref(d))
        return code, size

    code, size = call()
    assert code == ENOSPC and size > 0
    lists = dict(target_idx=0x900, target_k=64, draft_idx=0xA00, draft_k=4096)
    assert call(**lists)[0] == ENOSPC and call(lengths=0x40)[0] == ENOSPC and call(draft_prob=None)[0] == ENOSPC
    assert call(n=0, tokens=None, accept_u=None, draft_prob=None)[0] == ENOSPC
    for bad in (dict(B=0), dict(B=-1), dict(n=-1), dict(vocab=0), dict(tokens=None), dict(tokens=0x101), dict(target_prob=None),
                dict(target_prob=0x202), dict(accept_u=None), dict(sample_u=None), dict(lengths=0x41), dict(n=0),
                dict(draft_idx=0x900, draft_k=5, draft_prob=None), dict(target_idx=0x900, target_k=0),
                dict(draft_idx=0x900, draft_k=0), dict(draft_idx=0x900, draft_k=-3), dict(target_idx=0x901, target_k=4)):
        assert call(**bad) == (EINVAL, 0), bad
    for bad in (dict(B=4097), dict(n=64), dict(vocab=(1 << 22) + 1), dict(target_idx=0x900, target_k=4097),
                dict(draft_idx=0x900, draft_k=4097)):
        assert call(**bad) == (EUNSUPPORTED, 0), bad
    for bad in (dict(out=None), dict(acc=None), dict(ws=None), dict(out=0x602), dict(ws=0x810)):
        assert call(**bad)[0] == EINVAL, bad
    assert lib.hire_verify_draft(None, 0x600, 0x700, 0x800, 1 << 20, None) == EINVAL
    assert call(B=4096, vocab=1 << 22)[1] > 0
