"""Refusals of the dense 8-bit scores, the check of drafted labels and dropout: the C entry points return a status before
anything touches a device, the binding raises before it calls them (no GPU needed)."""
import ctypes

import pytest
import torch

EINVAL, ESHAPE, EWORKSPACE, EDTYPE = -1, -2, -3, -5
P = ctypes.c_void_p(4096)                                  # an aligned address that no accepted call is made with
ODD = ctypes.c_void_p(4100)


@pytest.fixture(scope="module")
def lib():
    from paper_2409_20156_amd import binding
    return binding.load_library()


def _size(fn, *args):
    n = ctypes.c_size_t(0)
    return fn(*args, ctypes.byref(n)), n.value


def test_quantize_rows(lib):
    def call(X=P, N=10, d=64, t=1, ids=None, m=0, count=None, Q=P, scale=P):
        return lib.xc_quantize_rows(X, N, d, t, ids, m, count, Q, scale, None)
    assert call(t=2) == EDTYPE
    assert call(N=0) == ESHAPE and call(d=60) == ESHAPE and call(d=0) == ESHAPE and call(d=131080) == ESHAPE
    assert call(d=66, t=0) == ESHAPE and call(m=-1, ids=P) == ESHAPE
    assert call(X=None) == EINVAL and call(Q=None) == EINVAL and call(scale=None) == EINVAL
    assert call(X=ODD) == EINVAL and call(Q=ODD) == EINVAL and call(scale=ODD) == EINVAL
    assert call(ids=ODD, m=4) == EINVAL and call(count=P) == EINVAL and call(ids=P, m=4, count=ODD) == EINVAL
    assert call(ids=P, m=0) == 0                           # an empty list: nothing to do


def test_scores(lib):
    rc, need = _size(lib.xc_scores_workspace, 100, 72)
    assert rc == 0 and need >= 100 * (80 + 4)
    assert _size(lib.xc_scores_workspace, 0, 72)[0] == ESHAPE and _size(lib.xc_scores_workspace, 1, 131073)[0] == ESHAPE
    assert lib.xc_scores_workspace(100, 72, None) == EINVAL

    def call(Z=P, B=100, d=72, t=1, Q=P, scale=P, L=1000, out_t=0, out=P, ws=P, ws_bytes=need):
        return lib.xc_scores_quantized(Z, B, d, t, Q, scale, L, out_t, out, ws, ws_bytes, None)
    assert call(t=5) == EDTYPE and call(out_t=2) == EDTYPE
    assert call(B=0) == ESHAPE and call(L=0) == ESHAPE and call(L=1 << 31) == ESHAPE and call(d=70) == ESHAPE
    assert call(d=66, t=0) == ESHAPE and call(d=131080) == ESHAPE
    for name in ("Z", "Q", "scale", "out", "ws"):
        assert call(**{name: None}) == EINVAL and call(**{name: ODD}) == EINVAL
    assert call(ws_bytes=need - 1) == EWORKSPACE


def test_verify(lib):
    rc, need = _size(lib.xc_verify_workspace, 7, 50021)
    assert rc == 0 and need > 0
    assert _size(lib.xc_verify_workspace, 0, 10)[0] == ESHAPE and _size(lib.xc_verify_workspace, 1, 1 << 31)[0] == ESHAPE
    assert lib.xc_verify_workspace(7, 50021, None) == EINVAL

    def call(drafts=P, B=7, n=3, V=50021, target=P, draft=P, t=0, u=P, tokens=P, accepted=P, ws=P, ws_bytes=need):
        return lib.xc_verify_drafts(drafts, B, n, V, target, draft, t, u, tokens, accepted, ws, ws_bytes, None)
    assert call(t=2) == EDTYPE
    assert call(B=0) == ESHAPE and call(n=-1) == ESHAPE and call(n=1025) == ESHAPE and call(V=0) == ESHAPE and call(V=1 << 31) == ESHAPE
    for name in ("drafts", "target", "u", "tokens", "accepted", "ws"):
        assert call(**{name: None}) == EINVAL and call(**{name: ODD}) == EINVAL
    assert call(draft=ODD) == EINVAL
    assert call(ws_bytes=need - 1) == EWORKSPACE


def test_dropout(lib):
    def call(X=P, t=0, B=4, d=9, rate=0.1, seed=1, row0=0, Y=ctypes.c_void_p(8192), out_t=0):
        return lib.xc_dropout(X, t, B, d, rate, seed, row0, Y, out_t, None)
    assert call(t=2) == EDTYPE and call(out_t=-1) == EDTYPE
    assert call(B=0) == ESHAPE and call(d=0) == ESHAPE and call(d=1 << 31) == ESHAPE and call(B=1 << 59, d=4) == ESHAPE
    for rate in (-0.1, 1.0, 0.999999, float("nan"), float("inf")):
        assert call(rate=rate) == EINVAL
    assert call(row0=-1) == EINVAL
    assert call(X=None) == EINVAL and call(Y=None) == EINVAL and call(X=ODD) == EINVAL and call(Y=ODD) == EINVAL
    assert call(Y=P, out_t=1) == EINVAL                    # in place, but the types differ
    assert call(X=ctypes.c_void_p(8192 - 128)) == EINVAL and call(X=ctypes.c_void_p(8192 + 128)) == EINVAL       # 144 bytes each: they overlap
    assert call(X=ctypes.c_void_p(8192 + 64), out_t=1) == EINVAL and call(X=ctypes.c_void_p(8192 - 64), t=1) == EINVAL     # 72 bytes of bf16


def test_binding_refuses_before_it_calls():
    import paper_2409_20156_amd as xc
    Z, Q, s = torch.zeros((3, 24)), torch.zeros((5, 32), dtype=torch.int8), torch.zeros(5)
    i32 = torch.int32
    with pytest.raises(RuntimeError, match="no CPU path"):
        xc.quantize_rows(Z)
    with pytest.raises(RuntimeError, match="no CPU path"):
        xc.scores_quantized(Z, Q, s)
    with pytest.raises(RuntimeError, match="no CPU path"):
        xc.dropout(Z, 0.1, 1)
    with pytest.raises(RuntimeError, match="no CPU path"):
        xc.verify_drafts(torch.zeros((2, 3), dtype=i32), torch.zeros((2, 4, 9)), None, torch.zeros((2, 4)))
    with pytest.raises(TypeError):
        xc.quantize_rows(Z.half())
    with pytest.raises(TypeError):
        xc.scores_quantized(Z, Q, s, dtype=torch.float16)
    with pytest.raises(TypeError):
        xc.dropout(Z.half(), 0.1, 1)
    for bad in (Q[:, :16], Q[0], torch.zeros((5, 24), dtype=torch.int8)):
        with pytest.raises(ValueError):
            xc.scores_quantized(Z, bad, s)
    with pytest.raises(ValueError):
        xc.scores_quantized(Z, Q, s[:4])
    with pytest.raises(ValueError):
        xc.scores_quantized(Z, Q, s, out=torch.zeros((3, 6)))
    with pytest.raises(ValueError):
        xc.quantize_rows(Z, rows=torch.zeros(2, dtype=i32))            # no earlier rows to keep
    with pytest.raises(ValueError):
        xc.quantize_rows(Z, count=torch.zeros(1, dtype=i32))
    with pytest.raises(ValueError):
        xc.quantize_rows(Z, out=(Q, s))
    d, t, u = torch.zeros((2, 3), dtype=i32), torch.zeros((2, 4, 9)), torch.zeros((2, 4))
    for args in ((d, t[:, :3], None, u), (d, t, t, u), (d, t, None, u[:, :3]), (d[0], t, None, u), (d, t[0], None, u),
                 (d, t, t[:, :3].bfloat16(), u)):
        with pytest.raises(ValueError):
            xc.verify_drafts(*args)
    with pytest.raises(ValueError):
        xc.dropout(Z, 0.1, 1, out=torch.zeros((3, 25)))
    with pytest.raises(ValueError):
        xc.dropout(Z[0], 0.1, 1)
