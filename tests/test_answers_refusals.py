"""Refusals of the 4-bit rows and scores, the log probabilities, their gradient and the loss against a teacher: the C entry points return
a status before anything touches a device, the binding raises before it calls them (no GPU needed)."""
import ctypes
import math

import pytest
import torch

from tests.test_overlap_refusals import _need, _overlaps, lib  # noqa: F401  (lib: a fixture)

EINVAL, ESHAPE, EWORKSPACE, EDTYPE = -1, -2, -3, -5
P = ctypes.c_void_p(4096)                                  # an aligned address that no accepted call is made with
ODD = ctypes.c_void_p(4100)


def _size(fn, *args):
    n = ctypes.c_size_t(0)
    return fn(*args, ctypes.byref(n)), n.value


def test_microscale_rows(lib):  # noqa: F811
    def call(X=P, N=10, d=64, t=1, ids=None, m=0, count=None, Q=P, scale=P):
        return lib.xc_microscale_rows(X, N, d, t, ids, m, count, Q, scale, None)
    assert call(t=2) == EDTYPE
    assert call(N=0) == ESHAPE and call(N=1 << 31) == ESHAPE and call(d=60) == ESHAPE and call(d=0) == ESHAPE and call(d=131080) == ESHAPE
    assert call(d=66, t=0) == ESHAPE and call(m=-1, ids=P) == ESHAPE
    assert call(X=None) == EINVAL and call(Q=None) == EINVAL and call(scale=None) == EINVAL
    assert call(X=ODD) == EINVAL and call(Q=ODD) == EINVAL and call(scale=ODD) == EINVAL
    assert call(ids=ODD, m=4) == EINVAL and call(count=P) == EINVAL and call(ids=P, m=4, count=ODD) == EINVAL
    far = [ctypes.c_void_p((1 << 40) + (i << 20)) for i in range(4)]
    assert call(X=far[0], Q=far[1], scale=far[2], ids=far[3], m=0) == 0                # an empty list: nothing to do


def test_scores_microscaled(lib):  # noqa: F811
    rc, need = _size(lib.xc_scores_microscaled_workspace, 100, 72)
    assert rc == 0 and need >= 100 * (64 + 4)
    assert _size(lib.xc_scores_microscaled_workspace, 0, 72)[0] == ESHAPE and _size(lib.xc_scores_microscaled_workspace, 1, 131073)[0] == ESHAPE
    assert lib.xc_scores_microscaled_workspace(100, 72, None) == EINVAL

    def call(Z=P, B=100, d=72, t=1, Q=P, scale=P, L=1000, out_t=0, out=P, ws=P, ws_bytes=need):
        return lib.xc_scores_microscaled(Z, B, d, t, Q, scale, L, out_t, out, ws, ws_bytes, None)
    assert call(t=5) == EDTYPE and call(out_t=2) == EDTYPE
    assert call(B=0) == ESHAPE and call(L=0) == ESHAPE and call(L=1 << 31) == ESHAPE and call(d=70) == ESHAPE
    assert call(d=66, t=0) == ESHAPE and call(d=131080) == ESHAPE and call(B=1 << 20, L=(1 << 20) + 1) == ESHAPE
    for name in ("Z", "Q", "scale", "out", "ws"):
        assert call(**{name: None}) == EINVAL and call(**{name: ODD}) == EINVAL
    assert call(ws_bytes=need - 1) == EWORKSPACE


def test_label_logprobs(lib):  # noqa: F811
    rc, need = _size(lib.xc_label_logprobs_workspace, 7, 50021, 20, 0)
    assert rc == 0 and need > 0
    assert _size(lib.xc_label_logprobs_workspace, 7, 50021, 20, 2)[0] == EDTYPE
    for args in ((0, 10, 1), (1, 0, 0), (1, 1 << 31, 1), (1, 10, -1), (1, 10, 11), (1, 1000, 129)):
        assert _size(lib.xc_label_logprobs_workspace, *args, 0)[0] == ESHAPE
    assert lib.xc_label_logprobs_workspace(7, 50021, 20, 0, None) == EINVAL

    def call(X=P, ld=50021, B=7, V=50021, t=0, T=1.0, labels=P, n=3, k=20, logp=P, entropy=P, norm=P, top=P, top_logp=P, ws=P, ws_bytes=need):
        return lib.xc_label_logprobs(X, ld, B, V, t, T, labels, n, k, logp, entropy, norm, top, top_logp, ws, ws_bytes, None)
    assert call(t=2) == EDTYPE
    assert call(B=0) == ESHAPE and call(V=0) == ESHAPE and call(V=1 << 31, ld=1 << 31) == ESHAPE and call(ld=50020) == ESHAPE
    assert call(B=1 << 30, ld=1 << 20) == ESHAPE and call(n=-1) == ESHAPE and call(n=257) == ESHAPE and call(k=-1) == ESHAPE and call(k=129) == ESHAPE
    assert call(V=19, ld=19) == ESHAPE                     # more alternatives than labels
    for T in (0.0, -1.0, 1e-7, 1e7, math.inf, math.nan):
        assert call(T=T) == EINVAL
    for name in ("X", "labels", "logp", "entropy", "norm", "top", "top_logp", "ws"):
        assert call(**{name: None}) == EINVAL and call(**{name: ODD}) == EINVAL
    assert call(ws_bytes=need - 1) == EWORKSPACE


def test_label_logprobs_grad(lib):  # noqa: F811
    def call(X=P, ld=100, B=7, V=100, t=0, T=1.0, labels=P, n=3, dlogp=P, norm=P, entropy=P, dentropy=P, dX=P, ldd=100, out_t=0):
        return lib.xc_label_logprobs_grad(X, ld, B, V, t, T, labels, n, dlogp, norm, entropy, dentropy, dX, ldd, out_t, None)
    assert call(t=2) == EDTYPE and call(out_t=-1) == EDTYPE
    assert call(B=0) == ESHAPE and call(V=0) == ESHAPE and call(ld=99) == ESHAPE and call(ldd=99) == ESHAPE and call(n=257) == ESHAPE and call(n=-1) == ESHAPE
    for T in (0.0, -1.0, math.nan):
        assert call(T=T) == EINVAL
    for name in ("X", "labels", "dlogp", "norm", "dX"):
        assert call(**{name: None}) == EINVAL and call(**{name: ODD}) == EINVAL
    assert call(entropy=None) == EINVAL and call(entropy=ODD) == EINVAL and call(dentropy=ODD) == EINVAL
    assert call(dX=P, out_t=1) == EINVAL and call(dX=P, ldd=104) == EINVAL             # in place, but types or distances differ


def test_distill(lib):  # noqa: F811
    rc, need = _size(lib.xc_distill_workspace, 7, 50021, 1)
    assert rc == 0 and need > 0
    assert _size(lib.xc_distill_workspace, 7, 50021, 2)[0] == EDTYPE and _size(lib.xc_distill_workspace, 0, 5, 0)[0] == ESHAPE
    assert lib.xc_distill_workspace(7, 50021, 1, None) == EINVAL

    def call(X=P, ld=50021, B=7, V=50021, t=1, T=1.0, labels=P, teacher=P, K=20, tail=0, weight=None, loss=P, dX=P, ldd=50021, out_t=1, ws=P, ws_bytes=need):
        return lib.xc_distill(X, ld, B, V, t, T, labels, teacher, K, tail, weight, loss, dX, ldd, out_t, ws, ws_bytes, None)
    assert call(t=2) == EDTYPE and call(out_t=2) == EDTYPE
    assert call(B=0) == ESHAPE and call(V=0) == ESHAPE and call(ld=50020) == ESHAPE and call(ldd=50020) == ESHAPE and call(K=0) == ESHAPE and call(K=257) == ESHAPE
    assert call(T=0.0) == EINVAL and call(T=math.nan) == EINVAL and call(tail=2) == EINVAL
    for name in ("X", "labels", "teacher", "loss", "ws"):
        assert call(**{name: None}) == EINVAL and call(**{name: ODD}) == EINVAL
    assert call(dX=ODD) == EINVAL and call(weight=ODD) == EINVAL
    assert call(ws_bytes=need - 1) == EWORKSPACE


# ---- arrays over each other
@pytest.mark.parametrize("t,N,d", [(0, 100, 60), (1, 100, 72), (1, 1, 8), (1, 5, 20000)])
@pytest.mark.parametrize("m,counted", [(0, False), (7, False), (50, True)])
def test_overlap_microscale_rows(lib, t, N, d, m, counted):  # noqa: F811
    pitch = (d + 127) // 128 * 128
    sizes = {"Q": N * pitch // 2, "scale": N * pitch // 32, "X": N * d * (2 if t else 4), "ids": m * 4, "count": 4 if counted else 0}
    for w, o, at in _overlaps(sizes, ("Q", "scale")):
        rc = lib.xc_microscale_rows(at["X"], N, d, t, at["ids"] if m else None, m, at["count"] if counted else None, at["Q"], at["scale"], None)
        assert rc == EINVAL, (w, o)


@pytest.mark.parametrize("t,out_t", [(0, 0), (1, 1)])
@pytest.mark.parametrize("B,d,L", [(3, 72, 1000), (300, 4096, 7), (1, 8, 1)])
def test_overlap_scores(lib, t, out_t, B, d, L):  # noqa: F811
    need, pitch = _need(lib.xc_scores_microscaled_workspace, B, d), (d + 127) // 128 * 128
    sizes = {"out": B * L * (2 if out_t else 4), "ws": need, "Z": B * d * (2 if t else 4), "Q": L * pitch // 2, "scale": L * pitch // 32}
    for w, o, at in _overlaps(sizes, ("out", "ws")):
        rc = lib.xc_scores_microscaled(at["Z"], B, d, t, at["Q"], at["scale"], L, out_t, at["out"], at["ws"], need, None)
        assert rc == EINVAL, (w, o)


@pytest.mark.parametrize("t", [0, 1])
@pytest.mark.parametrize("B,V,ld,n,k", [(7, 50021, 50021, 3, 20), (2, 9, 12, 0, 0), (1, 300, 300, 1, 0), (300, 70, 70, 0, 5)])
def test_overlap_label_logprobs(lib, t, B, V, ld, n, k):  # noqa: F811
    need, e = _need(lib.xc_label_logprobs_workspace, B, V, k, t), 2 if t else 4
    sizes = {"logp": B * n * 4, "entropy": B * 4, "norm": B * 8, "top": B * k * 4, "top_logp": B * k * 4, "ws": need,
             "X": ((B - 1) * ld + V) * e, "labels": B * n * 4}
    written = [w for w in ("logp", "entropy", "norm", "top", "top_logp", "ws") if sizes[w]]
    for w, o, at in _overlaps(sizes, written):
        rc = lib.xc_label_logprobs(at["X"], ld, B, V, t, 1.0, at["labels"] if n else None, n, k, at["logp"] if n else None, at["entropy"], at["norm"],
                                   at["top"] if k else None, at["top_logp"] if k else None, at["ws"], need, None)
        assert rc == EINVAL, (w, o)


@pytest.mark.parametrize("t,out_t,ldd", [(0, 0, 301), (1, 0, 300), (0, 1, 300), (1, 1, 310)])
@pytest.mark.parametrize("B,n,with_entropy", [(7, 3, True), (2, 0, True), (5, 1, False)])
def test_overlap_label_logprobs_grad(lib, t, out_t, ldd, B, n, with_entropy):  # noqa: F811
    sizes = {"dX": ((B - 1) * ldd + 300) * (2 if out_t else 4), "X": B * 300 * (2 if t else 4), "labels": B * n * 4, "dlogp": B * n * 4, "norm": B * 8,
             "entropy": B * 4 if with_entropy else 0, "dentropy": B * 4 if with_entropy else 0}
    for w, o, at in _overlaps(sizes, ("dX",)):
        rc = lib.xc_label_logprobs_grad(at["X"], 300, B, 300, t, 1.0, at["labels"] if n else None, n, at["dlogp"] if n else None, at["norm"],
                                        at["entropy"] if with_entropy else None, at["dentropy"] if with_entropy else None, at["dX"], ldd, out_t, None)
        assert rc == EINVAL, (w, o)


@pytest.mark.parametrize("t,out_t,ldd", [(0, 0, 301), (1, 0, 300), (1, 1, 310)])
@pytest.mark.parametrize("B,K,weighted,grad", [(7, 3, True, True), (2, 256, False, True), (5, 1, True, False)])
def test_overlap_distill(lib, t, out_t, ldd, B, K, weighted, grad):  # noqa: F811
    need = _need(lib.xc_distill_workspace, B, 300, t)
    sizes = {"loss": B * 4, "ws": need, "dX": ((B - 1) * ldd + 300) * (2 if out_t else 4) if grad else 0, "X": B * 300 * (2 if t else 4), "labels": B * K * 4,
             "teacher": B * K * 4, "weight": B * 4 if weighted else 0}
    for w, o, at in _overlaps(sizes, ("loss", "ws", "dX") if grad else ("loss", "ws")):
        rc = lib.xc_distill(at["X"], 300, B, 300, t, 1.0, at["labels"], at["teacher"], K, 1, at["weight"] if weighted else None, at["loss"],
                            at["dX"] if grad else None, ldd, out_t, at["ws"], need, None)
        assert rc == EINVAL, (w, o)


def test_binding_refuses_before_it_calls():
    import paper_2409_20156_amd as xc
    Z, Q, s = torch.zeros((3, 24)), torch.zeros((5, 64), dtype=torch.uint8), torch.zeros((5, 4), dtype=torch.uint8)
    i32 = torch.int32
    assert xc.microscaled_pitch(24) == 128 and xc.microscaled_pitch(129) == 256
    X, lab, t = torch.zeros((3, 50)), torch.zeros((3, 4), dtype=i32), torch.zeros((3, 4))
    norm, one = torch.zeros((3, 2)), torch.zeros(3)
    for call in (lambda: xc.microscale_rows(Z), lambda: xc.scores_microscaled(Z, Q, s), lambda: xc.label_logprobs(X, lab, top=3),
                 lambda: xc.label_logprobs_grad(X, lab, t, norm), lambda: xc.distill(X, lab, t)):
        with pytest.raises(RuntimeError, match="no CPU path"):
            call()
    for call in (lambda: xc.microscale_rows(Z.half()), lambda: xc.scores_microscaled(Z, Q, s, dtype=torch.float16), lambda: xc.label_logprobs(X.half(), lab),
                 lambda: xc.label_logprobs_grad(X, lab, t, norm, dtype=torch.float16), lambda: xc.distill(X, lab, t, dtype=torch.float16),
                 lambda: xc.distill(X.double(), lab, t)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: xc.scores_microscaled(Z, Q[:, :32], s), lambda: xc.scores_microscaled(Z, Q, s[:4]), lambda: xc.scores_microscaled(Z, Q, s, out=torch.zeros((3, 6))),
                 lambda: xc.microscale_rows(Z, rows=torch.zeros(2, dtype=i32)), lambda: xc.microscale_rows(Z, count=torch.zeros(1, dtype=i32)),
                 lambda: xc.microscale_rows(Z, out=(Q, s)), lambda: xc.label_logprobs(X[0], lab), lambda: xc.label_logprobs(X, lab[:2]),
                 lambda: xc.label_logprobs(X, lab, out={"logp": torch.zeros((3, 5))}), lambda: xc.label_logprobs_grad(X, lab, t[:, :3], norm),
                 lambda: xc.label_logprobs_grad(X, lab, t, norm[:, :1]), lambda: xc.label_logprobs_grad(X, lab, t, norm, dentropy=one),
                 lambda: xc.label_logprobs_grad(X, lab, t, norm, out=torch.zeros((3, 51))), lambda: xc.distill(X, lab, t[:, :3]), lambda: xc.distill(X, lab[0], t),
                 lambda: xc.distill(X, lab, t, weight=one[:2]), lambda: xc.distill(X, lab, t, out=(one, None)), lambda: xc.distill(X, lab, t, out=(one, torch.zeros((3, 49))))):
        with pytest.raises(ValueError):
            call()
    from paper_2409_20156_amd import binding
    cuda_like = type("T", (), {"dim": lambda self: 2, "is_cuda": True, "shape": (3, 50), "data_ptr": lambda self: 4096, "stride": None})
    for strides, fits in (((50, 1), True), ((64, 1), True), ((49, 1), False), ((1, 3), False), ((0, 1), False)):
        one_ = cuda_like()
        one_.stride = lambda i, strides=strides: strides[i]
        if fits:
            assert binding._rows_at(one_, "X") == (4096, strides[0])
        else:
            with pytest.raises(ValueError):
                binding._rows_at(one_, "X")


def test_scales_of_a_range_of_rows(lib):  # noqa: F811
    """A row of up to 128 elements has 4 bytes of scales: those of a range of rows begin at any multiple of 4."""
    far = [(1 << 40) + (i << 20) for i in range(6)]
    rc, need = _size(lib.xc_scores_microscaled_workspace, 100, 72)
    assert rc == 0
    for by in range(16):
        # (a workspace that is too small, and an empty list, are found behind the addresses: nothing is launched)
        scores = lib.xc_scores_microscaled(far[0], 100, 72, 1, far[1], far[2] + by, 1000, 0, far[3], far[4], need - 1, None)
        rows = lib.xc_microscale_rows(far[0], 10, 64, 1, far[1], 0, None, far[2], far[3] + by, None)
        assert (scores, rows) == ((EWORKSPACE, 0) if by % 4 == 0 else (EINVAL, EINVAL)), by
