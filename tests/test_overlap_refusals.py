"""Arrays that a call writes may overlap neither each other nor what it reads: refused by the C entry points before anything touches
a device (no GPU needed).  Arrays are laid out one behind the other at made-up addresses, and one of them is moved over another."""
import ctypes

import pytest

EINVAL = -1
BASE = 1 << 40


@pytest.fixture(scope="module")
def lib():
    from paper_2409_20156_amd import binding
    return binding.load_library()


def _need(fn, *args):
    n = ctypes.c_size_t(0)
    assert fn(*args, ctypes.byref(n)) == 0
    return n.value


def _layout(sizes):
    at, out = BASE, {}
    for name, size in sizes.items():
        out[name] = at
        at += (size + 15) // 16 * 16
    return out


def _overlaps(sizes, written):
    """Every way to lay one written array over another array: its first bytes on the other's last and the reverse."""
    for w in written:
        for o in sizes:
            if o == w or sizes[o] == 0:
                continue
            base = _layout(sizes)
            yield w, o, {**base, w: base[o]}
            if sizes[o] > 16:
                yield w, o, {**base, w: base[o] + (sizes[o] - 1) // 16 * 16}
            if sizes[w] > 16:
                yield w, o, {**base, w: base[o] - (sizes[w] - 1) // 16 * 16}


@pytest.mark.parametrize("t", [0, 1])
@pytest.mark.parametrize("B,n,V,with_draft", [(7, 3, 50021, True), (2, 5, 9, True), (4, 2, 300, False), (1, 0, 100, False)])
def test_verify(lib, t, B, n, V, with_draft):
    e = 2 if t else 4
    need = _need(lib.xc_verify_workspace, B, V)
    sizes = {"tokens": B * (n + 1) * 4, "accepted": B * 4, "ws": need, "drafts": B * n * 4, "u": B * (n + 1) * 4,
             "target": B * (n + 1) * V * e, "draft": B * n * V * e if with_draft else 0}
    for w, o, at in _overlaps(sizes, ("tokens", "accepted", "ws")):
        rc = lib.xc_verify_drafts(at["drafts"] if n else None, B, n, V, at["target"], at["draft"] if with_draft else None, t, at["u"],
                                  at["tokens"], at["accepted"], at["ws"], need, None)
        assert rc == EINVAL, (w, o)


@pytest.mark.parametrize("t,N,d", [(0, 100, 60), (1, 100, 72), (1, 1, 8), (1, 5, 20000)])
@pytest.mark.parametrize("m,counted", [(0, False), (7, False), (50, True)])
def test_quantize_rows(lib, t, N, d, m, counted):
    pitch = (d + 15) // 16 * 16
    sizes = {"Q": N * pitch, "scale": N * 4, "X": N * d * (2 if t else 4), "ids": m * 4, "count": 4 if counted else 0}
    for w, o, at in _overlaps(sizes, ("Q", "scale")):
        rc = lib.xc_quantize_rows(at["X"], N, d, t, at["ids"] if m else None, m, at["count"] if counted else None, at["Q"], at["scale"], None)
        assert rc == EINVAL, (w, o)


@pytest.mark.parametrize("t,out_t", [(0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("B,d,L", [(3, 72, 1000), (40, 72, 1000), (300, 4096, 7), (1, 8, 1)])
def test_scores(lib, t, out_t, B, d, L):
    need = _need(lib.xc_scores_workspace, B, d)
    sizes = {"out": B * L * (2 if out_t else 4), "ws": need, "Z": B * d * (2 if t else 4), "Q": L * ((d + 15) // 16 * 16), "scale": L * 4}
    for w, o, at in _overlaps(sizes, ("out", "ws")):
        rc = lib.xc_scores_quantized(at["Z"], B, d, t, at["Q"], at["scale"], L, out_t, at["out"], at["ws"], need, None)
        assert rc == EINVAL, (w, o)
