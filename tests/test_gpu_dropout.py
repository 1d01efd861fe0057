"""Dropout and its gradient against the oracle: the same elements dropped, the others within two roundings (scale and
product, 2 * 2^-24 relative; bf16 results 2^-8 more)."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _check(X, Y, rate, seed, row0=0):
    keep = so.dropout_kept(X.shape[0], X.shape[1], rate, seed, row0)
    want = np.where(keep, X.double().numpy() * (65536 / (65536 - so.dropout_least(rate))), 0.0)
    got = Y.cpu().double().numpy()
    assert (got[~keep] == 0).all()
    bound = np.abs(want) * (2.01 * 2.0 ** -24 + (2.0 ** -8 if Y.dtype == BF16 else 0))
    assert (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("t,out_t", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("B,d", [(1, 1), (1, 3), (2, 4), (3, 5), (7, 7), (5, 8), (300, 1), (9, 12), (33, 16), (17, 63), (4, 64), (65, 72),
                                 (3, 255), (8, 768), (10, 1001), (2, 4096), (2, 8193), (1, 30000)])
def test_matches_the_oracle(t, out_t, B, d):
    import paper_2409_20156_amd as xc
    seed = 0x9876543210ABCDEF + B * 1000 + d
    X = torch.tensor(np.random.default_rng(d).normal(size=(B, d)), dtype=F32).to(t)
    flat = torch.full((B * d + 128,), 77.0, dtype=out_t, device=DEV)
    Y = flat[64:B * d + 64].view(B, d)
    rate = (0.0, 0.1, 0.5, 0.93)[(B + d) % 4]
    got = xc.dropout(X.to(DEV), rate, seed, out=Y)
    torch.cuda.synchronize()
    assert got is Y and (flat[:64] == 77).all() and (flat[B * d + 64:] == 77).all()
    _check(X, Y, rate, seed)
    grad = xc.dropout_grad(X.to(DEV), rate, seed, dtype=out_t)
    assert grad.dtype == out_t and torch.equal(grad, Y)


@pytest.mark.parametrize("rate", [0.0, 1e-6, 1.0 / 65536, 0.3, 0.99999])
def test_rates_at_the_ends(rate):
    import paper_2409_20156_amd as xc
    X = torch.randn((64, 128))
    Y = xc.dropout(X.to(DEV), rate, 5)
    _check(X, Y, rate, 5)
    if so.dropout_least(rate) == 0:
        assert torch.equal(Y.cpu(), X)


def test_dropped_elements_are_zero_whatever_they_held():
    import paper_2409_20156_amd as xc
    X = torch.full((8, 100), float("nan"))
    X[::2] = float("inf")
    X[1::4] = 3.4e38
    Y = xc.dropout(X.to(DEV), 0.5, 11).cpu()
    keep = torch.tensor(so.dropout_kept(8, 100, 0.5, 11))
    assert (Y[~keep] == 0).all()
    assert (Y[::2][keep[::2]] == float("inf")).all() and (Y[1::4][keep[1::4]] == float("inf")).all() and Y[3::4][keep[3::4]].isnan().all()


def test_rows_of_a_shard_and_large_row_numbers():
    import paper_2409_20156_amd as xc
    X = torch.randn((40, 72), device=DEV).to(BF16)
    every = xc.dropout(X, 0.2, 3)
    assert torch.equal(xc.dropout(X[16:].contiguous(), 0.2, 3, row0=16), every[16:])
    far = xc.dropout(X, 0.2, 3, row0=(1 << 40) + 5)
    _check(X.cpu(), far, 0.2, 3, (1 << 40) + 5)
    assert not torch.equal(far, every)


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("d", [64, 71])
def test_in_place(t, d):
    import paper_2409_20156_amd as xc
    X = torch.randn((333, d), device=DEV).to(t)
    want = xc.dropout(X, 0.3, 8)
    assert xc.dropout(X, 0.3, 8, out=X) is X and torch.equal(X, want)


def test_negative_seeds_count_modulo_two_to_the_64():
    import paper_2409_20156_amd as xc
    X = torch.randn((5, 40), device=DEV)
    assert torch.equal(xc.dropout(X, 0.4, -3), xc.dropout(X, 0.4, (1 << 64) - 3))


def test_gradient_is_that_of_differences():
    """sum(dY * dropout(X)) is linear in X, so a difference quotient has rounding errors alone."""
    import paper_2409_20156_amd as xc
    B, d = 6, 33
    g = torch.Generator().manual_seed(4)
    X, dY, V = (torch.randn((B, d), generator=g).to(DEV) for _ in range(3))
    grad = xc.dropout_grad(dY, 0.3, 21).double()
    f = lambda x: (dY.double() * xc.dropout(x, 0.3, 21).double()).sum()  # noqa: E731
    h = 2.0 ** -3
    got = (f(X + h * V) - f(X - h * V)) / (2 * h)
    want = (grad * V.double()).sum()
    # X +- h V, the product and the gradient are rounded to 24 bits: three roundings of terms no larger than these
    bound = 3.01 * 2.0 ** -24 / h * (dY.abs().double() * (X.abs() + h * V.abs()).double()).sum() * 65536 / (65536 - so.dropout_least(0.3))
    assert abs(got - want) <= bound


def test_offsets_beyond_32_bits():
    import paper_2409_20156_amd as xc
    B, d = 2_200_000, 1000                                 # 2.2e9 elements
    X = torch.ones((B, d), dtype=BF16, device=DEV)
    xc.dropout(X, 0.5, 17, out=X)
    for r in (0, 1, 2_147_483, 2_147_484, B - 1):
        assert (X[r].float().cpu().numpy() == 2.0 * so.dropout_kept(1, d, 0.5, 17, row0=r)[0]).all()


def test_more_rows_than_one_launch_takes():
    import paper_2409_20156_amd as xc
    B = (1 << 31) + 300                                    # of one element
    X = torch.ones((B, 1), dtype=BF16, device=DEV)
    xc.dropout(X, 0.5, 19, row0=7, out=X)
    for r in (0, (1 << 31) - 150, (1 << 31), B - 100):
        n = min(B - r, 200)
        want = xc.dropout(torch.ones((n, 1), dtype=BF16, device=DEV), 0.5, 19, row0=7 + r)
        assert torch.equal(X[r:r + n], want)
        assert (want.cpu().float().numpy() == 2.0 * so.dropout_kept(n, 1, 0.5, 19, row0=7 + r)).all()


def test_another_stream_and_a_replayed_graph():
    import paper_2409_20156_amd as xc
    X = torch.randn((100, 768), device=DEV).to(BF16)
    want = xc.dropout(X, 0.1, 2)
    out = torch.zeros_like(X)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        xc.dropout(X, 0.1, 2, out=out)
    side.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        xc.dropout(X, 0.1, 2, out=out)
    for k in range(3):
        X.copy_(torch.randn((100, 768)))
        want = xc.dropout(X, 0.1, 2)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_an_encoder_gets_its_gradient_by_hand():
    """No call records anything for autograd; the gradient of a loss that is linear in the dropped embeddings, put into the encoder by
    hand, is what autograd gives through a mask written out.  Entries are small integers and the kept are doubled: sums are exact."""
    import paper_2409_20156_amd as xc
    g = torch.Generator().manual_seed(6)
    x, A, C = (torch.randint(-8, 9, s, generator=g).float() for s in ((12, 20), (20, 24), (12, 24)))
    keep = torch.tensor(so.dropout_kept(12, 24, 0.5, 9))
    ref = A.clone().requires_grad_()
    (C * ((x @ ref) * 2.0 * keep)).sum().backward()
    enc = A.to(DEV).requires_grad_()
    Z = x.to(DEV) @ enc
    Zd = xc.dropout(Z, 0.5, 9)
    assert Z.requires_grad and not Zd.requires_grad and Zd.grad_fn is None
    assert torch.equal(Zd.cpu(), (x @ A) * 2.0 * keep)
    Z.backward(xc.dropout_grad(C.to(DEV), 0.5, 9))
    assert torch.equal(enc.grad.cpu(), ref.grad)
