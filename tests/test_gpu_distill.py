"""The loss against a teacher's top labels and its gradient, against the oracle.

Bounds (u = 2^-24).  A sum over a row is off by D = u (60 + 3 E|d|) relative (see the log probabilities' tests); what is formed from it
is formed in 64 bits.  The loss: without a tail, its derivative by log S is Q = 1, so w T^2 D; with one, the others' sum S_r enters it by
p_r - q_r times its error, in second order by as much again, and the result is rounded: u of it.  (1e-6 D for what 64 bits lose.)  The
gradient, other labels: (Q p_r - q_r) r with r off by u (20 + 8 |log r|) + D relative and p_r by p_r (1 - p_r) D; listed ones: p off
by u (20 + 8 |log p|) + D, q by u (20 + 6 |log q|).  A result in bf16 is rounded once more: 2^-8 of it."""
import numpy as np
import pytest
import torch

from oracle import answers_oracle as ao
from tests.test_gpu_logprobs import BF16, DEV, F32, U, _close, _np, _sizes

pytestmark = pytest.mark.gpu


def _case(seed, B, V, K, dtype, tail, masked=0.0, padded=False):
    g = torch.Generator().manual_seed(seed)
    X = 2.5 * torch.randn((B, V), generator=g)
    X[torch.rand((B, V), generator=g) < masked] = -float("inf")
    t = (X + torch.randn((B, V), generator=g)).log_softmax(-1)
    k = min(K, V)
    top = t.topk(k, dim=-1)
    labels = torch.full((B, K), -1, dtype=torch.int32)
    teacher = torch.zeros((B, K))
    labels[:, :k], teacher[:, :k] = top.indices.to(torch.int32), top.values
    if not tail:
        teacher += 3.0                                     # logits need not be normalised
    if padded:
        labels[torch.rand((B, K), generator=g) < 0.3] = -1
    weight = torch.rand(B, generator=g) + 0.1
    weight[::5] = 0.0
    return X.to(dtype), labels, teacher, weight


def _check(X, labels, teacher, weight, T=1.0, tail=False, out=None, given=None, target=None):
    import paper_2409_20156_amd as xc
    out = out or X.dtype
    B, V = X.shape
    xd = X.to(DEV) if given is None else given
    w = weight.to(DEV) if weight is not None else None
    alone, none = xc.distill(xd, labels.to(DEV), teacher.to(DEV), temperature=T, tail=tail, weight=w, grad=False)
    assert none is None
    buf = None if target is None else (torch.empty(B, device=DEV), target)
    loss, dX = xc.distill(xd, labels.to(DEV), teacher.to(DEV), temperature=T, tail=tail, weight=w, dtype=out, out=buf)
    torch.cuda.synchronize()
    x = _np(X)
    w64 = weight.double().numpy() if weight is not None else None
    want, grad, parts = ao.distill(x, labels.numpy(), teacher.double().numpy(), T, tail, w64)
    size = np.abs(w64) if w64 is not None else np.ones(B)
    _, mean = _sizes(x, T)
    D = U * (60 + 3 * mean)
    first = np.abs(parts["p_r"] - parts["q_r"]) if tail else parts["mass"]
    tol = size * T * T * (D * first + D * D + 1e-6 * D) + U * np.abs(want)
    _close(_np(loss), want, np.where(np.isfinite(tol), tol, 0))
    _close(_np(alone), want, np.where(np.isfinite(tol), tol, 0))
    lp = np.where(np.isfinite(parts["logp"]), np.abs(parts["logp"]), 0)
    p, q, mass = np.exp(parts["logp"]), parts["q"], parts["mass"][:, None]
    p_r, q_r = parts["p_r"][:, None], parts["q_r"][:, None]
    d = D[:, None]
    with np.errstate(divide="ignore", invalid="ignore"):
        lq = np.where(q > 0, np.abs(np.log(np.where(q > 0, q, 1))), 0)
        if tail:
            r = np.where(p_r > 0, p / p_r, 0)
            lr = np.where(p_r > 0, lp + np.abs(np.log(np.where(p_r > 0, p_r, 1))), 0)
            other = np.abs(mass * p_r - q_r) * r * (U * (20 + 8 * lr) + d) + mass * p_r * (1 - p_r) * d * r
        else:
            other = p * (U * (20 + 8 * lp) + d)
    tol = np.where(parts["listed"], mass * p * (U * (20 + 8 * lp) + d) + q * U * (20 + 6 * lq), other)
    tol = (size * T)[:, None] * tol + (2.0 ** -8 if out == BF16 else 2 * U) * np.abs(grad) + 1e-35
    _close(_np(dX), grad, np.where(np.isfinite(tol), tol, 0))
    return loss, dX


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("B,V,K", [(1, 1, 1), (2, 2, 1), (3, 5, 5), (4, 8, 3), (5, 9, 2), (3, 17, 256), (33, 100, 7), (2, 4096, 16), (7, 4103, 64), (9, 8193, 33), (2, 50021, 128),
                                   (1, 131072, 64), (600, 777, 4), (5, 3000, 256), (1, 300007, 20), (260, 16387, 8), (520, 9001, 12),
                                   (70, 40001, 20), (66, 70001, 33), (75, 40001, 20), (73, 70001, 33), (300, 8200, 5)])
def test_matches_the_oracle(B, V, K, dtype, out, tail):
    _check(*_case(B + V + K, B, V, K, dtype, tail), tail=tail, out=out)


@pytest.mark.parametrize("dtype,V", [(F32, 41000), (BF16, 82003)])
def test_listed_labels_at_the_same_places_of_every_block(dtype, V):
    """Rows that workgroups go through in blocks of 1024 pieces of 16 bytes: listed labels lie in the same pieces of every block, whose marks
    share their memory.  Equal rows that begin at the same place of a piece (every 8th one does) have equal results, bit for bit,
    whichever workgroups had them."""
    import paper_2409_20156_amd as xc
    B, rows, K = 520, 4, 120
    n = 1024 * (4 if dtype == F32 else 8)
    X, _, _, _ = _case(3, rows, V, 1, dtype, True)
    places = torch.tensor([5, 6, 700, 2051, 2052, 2053, 3300, n - 9, n - 8, n - 1])
    labels = torch.cat([places + i * n for i in range(V // n + 1)])
    labels = labels[labels < V][:K].to(torch.int32)[None].repeat(rows, 1)
    X.scatter_(1, labels.long(), 6.0)                      # they have most of the probability: one that is missed shows
    teacher = X.double().log_softmax(-1).gather(1, labels.long()).float() - 0.4
    many = lambda t: t.repeat(B // rows, 1).contiguous().to(DEV)
    loss, none = xc.distill(many(X), many(labels), many(teacher), tail=True, grad=False)
    got = _np(loss).reshape(-1, 8)
    assert none is None and (got == got[0]).all()
    want, _, parts = ao.distill(_np(X), labels.numpy(), teacher.double().numpy(), 1.0, True, None)
    _, mean = _sizes(_np(X), 1.0)
    D = U * (60 + 3 * mean)
    first = np.abs(parts["p_r"] - parts["q_r"])
    tol = D * first + D * D + 1e-6 * D + U * np.abs(want)
    _close(got[0], np.tile(want, 2), np.tile(tol, 2))


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T", [0.3, 2.0, 8.0])
def test_temperatures_masks_and_padding(T, tail):
    for dtype in (F32, BF16):
        X, labels, teacher, weight = _case(17, 30, 2003, 20, dtype, tail, masked=0.4, padded=True)
        _check(X, labels, teacher, weight, T=T, tail=tail)
        _check(X, labels, teacher, None, T=T, tail=tail)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [6, 777, 9001])
def test_edges(V, dtype, tail):
    X, labels, teacher, weight = _case(V, 20, V, 5, dtype, tail, masked=0.2)
    inf = float("inf")
    weight[:] = 1.0
    X[0] = -inf                                            # nothing is left, and the row counts for nothing
    weight[0] = 0.0
    X[1] = -inf                                            # ... and it does count
    X[2] = torch.finfo(dtype).min
    X[3, labels[3, 0]] = -inf                              # the student rules out what the teacher expects
    labels[4] = -1                                         # no teacher
    labels[5] = labels[5, 0]                               # one label at every place
    teacher[5] = float(np.log(0.1))
    labels[6, 1], labels[6, 2] = V, -7
    teacher[7] = -inf
    teacher[8, 1:] = -inf
    X[9, V // 2] = float("nan")
    X[10, V // 2] = float("nan")
    weight[10] = 0.0
    weight[11] = -2.0
    X[12] = -inf                                           # no label but the listed ones
    X[12, labels[12].long()] = torch.arange(5).to(dtype)
    X[13] = -30.0
    X[13, labels[13].long()] = 40.0                        # hardly any weight on the others
    X[14, labels[14].long()] = -40.0                       # hardly any on the listed ones
    teacher[15] = float(np.log(0.2))                       # nothing left for the others
    teacher[16] = float(np.log(0.25))                      # more than all
    loss, dX = _check(X, labels, teacher, weight, tail=tail)
    assert (loss[[0, 4, 10]] == 0).all() and (dX[[0, 4, 10]] == 0).all()


@pytest.mark.parametrize("tail", [False, True])
def test_teacher_values_that_are_no_numbers(tail):
    X, labels, teacher, weight = _case(4, 6, 300, 5, F32, tail)
    weight[:] = 1.0
    teacher[2, 3] = float("nan")
    import paper_2409_20156_amd as xc
    loss, dX = xc.distill(X.to(DEV), labels.to(DEV), teacher.to(DEV), tail=tail, weight=weight.to(DEV))
    assert loss.isnan().nonzero().flatten().tolist() == [2] and dX[2].isnan().any() and not dX[[0, 1, 3, 4, 5]].isnan().any()


@pytest.mark.parametrize("tail", [False, True])
def test_gradient_against_differences(tail):
    import paper_2409_20156_amd as xc
    X, labels, teacher, _ = _case(11, 3, 40, 6, F32, tail)
    _, dX = xc.distill(X.to(DEV), labels.to(DEV), teacher.to(DEV), tail=tail, temperature=1.5)
    h = 2.0 ** -6
    for v in [0, 11, 39] + labels[:, 0].tolist():
        f = []
        for sign in (1, -1):
            Y = X.clone()
            Y[:, v] += sign * h
            f.append(_np(xc.distill(Y.to(DEV), labels.to(DEV), teacher.to(DEV), tail=tail, temperature=1.5, grad=False)[0]))
        assert np.abs((f[0] - f[1]) / (2 * h) - _np(dX)[:, v]).max() < 2e-3


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,V,ld", [(7, 64, 64), (7, 1001, 1001), (7, 1001, 1005), (4, 9001, 9009), (300, 3001, 3001)])
def test_in_place_and_rows_further_apart(B, V, ld, dtype, tail):
    X, labels, teacher, weight = _case(V, B, V, 9, dtype, tail)
    _, want = _check(X, labels, teacher, weight, tail=tail)
    buf = torch.full((B, ld), 9.0, dtype=dtype, device=DEV)
    buf[:, :V] = X.to(DEV)
    _, got = _check(X, labels, teacher, weight, tail=tail, given=buf[:, :V], target=buf[:, :V])
    assert torch.equal(got, want) and (buf[:, V:] == 9).all()
    wide = torch.full((B + 2, ld + 3), 9.0, dtype=F32, device=DEV)
    _check(X, labels, teacher, weight, tail=tail, out=F32, target=wide[:B, :V])
    assert (wide[:, V:] == 9).all() and (wide[B:] == 9).all()


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,V,K", [(6, 50, 5), (4, 4096, 256), (300, 9001, 70), (5, 70001, 130), (70, 131072, 66), (80, 40003, 64)])
def test_labels_listed_several_times(B, V, K, dtype, tail):
    """A label's probability is the sum over its places, in the loss as well as in the gradient: rows that a workgroup holds, rows in two
    launches, in three (in place), the loss alone; repeats next to each other and 64 places and more apart."""
    g = torch.Generator().manual_seed(B + K)
    X = (2.5 * torch.randn((B, V), generator=g)).to(dtype)
    pool = torch.randperm(V, generator=g)[: max(2, K // 3)]
    labels = pool[torch.randint(0, len(pool), (B, K), generator=g)].to(torch.int32)
    labels[0] = labels[0, 0]
    labels[1, ::2] = labels[1, 0]
    labels[2, -1] = labels[2, 0]
    labels[3, torch.rand(K, generator=g) < 0.4] = -1
    share = torch.rand((B, K), generator=g) + 0.01
    teacher = (0.9 * share / share.sum(1, keepdim=True)).log()           # a tenth is left for the others
    if not tail:
        teacher += 2.0
    weight = torch.rand(B, generator=g) + 0.1
    _check(X, labels, teacher, weight, tail=tail)
    place = X.to(DEV)
    _check(X, labels, teacher, weight, tail=tail, given=place, target=place)


def test_a_label_that_is_listed_twice_and_has_all_of_both_distributions():
    import paper_2409_20156_amd as xc
    X = torch.full((1, 50), -80.0, device=DEV)
    X[0, 3] = 20.0
    loss, dX = xc.distill(X, torch.tensor([[3, 3]], dtype=torch.int32, device=DEV), torch.zeros((1, 2), device=DEV))
    # (log S is off by 60 u: all of the sum is one exponential)
    assert abs(loss.item()) <= 60 * U and dX.abs().max().item() <= 40 * U
