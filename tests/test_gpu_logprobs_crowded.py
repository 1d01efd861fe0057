"""Top labels of rows in which more labels reach a threshold than a workgroup holds, in the first block of a row and in the stretches of several
blocks behind it: equal scores, steps, scores that grow along the row, masks of the type's lowest value.  Bounds: tests/test_gpu_logprobs.py."""
import numpy as np
import pytest
import torch

from oracle import answers_oracle as ao
from tests.test_gpu_logprobs import BF16, DEV, F32, U, _check, _close, _np, _sizes

pytestmark = pytest.mark.gpu


def _crowded(V, dtype):
    """Rows, each of them crowded in another way."""
    g = torch.Generator().manual_seed(V)
    low, at = torch.finfo(dtype).min, torch.arange(V)
    X = [torch.zeros(V),                                   # one value
         torch.where(at % 2 == 0, 0.0, -0.0),              # equal scores, of which some are -0
         torch.randint(0, 3, (V,), generator=g).float(),   # three values
         at * 0.01 - 3,                                    # growing
         torch.floor(at / 500) * 0.25,                     # growing by steps, each of which fills more than the list
         -torch.floor(at / 3000) * 0.25]                   # falling by steps
    late = 0.5 * torch.randn(V, generator=g)
    late[V // 3:] = 7.0                                    # equal scores behind the first blocks
    X.append(late)
    last = torch.ones(V)
    last[-5:] = 2.0                                        # the row's last elements are the best, the others equal
    X.append(last)
    few = torch.full((V,), low)
    few[100:103] = torch.tensor([1.0, 3.0, 2.0])
    few[V - 1] = 2.5                                       # a mask of the type's lowest value with a few labels left
    X.append(few)
    gone = torch.full((V,), -float("inf"))
    gone[V // 2::3] = 0.5                                  # labels that are not there, then equal ones
    X.append(gone)
    better = torch.zeros(V)
    better[V // 2:V // 2 + 60] = torch.linspace(1, 2, 60)  # equal scores, then some better ones, then more
    better[V - 300:V - 100] = torch.linspace(1.5, 3, 200)
    X.append(better)
    inf = torch.zeros(V)
    inf[1::2] = float("inf")                               # the largest there is
    X.append(inf)
    nan = torch.ones(V)
    nan[::7] = float("nan")                                # what is no number is never among the best
    X.append(nan)
    return torch.stack(X).to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [30011, 70003, 100005])
def test_segments_of_several_blocks(V, dtype):
    """Of 512 rows or more each is one workgroup's, which goes through it in several blocks."""
    import paper_2409_20156_amd as xc
    X = _crowded(V, dtype)
    n, times = X.shape[0], 41
    x = _np(X)
    labels = torch.tensor([[0, V - 1, V // 3]], dtype=torch.int32).repeat(n, 1)
    want = ao.label_logprobs(x, labels.numpy(), 1.0, 128)
    d, mean = _sizes(x, 1.0)
    d = np.where(np.isfinite(d), d, 0)
    tol = U * (60 + 3 * mean + np.abs(np.where(np.isfinite(want["norm"][:, 1]), want["norm"][:, 1], 0)))
    xd, ld = X.repeat(times, 1).to(DEV), labels.repeat(times, 1).to(DEV)
    assert xd.shape[0] >= 512
    for k in (1, 5, 37, 128):
        r = xc.label_logprobs(xd, ld, top=k)
        top = r["top"].cpu().numpy().reshape(times, n, k)
        for i in range(n):
            assert (top[:, i] == want["top"][i, :k]).all(), (i, k)
        far = np.take_along_axis(d, np.clip(want["top"][:, :k], 0, V - 1), 1)
        for t in range(times):
            _close(_np(r["top_logp"])[t * n:(t + 1) * n], want["top_logp"][:, :k], tol[:, None] + 5 * U * far)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [5000, 40003, 300007])
def test_segments_that_are_joined(V, dtype):
    X = _crowded(V, dtype)
    labels = torch.tensor([[0, V - 1, V // 3]], dtype=torch.int32).repeat(X.shape[0], 1)
    for k in (1, 20, 128):
        _check(X, labels, top=k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,V", [(13, 9000), (600, 30016)])
def test_a_row_does_not_depend_on_the_others(B, V, dtype):
    """The same row among others, and among rows of masks, infinities and what is no number."""
    import paper_2409_20156_amd as xc
    g = torch.Generator().manual_seed(B)
    X = (2.5 * torch.randn((B, V), generator=g)).to(dtype).to(DEV)
    labels = torch.randint(0, V, (B, 4), generator=g).to(torch.int32).to(DEV)
    Y = X.clone()
    keep = torch.arange(B, device=DEV) % 3 == 1
    for i, v in enumerate((float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).min, 0.0)):
        rows = torch.arange(B, device=DEV) % 10 == 2 * i
        Y[rows & ~keep] = v
    a, b = xc.label_logprobs(X, labels, top=30), xc.label_logprobs(Y, labels, top=30)
    for name in a:
        assert torch.equal(a[name][keep], b[name][keep]), name
    assert b["entropy"].isnan().any()
