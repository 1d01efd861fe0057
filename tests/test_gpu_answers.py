"""The operators on scores one after the other, as they are used: a teacher's classifier in 4 bits, its scores, their top labels and log
probabilities, the student's loss against them and its gradient; training on labels drawn from the scores; on other streams and in graphs."""
import numpy as np
import pytest
import torch

from oracle import answers_oracle as ao

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _inputs(seed, B, L, d, dtype=BF16):
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn((L, d), generator=g) * 3 * d ** -0.5).to(dtype)
    S = (W.float() + torch.randn((L, d), generator=g) * d ** -0.5).to(dtype)
    Z = torch.randn((B, d), generator=g).to(dtype)
    return W.to(DEV), S.to(DEV), Z.to(DEV)


class Chain:
    """Buffers of one chain, allocated once."""

    def __init__(self, B, L, d, k):
        import paper_2409_20156_amd as xc
        self.xc, self.k = xc, k
        pitch = xc.microscaled_pitch(d)
        self.rows = (torch.empty((L, pitch // 2), dtype=torch.uint8, device=DEV), torch.empty((L, pitch // 32), dtype=torch.uint8, device=DEV))
        self.scores = torch.empty((B, L), dtype=F32, device=DEV)
        self.student = torch.empty((B, L), dtype=BF16, device=DEV)
        self.ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in (
            xc.scores_microscaled_workspace(B, d), xc.label_logprobs_workspace(B, L, k, xc.XC_F32), xc.distill_workspace(B, L, xc.XC_BF16),
            xc.label_logprobs_workspace(B, L, 0, xc.XC_BF16))]
        f = dict(device=DEV, dtype=F32)
        self.out = {"logp": torch.empty((B, 1), **f), "entropy": torch.empty(B, **f), "norm": torch.empty((B, 2), **f),
                    "top": torch.empty((B, k), dtype=torch.int32, device=DEV), "top_logp": torch.empty((B, k), **f)}
        self.back = {"logp": torch.empty((B, k), **f), "entropy": torch.empty(B, **f), "norm": torch.empty((B, 2), **f)}
        self.loss, self.dX, self.dlogp = torch.empty(B, **f), torch.empty((B, L), dtype=BF16, device=DEV), torch.full((B, k), -0.1, **f)
        self.dX2, self.one = torch.empty((B, L), dtype=BF16, device=DEV), torch.zeros((B, 1), dtype=torch.int32, device=DEV)

    def run(self, W, S, Z):
        xc = self.xc
        xc.microscale_rows(W, out=self.rows)
        xc.scores_microscaled(Z, *self.rows, workspace=self.ws[0], out=self.scores)
        r = xc.label_logprobs(self.scores, self.one, top=self.k, workspace=self.ws[1], out=self.out)
        self.student.copy_(Z.float() @ S.float().t())
        xc.distill(self.student, r["top"], r["top_logp"], tail=True, workspace=self.ws[2], out=(self.loss, self.dX))
        b = xc.label_logprobs(self.student, r["top"], workspace=self.ws[3], out=self.back)
        xc.label_logprobs_grad(self.student, r["top"], self.dlogp, b["norm"], out=self.dX2)

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.scores, *self.out.values(), *self.back.values(), self.loss, self.dX, self.dX2)]


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("B,L,d,k", [(3, 500, 64, 5), (40, 9001, 136, 32)])
def test_a_student_learns_from_a_teacher_in_4_bits(B, L, d, k):
    W, S, Z = _inputs(B, B, L, d)
    c = Chain(B, L, d, k)
    c.run(W, S, Z)
    torch.cuda.synchronize()
    z, w = (ao.values(*ao.microscale_rows(t.double().cpu().numpy())) for t in (Z, W))
    scores = z @ w.T
    # (fp32 sums of 2 to 5 products of 128; the scores reach about 20)
    assert np.abs(c.scores.double().cpu().numpy() - scores).max() < 1e-4
    shown = c.scores.double().cpu().numpy()
    r = ao.label_logprobs(shown, np.zeros((B, 1), dtype=int), 1.0, k)
    assert (c.out["top"].cpu().numpy() == r["top"]).all()
    # (2^-24 (60 + 3 E|d| + |log S|) with E|d| and |log S| below 20 is 8e-6; the loss's and the gradients' sums are no further off)
    assert np.abs(c.out["top_logp"].cpu().numpy() - r["top_logp"]).max() < 2e-5
    student = c.student.double().cpu().numpy()
    loss, dX, _ = ao.distill(student, r["top"], c.out["top_logp"].double().cpu().numpy(), 1.0, True)
    assert np.abs(c.loss.cpu().numpy() - loss).max() < 2e-5
    assert np.abs(c.dX.double().cpu().numpy() - dX).max() < 2.0 ** -8
    back = ao.label_logprobs_grad(student, r["top"], np.full((B, k), float(np.float32(-0.1))), 1.0)
    assert np.abs(c.dX2.double().cpu().numpy() - back).max() < 2.0 ** -8 * np.abs(back).max() + 1e-6


def test_other_streams_give_the_same():
    W, S, Z = _inputs(1, 20, 4001, 128)
    a, b = Chain(20, 4001, 128, 16), Chain(20, 4001, 128, 16)
    a.run(W, S, Z)
    want = a.results()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        b.run(W, S, Z)
    a.run(W, S, Z)                                         # at the same time, on buffers of its own
    torch.cuda.synchronize()
    assert _same(a.results(), want) and _same(b.results(), want)


def test_captured_and_replayed():
    W, S, Z = _inputs(2, 24, 20003, 256)
    a, b = Chain(24, 20003, 256, 20), Chain(24, 20003, 256, 20)
    graphs = []
    for c in (a, b):
        c.run(W, S, Z)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run(W, S, Z)
        graphs.append(graph)
    eager = Chain(24, 20003, 256, 20)
    for turn in range(5):
        V, R, Y = _inputs(10 + turn, 24, 20003, 256)
        W.copy_(V), S.copy_(R), Z.copy_(Y)
        eager.run(W, S, Z)
        want = eager.results()
        for graph in graphs:
            graph.replay()
        for c in (a, b):
            assert _same(c.results(), want), turn
        (torch.randn((512, 512), device=DEV) @ torch.randn((512, 512), device=DEV)).sum().item()
        graphs[turn % 2].replay()                          # once more, and each by itself
        assert _same((a, b)[turn % 2].results(), want)


def test_a_search_teaches_the_student():
    """`mine_negatives` gives a teacher's top labels and logits as they are."""
    import paper_2409_20156_amd as xc
    W, S, Z = _inputs(5, 30, 3000, 64)
    ids, logits = xc.mine_negatives(Z, W, 16, want_scores=True)
    student = (Z.float() @ S.float().t()).contiguous()
    loss, dX = xc.distill(student, ids, logits)
    want, grad, _ = ao.distill(student.double().cpu().numpy(), ids.cpu().numpy(), logits.double().cpu().numpy())
    # (log S is off by u (60 + 3 E|d|), E|d| below 20; a gradient by 1e-5 of p at most)
    assert np.abs(loss.cpu().numpy() - want).max() < 1e-5 and np.abs(dX.cpu().numpy() - grad).max() < 1e-5


def test_nothing_is_allocated_with_buffers():
    W, S, Z = _inputs(3, 16, 5000, 128)
    c = Chain(16, 5000, 128, 8)
    xc = c.xc
    c.run(W, S, Z)
    torch.cuda.synchronize()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    xc.microscale_rows(W, out=c.rows)
    xc.scores_microscaled(Z, *c.rows, workspace=c.ws[0], out=c.scores)
    xc.label_logprobs(c.scores, c.one, top=8, workspace=c.ws[1], out=c.out)
    xc.distill(c.student, c.out["top"], c.out["top_logp"], tail=True, workspace=c.ws[2], out=(c.loss, c.dX))
    xc.label_logprobs_grad(c.student, c.out["top"], c.dlogp, c.back["norm"], out=c.dX2)
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before


def _equal_bits(a, b):
    assert torch.equal(a.view(torch.int32) if a.dtype == F32 else a, b.view(torch.int32) if b.dtype == F32 else b)


def _rows_by_themselves(X, lo, n, k, K):
    """What the calls on a soft-max give for the rows from lo on, in a call of their own: of 512 rows or more and
    from a multiple of 8 on, so that they are cut and lie alike."""
    import paper_2409_20156_amd as xc
    B, V = X.shape
    g = torch.Generator(device=DEV).manual_seed(5)
    labels = torch.randint(-1, V, (B, K), generator=g, dtype=torch.int32, device=DEV)
    teacher = torch.randn((B, K), generator=g, device=DEV)
    given, few = labels[:, :n].contiguous(), lambda t: t[lo:].clone()
    r, part = xc.label_logprobs(X, given, top=k), xc.label_logprobs(few(X), few(given), top=k)
    for name in r:
        if r[name] is not None:
            _equal_bits(few(r[name]), part[name])
    dlogp = torch.randn((B, n), generator=g, device=DEV)
    _equal_bits(few(xc.label_logprobs_grad(X, given, dlogp, r["norm"])), xc.label_logprobs_grad(few(X), few(given), few(dlogp), part["norm"]))
    del r, part, dlogp
    loss, dX = xc.distill(X, labels, teacher)
    want, dx = xc.distill(few(X), few(labels), few(teacher))
    _equal_bits(few(loss), want)
    _equal_bits(few(dX), dx)
    assert torch.isfinite(want).all()


@pytest.mark.parametrize("B,V,dtype,k", [(17000, 131072, BF16, 4), ((1 << 24) + 700, 8, F32, 3), ((1 << 21) + 704, 999, BF16, 0)])
def test_scores_beyond_32_bits_and_more_rows_than_a_launch_takes(B, V, dtype, k):
    _rows_by_themselves(torch.empty((B, V), dtype=dtype, device=DEV).normal_(), B - 600, 2, k, 6)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("B,L,d", [(800, 5600000, 768), (2200, 2000000, 1152), (2, 5600000, 1032)])
def test_4_bit_rows_and_scores_beyond_32_bits(B, L, d):
    import paper_2409_20156_amd as xc
    W = torch.empty((L, d), dtype=BF16, device=DEV).normal_()
    Z = torch.empty((B, d), dtype=BF16, device=DEV).normal_()
    Q, s = xc.microscale_rows(W)
    Q1, s1 = xc.microscale_rows(W[-2000:].clone())
    _equal_bits(Q[-2000:], Q1)
    _equal_bits(s[-2000:], s1)
    del W
    out = xc.scores_microscaled(Z, Q, s, dtype=BF16)
    lo = max(B - 20, 0)
    _equal_bits(out[:, -2000:].contiguous(), xc.scores_microscaled(Z, Q1, s1, dtype=BF16))
    _equal_bits(out[lo:], xc.scores_microscaled(Z[lo:].clone(), Q, s, dtype=BF16))
    del out
    torch.cuda.empty_cache()


def test_which_kernels_a_call_launches():
    """By the names of the event timing: one launch where a workgroup holds a row or brings the queries to 4 bits itself, more of them elsewhere."""
    import paper_2409_20156_amd as xc
    from paper_2409_20156_amd import binding

    def kernels(call):
        call()                                             # (outputs and workspaces that torch allocates)
        torch.cuda.synchronize()
        binding.profile_reset()
        binding.profile_enable(True)
        try:
            call()
        finally:
            binding.profile_enable(False)
        prof = binding.profile_collect()
        binding.profile_reset()
        return {name: n for name, (_, n) in prof.items() if n}

    X = {(B, V): torch.randn((B, V), device=DEV).to(BF16) for B, V in ((2, 4096), (16, 131072), (300, 32000), (70, 131072))}
    labels = {key: torch.zeros((key[0], 3), dtype=torch.int32, device=DEV) for key in X}
    teacher = {key: torch.zeros((key[0], 3), device=DEV) for key in X}
    for key, want in (((2, 4096), {"logprobs": 1}), ((16, 131072), {"logprobs": 1, "logprobs_join": 1}), ((300, 32000), {"logprobs": 1, "logprobs_join": 1})):
        assert kernels(lambda: xc.label_logprobs(X[key], labels[key], top=2)) == want, key
    norm = xc.label_logprobs(X[2, 4096], labels[2, 4096])["norm"]
    assert kernels(lambda: xc.label_logprobs_grad(X[2, 4096], labels[2, 4096], teacher[2, 4096], norm)) == {"logprobs_grad": 1}
    split = {"distill_sums": 1, "distill_terms": 1, "distill_grad": 1}
    for key, grad, place, want in (((2, 4096), True, False, {"distill_grad": 1}), ((300, 32000), True, True, {"distill_grad": 1}),
                                   ((16, 131072), True, False, {"distill_sums": 1, "distill_grad": 1}), ((16, 131072), True, True, split),
                                   ((70, 131072), True, False, split), ((2, 4096), False, False, {"distill_sums": 1, "distill_terms": 1})):
        x, out = X[key], None
        if place:
            x = x.clone()
            out = (torch.empty(key[0], device=DEV), x)
        assert kernels(lambda: xc.distill(x, labels[key], teacher[key], grad=grad, out=out)) == want, (key, grad, place)
    for B, L, d, n in ((1, 100, 64, 1), (16, 100, 1024, 1), (17, 100, 64, 2), (4, 100, 4096, 1), (5, 100, 4096, 2), (2, 100, 4104, 2), (300, 2000, 768, 2)):
        W, Z = torch.randn((L, d), device=DEV), torch.randn((B, d), device=DEV)
        Q, s = xc.microscale_rows(W)
        assert kernels(lambda: xc.scores_microscaled(Z, Q, s)) == ({"scores_micro": 1} if n == 1 else {"microscale": 1, "scores_micro": 1}), (B, L, d)
        assert kernels(lambda: xc.microscale_rows(W)) == {"microscale": 1}
