"""Drafted labels checked against the classifier's probabilities: labels and counts equal to the oracle's.

Sums are held in 64 bits on both sides; a label could differ only where a random number times the sum comes within about
2^-45 of a running sum, which the random inputs here do not (and where sums are exact in 64 bits there is nothing to differ)."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _case(seed, B, n, V, dtype, looked_up=False, noise=0.6, sigma=2.5):
    g = torch.Generator().manual_seed(seed)
    logits = sigma * torch.randn((B, n + 1, V), generator=g)
    drafted = logits[:, :n] + noise * torch.randn((B, n, V), generator=g)
    x = (drafted - torch.empty_like(drafted).exponential_(generator=g).log()).argmax(-1).to(torch.int32).reshape(B, n)
    if looked_up and n:
        hit = torch.rand((B, n, 1), generator=g) < 0.7     # the target expects these too
        at = x[:, :, None].long()
        sure = logits[:, :n].logsumexp(-1, keepdim=True) + 2.0
        logits[:, :n].scatter_(2, at, torch.where(hit, sure, logits[:, :n].gather(2, at)))
    u = torch.rand((B, n + 1), generator=g)
    return x, logits.softmax(-1).to(dtype), None if looked_up else drafted.softmax(-1).to(dtype), u


def _run(x, p, q, u, **kw):
    import paper_2409_20156_amd as xc
    tokens, accepted = xc.verify_drafts(x.to(DEV), p.to(DEV), q.to(DEV) if q is not None else None, u.to(DEV), **kw)
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), accepted.cpu().numpy()


def _check(x, p, q, u):
    got = _run(x, p, q, u)
    want = so.verify_drafts(x.numpy(), p.double().numpy(), q.double().numpy() if q is not None else None, u.double().numpy())
    assert (got[1] == want[1]).all() and (got[0] == want[0]).all()
    return got


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,n,V", [(1, 0, 1), (1, 1, 1), (3, 2, 2), (5, 3, 7), (2, 4, 8), (4, 1, 9), (9, 5, 63), (8, 3, 511), (7, 2, 512),
                                   (6, 4, 513), (5, 3, 4095), (5, 3, 4096), (5, 3, 4097), (16, 4, 1000), (3, 8, 8192), (2, 2, 50021),
                                   (64, 3, 3001), (300, 2, 777), (2, 63, 300), (2, 64, 301), (2, 65, 303), (1, 200, 100), (1, 3, 131072),
                                   (2, 1, 262144 + 5), (3, 2, 32768), (2, 2, 32769), (192, 1, 40001), (191, 1, 40001), (1, 1, 600011)])
@pytest.mark.parametrize("looked_up", [False, True])
def test_matches_the_oracle(B, n, V, dtype, looked_up):
    noise = 0.02 if n >= 60 else 0.6
    _check(*_case(B * 1009 + n * 31 + V, B, n, V, dtype, looked_up, noise))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_all_stand_all_fall_and_lists_that_end_early(dtype):
    B, n, V = 12, 6, 900
    x, p, q, u = _case(5, B, n, V, dtype)
    u[:3, :n] = 0.0                                        # all stand (u q = 0 < p)
    u[3:6, :n] = 0.99999994
    q[3:6] = 1.0                                           # all fall at the first
    x[6, 2], x[7, 0], x[8, 5], x[9, 3] = -1, V, -7, 2 ** 31 - 1
    u[6:10, :n] = 0.0
    got = _check(x, p, q, u)
    assert got[1][:3].tolist() == [n] * 3 and got[1][3:6].tolist() == [0] * 3 and got[1][6:10].tolist() == [2, 0, 5, 3]
    assert (got[0][6, 3:] == -1).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [5, 640, 5000, 20000, 70001])
def test_rows_with_zeros_infinities_and_nan(dtype, V):
    rng = np.random.default_rng(V)
    B, n = 40, 2
    x, p, q, u = _case(V, B, n, V, dtype)
    for b in range(B):
        bad = torch.tensor(rng.integers(0, V, size=max(1, V // 3)))
        if b % 5 == 0:
            p[b, :, bad] = 0
        elif b % 5 == 1:
            p[b, :, bad] = float("nan")
        elif b % 5 == 2:
            p[b, :, bad] = float("inf")
            q[b, :, bad[: len(bad) // 2]] = float("nan")
        elif b % 5 == 3:
            q[b, :, bad] = float("inf")
            p[b, :, bad] = -float("inf")
        elif b == 4:
            p[b] = 0                                       # nothing anywhere
        elif b == 9:
            q[b] = p[b, :n]
            q[b, 0, int(x[b, 0])] = 2.0                    # the first falls, and nothing of the target lies above the draft
            u[b, 0] = 0.999
        elif b == 14:
            p[b, 0] = 0
            p[b, 0, V - 1] = 1e-30                         # one small weight at the very end
            x[b, 0] = 0
        elif b == 19:
            p[b] = float("nan")
    _check(x, p, q, u)


@pytest.mark.parametrize("V", [9, 4096, 4100, 12288, 30000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_edges_between_weights_go_to_the_next_label(V, dtype):
    """Weights are multiples of 2^-20 and few, sums are exact: u * total meets a running sum exactly in many rows."""
    B = 64
    rng = np.random.default_rng(V)
    w = np.zeros((B, V))
    u = np.zeros((B, 1), dtype=np.float32)
    for b in range(B):
        at = rng.choice(V, size=min(V, 8), replace=False)
        w[b, at] = rng.integers(0, 4, size=at.size) * 2.0 ** -5
        w[b, at[0]] += 2.0 ** -5
        total = w[b].sum() * 32
        pick = [k for k in range(int(total)) if np.float32(k / total) * np.float64(total) == k] or [0]
        u[b, 0] = pick[b % len(pick)] / total
    u[-4:, 0] = [0.0, 0.99999994, 1.0, -1.0]               # (the last two are no numbers of [0, 1): still a label with a weight)
    _check(torch.zeros((B, 0), dtype=torch.int32), torch.tensor(w, dtype=dtype)[:, None], None, torch.tensor(u))


def test_a_random_number_that_is_none_gives_the_last_label_with_a_weight():
    p = torch.zeros((1, 1, 9000))
    p[0, 0, [5, 4500, 8000]] = 0.25
    got = _run(torch.zeros((1, 0), dtype=torch.int32), p, None, torch.tensor([[float("nan")]]))
    assert got[0].tolist() == [[8000]]


@pytest.mark.parametrize("B,V", [(400, 9001), (200, 20011), (200, 70001)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_sequence_does_not_depend_on_the_others(dtype, B, V):
    x, p, q, u = _case(77, B, 2, V, dtype)
    every = _run(x, p, q, u)
    for b in (0, 17, B - 1):
        one = _run(x[b:b + 1].clone(), p[b:b + 1].clone(), q[b:b + 1].clone(), u[b:b + 1].clone())
        assert (one[0][0] == every[0][b]).all() and one[1][0] == every[1][b]


@pytest.mark.parametrize("B,n,V", [(131071, 1, 3), (65536, 2, 8), (66000, 1, 17000)])
def test_more_sequences_than_one_launch_takes(B, n, V):
    import paper_2409_20156_amd as xc
    g = torch.Generator(device=DEV).manual_seed(B)
    p = torch.rand((B, n + 1, V), generator=g, device=DEV, dtype=F32).to(BF16)
    x = torch.randint(0, V, (B, n), generator=g, device=DEV, dtype=torch.int32)
    u = torch.rand((B, n + 1), generator=g, device=DEV)
    tokens, accepted = xc.verify_drafts(x, p, None, u)
    for b0, b1 in ((0, 5), (65533, 65536), (65534, min(B, 65540)), (B - 3, B)):
        some = xc.verify_drafts(x[b0:b1].clone(), p[b0:b1].clone(), None, u[b0:b1].clone())
        assert torch.equal(some[0], tokens[b0:b1]) and torch.equal(some[1], accepted[b0:b1])


def test_as_many_sequences_as_have_more_threads_than_32_bits_count():
    import paper_2409_20156_amd as xc
    B = (1 << 24) + 9
    p = torch.ones((B, 1, 1), dtype=BF16, device=DEV)
    p[B - 2] = 0
    tokens, accepted = xc.verify_drafts(torch.zeros((B, 0), dtype=torch.int32, device=DEV), p, None, torch.zeros((B, 1), device=DEV))
    assert int(tokens[B - 2]) == -1 and int(tokens.sum()) == -1 and int(accepted.sum()) == 0


def test_nothing_behind_the_outputs_is_written_and_the_workspace_may_hold_anything():
    import paper_2409_20156_amd as xc
    x, p, q, u = _case(8, 33, 3, 10007, F32)
    want = _run(x, p, q, u)
    flat = torch.full((33 * 4 + 64,), 77, dtype=torch.int32, device=DEV)
    acc = torch.full((33 + 31,), 77, dtype=torch.int32, device=DEV)
    need = xc.verify_workspace(33, 10007)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)        # sums that are no numbers
    got = _run(x, p, q, u, workspace=ws[:need], out=(flat[: 33 * 4].view(33, 4), acc[:33]))
    assert (got[0] == want[0]).all() and (got[1] == want[1]).all()
    assert (flat[33 * 4:] == 77).all() and (acc[33:] == 77).all() and (ws[need:] == 255).all()


def test_offsets_beyond_32_bits():
    import paper_2409_20156_amd as xc
    B, n, V = 40, 3, 14_000_003                            # 2.2e9 probabilities
    p = torch.zeros((B, n + 1, V), dtype=BF16, device=DEV)
    x = torch.tensor([[V - 1 - b, 5 * b, V // 2] for b in range(B)], dtype=torch.int32)
    for b in range(B):
        stand = b % (n + 1)
        for i in range(n + 1):
            p[b, i, int(x[b, i]) if i < stand else (V - 7 - 3 * b - i)] = 0.5
    u = torch.rand((B, n + 1), device=DEV) * 0.49
    tokens, accepted = xc.verify_drafts(x.to(DEV), p, None, u)
    tokens = tokens.cpu()
    assert accepted.cpu().tolist() == [b % 4 for b in range(B)]
    for b in range(B):
        a = b % 4
        assert tokens[b].tolist() == x[b, :a].tolist() + [V - 7 - 3 * b - a] + [-1] * (n - a)


@pytest.mark.parametrize("B,V", [(2, 40000), (300, 1000), (5, 20000)])
def test_another_stream_and_a_replayed_graph(B, V):
    import paper_2409_20156_amd as xc
    x, p, q, u = [t.to(DEV) for t in _case(3, B, 3, V, F32)]
    want = xc.verify_drafts(x, p, q, u)
    ws = torch.empty(xc.verify_workspace(B, V), dtype=torch.uint8, device=DEV)
    out = tuple(torch.zeros_like(t) for t in want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        xc.verify_drafts(x, p, q, u, workspace=ws, out=out)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        xc.verify_drafts(x, p, q, u, workspace=ws, out=out)
    for k in range(3):
        for dst, src in zip((x, p, q, u), _case(50 + k, B, 3, V, F32)):
            dst.copy_(src)
        want = xc.verify_drafts(x, p, q, u)
        out[0].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals_on_the_device():
    import paper_2409_20156_amd as xc
    x, p, q, u = [t.to(DEV) for t in _case(3, 2, 3, 101, F32)]
    with pytest.raises(ValueError):
        xc.verify_drafts(x, p.transpose(1, 2).contiguous().transpose(1, 2), q, u)
    with pytest.raises(TypeError):
        xc.verify_drafts(x.long(), p, q, u)
    with pytest.raises(TypeError):
        xc.verify_drafts(x, p, q, u.double())
    with pytest.raises(ValueError):
        xc.verify_drafts(x.cpu(), p, q, u)
    with pytest.raises(xc.XcError):
        xc.verify_drafts(x, p, q, u, workspace=torch.empty(0, dtype=torch.uint8, device=DEV))
    with pytest.raises(xc.XcError):
        xc.verify_drafts(x[1:], p[1:], q[1:], u[1:])       # rows from addresses that are no multiples of 16


@pytest.mark.parametrize("B,V,verify,sums", [(5, 3000, 1, 0), (3, 20000, 1, 0), (200, 40000, 1, 0), (3, 40000, 1, 1), (70000, 2, 2, 0)])
def test_event_timing_counts_every_launch(B, V, verify, sums):
    import paper_2409_20156_amd as xc
    from paper_2409_20156_amd import binding
    p, u = torch.rand((B, 2, V), device=DEV).to(BF16), torch.rand((B, 2), device=DEV)
    x = torch.zeros((B, 1), dtype=torch.int32, device=DEV)
    binding.profile_reset()
    binding.profile_enable(True)
    try:
        xc.verify_drafts(x, p, None, u)
    finally:
        binding.profile_enable(False)
    prof = binding.profile_collect()
    binding.profile_reset()
    assert {k: n for k, (_, n) in prof.items() if n} == {k: n for k, n in (("verify", verify), ("verify_sums", sums)) if n}
