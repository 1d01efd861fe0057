"""Rows in 8 bits and the scores of all labels from them, against the oracle: integers and scales equal, scores within the
roundings that their formula has (the sum to fp32 and two products: 3 * 2^-24 relative; bf16 results 2^-8 more)."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as so

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _rows(seed, n, d, dtype, spread=1.0):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(n, d)) * np.exp(spread * rng.normal(size=(n, 1)))
    return torch.tensor(x, dtype=F32).to(dtype)


def _guarded(shape, dtype, fill):
    """A tensor with 64 elements of `fill` on either side; returns it and a check that these are still there."""
    n = int(np.prod(shape))
    flat = torch.full((n + 128,), fill, dtype=dtype, device=DEV)

    def intact():
        assert (flat[:64] == fill).all() and (flat[n + 64:] == fill).all()
    return flat[64:n + 64].view(shape), intact


def _check_scores(got, P, a, Q, s, dtype):
    want = so.scores_quantized(P, a, Q, s)
    bound = np.abs(want) * (3.01 * 2.0 ** -24 + (2.0 ** -8 if dtype == BF16 else 0)) + 2.0 ** -148
    assert (np.abs(got.cpu().double().numpy() - want) <= bound).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,d", [(1, 8), (1, 16), (3, 24), (5, 64), (63, 72), (64, 136), (65, 256), (130, 768), (7, 1024),
                                 (33, 2056), (4, 4096), (3, 4104), (2, 8200), (2, 20008), (1, 131072), (1000, 40)])
def test_rows_in_8_bits(dtype, n, d):
    import paper_2409_20156_amd as xc
    X = _rows(n * 10007 + d, n, d, dtype)
    if n > 2:
        X[1] = 0
        X[2, d // 2] = -X[2].abs().max() * 2
        X[2, d // 3] = X[2].abs().max() / 2               # a half exactly: 63.5
    Q, checkQ = _guarded((n, xc.quantized_pitch(d)), torch.int8, 77)
    s, check_s = _guarded((n,), F32, 77.0)
    xc.quantize_rows(X.to(DEV), out=(Q, s))
    torch.cuda.synchronize()
    wantQ, want_s = so.quantize_rows(X.double().numpy())
    assert (Q.cpu().numpy() == wantQ).all() and (s.cpu().numpy() == want_s).all()
    checkQ()
    check_s()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_near_halves_and_at_the_ends_of_the_range(dtype):
    import paper_2409_20156_amd as xc
    rng = np.random.default_rng(8)
    X = torch.zeros((400, 64), dtype=F32)
    for i in range(400):
        m = np.float32(rng.uniform(1, 2)) if i % 2 else np.float32((127 + 127 * (i % 3)) / 128)
        k = rng.integers(-127, 127, size=64)
        X[i] = torch.tensor(np.float32((k + 0.5) * np.float64(m) / 127))      # as near a half as fp32 comes
        X[i, ::3] = torch.nextafter(X[i, ::3], torch.full((22,), 9.0))
        X[i, 5] = float(m)
        X[i] *= 2.0 ** float(rng.integers(-148, 127) if i < 200 else rng.integers(-20, 20))
    X[390] = 3.0e38
    X[391] = 1.0e-45                                       # the smallest fp32
    X[392, 3] = float("inf")
    X[393, 3] = float("nan")
    X[394, 63] = -float("inf")
    X = X.to(dtype)
    Q, s = xc.quantize_rows(X.to(DEV))
    wantQ, want_s = so.quantize_rows(X.double().numpy())
    got_s = s.cpu().numpy()
    assert (Q.cpu().numpy() == wantQ).all()
    assert ((got_s == want_s) | (np.isnan(got_s) & np.isnan(want_s))).all()


@pytest.mark.parametrize("count", [None, 0, 3, 50])
def test_only_the_rows_asked_for_are_written(count):
    import paper_2409_20156_amd as xc
    n, d = 300, 72
    X = _rows(5, n, d, BF16)
    ids = torch.tensor([7, 299, 0, 7, -1, 300, 2 ** 31 - 1, -5, 128, 64], dtype=torch.int32)
    Q = torch.full((n, 80), 55, dtype=torch.int8, device=DEV)
    s = torch.full((n,), -3.0, device=DEV)
    c = None if count is None else torch.tensor([count], dtype=torch.int32, device=DEV)
    out = xc.quantize_rows(X.to(DEV), rows=ids.to(DEV), count=c, out=(Q, s))
    assert out[0] is Q
    wantQ, want_s = so.quantize_rows(X.double().numpy())
    listed = [i for i in ids[:count].tolist() if 0 <= i < n]
    keep = np.ones(n, dtype=bool)
    keep[listed] = False
    gotQ, got_s = Q.cpu().numpy(), s.cpu().numpy()
    assert (gotQ[~keep] == wantQ[~keep]).all() and (got_s[~keep] == want_s[~keep]).all()
    assert (gotQ[keep] == 55).all() and (got_s[keep] == -3.0).all()
    xc.quantize_rows(X.to(DEV), rows=ids[:0].to(DEV), out=(Q, s))           # none
    assert (Q.cpu().numpy() == gotQ).all()


SHAPES = [  # B, L, d
    (1, 1, 8), (1, 15, 16), (2, 63, 24), (1, 64, 64), (1, 65, 72), (1, 1000, 768), (1, 4099, 4096), (3, 257, 136), (7, 300, 40),
    (15, 129, 64), (16, 128, 128), (17, 127, 256), (31, 500, 200), (32, 512, 768), (33, 511, 768), (40, 1030, 1000), (63, 333, 72),
    (64, 700, 512), (65, 255, 384), (96, 2049, 88), (127, 256, 320), (128, 1000, 768), (129, 257, 264), (200, 1537, 104),
    (255, 600, 192), (256, 256, 768), (257, 1023, 776), (300, 5003, 304), (513, 515, 1544), (1000, 777, 64), (5, 2000, 8208),
    (130, 300, 16400), (2, 70, 131072), (700, 3000, 8), (20, 9001, 72), (32, 16000, 200), (17, 12289, 776), (16, 33001, 1000),
    (9, 10001, 800), (100, 9001, 136), (33, 7900, 16), (1, 40000, 16), (3, 33000, 1032)]


@pytest.mark.parametrize("B,L,d", SHAPES)
@pytest.mark.parametrize("dtype,out_dtype", [(BF16, F32), (BF16, BF16), (F32, F32), (F32, BF16)])
def test_scores(B, L, d, dtype, out_dtype):
    import paper_2409_20156_amd as xc
    Z, W = _rows(B + 7 * d, B, d, dtype), _rows(L + 13 * d, L, d, dtype)
    if B > 4:
        Z[3] = 0
    if L > 20:
        W[17] = 0
    P, a = so.quantize_rows(Z.double().numpy())
    Q, s = so.quantize_rows(W.double().numpy())
    out, intact = _guarded((B, L), out_dtype, 77.0)
    ws, ws_intact = _guarded((xc.scores_workspace(B, d),), torch.uint8, 201)
    got = xc.scores_quantized(Z.to(DEV), torch.tensor(Q, device=DEV), torch.tensor(s, device=DEV), out=out, workspace=ws)
    torch.cuda.synchronize()
    assert got is out
    _check_scores(got, P, a, Q, s, out_dtype)
    intact()
    ws_intact()


def test_largest_integers_do_not_overflow():
    import paper_2409_20156_amd as xc
    d = 131072
    Z = torch.ones((3, d), device=DEV)
    Z[1] = -1
    Q, s = xc.quantize_rows(torch.ones((40, d), device=DEV))
    got = xc.scores_quantized(Z, Q, s).cpu().double()
    one = float(np.float32(1) / np.float32(127))
    want = 127.0 * 127 * d * one * one
    assert (got[0] / want - 1).abs().max() <= 3.01 * 2.0 ** -24 and torch.equal(got[1], -got[0])


def test_rows_that_are_not_finite_give_scores_that_are_no_numbers():
    import paper_2409_20156_amd as xc
    Z, W = _rows(1, 9, 64, F32), _rows(2, 70, 64, F32)
    Z[4, 3] = float("inf")
    W[33, 60] = float("nan")
    Q, s = xc.quantize_rows(W.to(DEV))
    got = xc.scores_quantized(Z.to(DEV), Q, s).cpu()
    want = torch.zeros((9, 70), dtype=torch.bool)
    want[4], want[:, 33] = True, True
    assert torch.equal(got.isnan(), want)


@pytest.mark.parametrize("B", [1, 40, 300])
def test_a_range_of_labels_and_every_batch_size_give_the_same_bits(B):
    import paper_2409_20156_amd as xc
    Z, W = _rows(3, 300, 200, BF16).to(DEV), _rows(4, 3000, 200, BF16).to(DEV)
    Q, s = xc.quantize_rows(W)
    every = xc.scores_quantized(Z, Q, s)
    part = xc.scores_quantized(Z[:B].contiguous(), Q[1000:2304], s[1000:2304])
    assert torch.equal(part, every[:B, 1000:2304])


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("B,L,d", [(290, 70001, 24), (137, 131072, 128), (290, 70004, 200), (261, 100000, 384), (500, 50021, 512),
                                   (700, 40000, 600), (290, 70001, 768), (1025, 30000, 768), (300, 30001, 776), (600, 20000, 1096),
                                   (2049, 8005, 2064), (430, 60001, 24), (400, 57856, 128), (450, 60004, 200), (500, 58000, 384),
                                   (390, 58001, 512), (256, 131072, 128), (255, 140001, 768), (253, 133000, 24), (140, 150001, 104), (300, 100010, 384), (385, 270000, 64),
                                   (2809, 20011, 232), (1000, 131071, 64), (600, 170000, 128)])
def test_large_calls_have_the_bits_of_small_ones(B, L, d, out_dtype):
    """The kernels of large calls against those of small ones, which the oracle checks above."""
    import paper_2409_20156_amd as xc
    g = torch.Generator(device=DEV).manual_seed(B + L + d)
    Z = torch.randn((B, d), device=DEV, generator=g).to(BF16)
    Q = torch.randint(-127, 128, (L, xc.quantized_pitch(d)), dtype=torch.int8, device=DEV, generator=g)
    Q[:, d:] = 0
    s = torch.rand(L, device=DEV, generator=g)
    out, intact = _guarded((B, L), out_dtype, 77.0)
    xc.scores_quantized(Z, Q, s, out=out)
    torch.cuda.synchronize()
    intact()
    # 32 queries at a time on all labels; then all queries on the first and last labels
    for q in list(range(0, B, 32))[:3] + [B - 30]:
        few = xc.scores_quantized(Z[q:q + 30].contiguous(), Q, s, dtype=out_dtype)
        assert torch.equal(out[q:q + 30], few)
    for l in (0, (L // 2) // 64 * 64, (L - 300) // 4 * 4):
        n = min(400, L - l)
        some = torch.cat([xc.scores_quantized(Z[q:q + 64].contiguous(), Q[l:l + n], s[l:l + n], dtype=out_dtype) for q in range(0, B, 64)])
        assert torch.equal(out[:, l:l + n], some)


def test_offsets_beyond_32_bits():
    import paper_2409_20156_amd as xc
    # 4.9 GB of rows, few queries; and 4.4 GB of scores
    L, d = 6_400_003, 768
    Q = torch.randint(-127, 128, (L, d), dtype=torch.int8, device=DEV)
    s = torch.rand(L, device=DEV)
    Z = _rows(9, 3, d, BF16)
    P, a = so.quantize_rows(Z.double().numpy())
    got = xc.scores_quantized(Z.to(DEV), Q, s)
    at = torch.tensor([0, 1, 2796202, 2796203, 5592405, 5592406, L - 130, L - 2, L - 1], device=DEV)
    _check_scores(got[:, at], P, a, Q[at].cpu().numpy(), s[at].cpu().numpy(), F32)
    del got, Q
    B, L, d = 2100, 1_050_001, 64
    Q = torch.randint(-127, 128, (L, d), dtype=torch.int8, device=DEV)
    Z = _rows(10, B, d, BF16)
    P, a = so.quantize_rows(Z.double().numpy())
    out = torch.zeros((B, L), dtype=BF16, device=DEV)
    xc.scores_quantized(Z.to(DEV), Q, s[:L], out=out)
    rows = torch.tensor([0, 1022, 1023, 2045, 2046, B - 1], device=DEV)
    at = torch.tensor([0, 1, 255, 256, 524288, L - 257, L - 256, L - 2, L - 1], device=DEV)
    _check_scores(out[rows][:, at], P[rows.cpu()], a[rows.cpu()], Q[at].cpu().numpy(), s[at].cpu().numpy(), BF16)


def test_another_stream_and_a_replayed_graph():
    import paper_2409_20156_amd as xc
    Z, W = _rows(11, 70, 768, BF16).to(DEV), _rows(12, 1500, 768, BF16).to(DEV)
    Q, s = xc.quantize_rows(W)
    want = xc.scores_quantized(Z, Q, s)
    ws = torch.empty(xc.scores_workspace(70, 768), dtype=torch.uint8, device=DEV)
    out = torch.zeros_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        xc.scores_quantized(Z, Q, s, workspace=ws, out=out)
    side.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    rows = (torch.zeros_like(Q), torch.zeros_like(s))
    with torch.cuda.graph(g):
        xc.quantize_rows(W, out=rows)
        xc.scores_quantized(Z, *rows, workspace=ws, out=out)
    for k in range(3):
        Z.copy_(_rows(20 + k, 70, 768, BF16))
        W.copy_(_rows(30 + k, 1500, 768, BF16))
        Q, s = xc.quantize_rows(W)
        want = xc.scores_quantized(Z, Q, s)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_two_calls_at_once_with_workspaces_of_their_own():
    import paper_2409_20156_amd as xc
    W = _rows(41, 20000, 512, BF16).to(DEV)
    Q, s = xc.quantize_rows(W)
    Z = [_rows(42 + i, 150, 512, BF16).to(DEV) for i in range(2)]
    want = [xc.scores_quantized(z, Q, s) for z in Z]
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for st, z in zip(side, Z):
        with torch.cuda.stream(st):
            got.append([xc.scores_quantized(z, Q, s) for _ in range(5)])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(x, w) for x in g)


def test_tensors_that_are_not_contiguous_or_not_aligned_are_refused():
    import paper_2409_20156_amd as xc
    Z = _rows(1, 8, 64, F32).to(DEV)
    Q, s = xc.quantize_rows(Z)
    with pytest.raises(ValueError):
        xc.scores_quantized(Z.t().contiguous().t(), Q, s)
    with pytest.raises(ValueError):
        xc.quantize_rows(Z.t().contiguous().t())
    with pytest.raises(xc.XcError):
        xc.scores_quantized(Z, Q[1:], s[1:])               # scales from an address that is no multiple of 16
    with pytest.raises(xc.XcError):
        xc.scores_quantized(Z, Q, s, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(TypeError):
        xc.scores_quantized(Z, Q.to(torch.uint8), s)
    with pytest.raises(ValueError):
        xc.scores_quantized(Z, Q, s.cpu())


def test_rows_that_a_training_step_touched_are_laid_out_again():
    """A step, its touched rows, the scores, a soft-max over them and drafted labels checked against it: used together."""
    import paper_2409_20156_amd as xc
    from oracle import astra_oracle as orc
    B, L, d, n = 24, 3000, 72, 3
    rng = np.random.default_rng(77)
    Z, W = _rows(50, B, d, BF16).to(DEV), _rows(51, L, d, BF16, 0.3).to(DEV)
    Q, s = xc.quantize_rows(W)
    pos = torch.tensor(rng.integers(0, L, (B, 2)), dtype=torch.int32, device=DEV)
    neg, logq = xc.sample_negatives(None, 0, 40, L, 5, B=B, device=DEV)
    Zd = xc.dropout(Z, 0.25, 5)
    step = xc.xc_step(Zd, W, pos, neg, logq, 0.5)
    dZ = xc.dropout_grad(step["dZ"], 0.25, 5)
    xc.quantize_rows(W, rows=step["touched"], count=step["n_touched"], out=(Q, s))
    allQ, all_s = xc.quantize_rows(W)
    assert torch.equal(Q, allQ) and torch.equal(s, all_s)
    scores = xc.scores_quantized(Z, Q, s)
    P, a = so.quantize_rows(Z.cpu().double().numpy())
    _check_scores(scores, P, a, Q.cpu().numpy(), s.cpu().numpy(), F32)
    # the step saw the dropped embeddings, and its gradient comes back through the same mask
    zd = so.dropout(Z.cpu().double().numpy(), 0.25, 5)
    assert (Zd.cpu().double().numpy() == orc.round_to_bf16(zd)).all()
    keep = so.dropout_kept(B, d, 0.25, 5)
    assert (dZ.cpu().numpy()[~keep] == 0).all()
    want = step["dZ"].cpu().double().numpy() * (65536 / (65536 - so.dropout_least(0.25)))
    assert (np.abs(dZ.cpu().double().numpy() - want)[keep] <= 2.01 * 2.0 ** -24 * np.abs(want)[keep]).all()
    # sequences of n drafts with n + 1 rows of scores each
    probs = scores.softmax(-1).view(B // (n + 1), n + 1, L)
    draft = (scores + 0.3 * torch.randn(scores.shape, device=DEV)).softmax(-1).view_as(probs)[:, :n].contiguous()
    x = torch.multinomial(draft.view(-1, L), 1).view(-1, n).to(torch.int32)
    u = torch.rand((B // (n + 1), n + 1), device=DEV)
    tokens, accepted = xc.verify_drafts(x, probs, draft, u)
    want = so.verify_drafts(x.cpu().numpy(), probs.cpu().double().numpy(), draft.cpu().double().numpy(), u.cpu().double().numpy())
    assert (tokens.cpu().numpy() == want[0]).all() and (accepted.cpu().numpy() == want[1]).all()
