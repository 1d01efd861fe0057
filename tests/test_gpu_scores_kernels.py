"""Every kernel that scores_quantized can take, at sizes that take it, bit for bit against the definition: the sums of the integers in 64 bits
(exact), then the three roundings of the formula.  tests/test_scores_choice.py checks that the sizes take the kernels they stand under."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32

CASES = {  # kernel -> (queries, labels, elements of a row)
    "online": [(1, 131072, 768), (1, 33001, 24), (16, 40007, 704), (9, 20000, 128)],
    "thin": [(1, 3453, 2872), (16, 5000, 776), (32, 5003, 72), (20, 8192, 1024)],
    "narrow": [(17, 9001, 72), (32, 30000, 1032), (25, 16384, 256)],
    "few": [(20, 33000, 776), (32, 40000, 72), (30, 32769, 1032), (5, 60000, 896), (32, 50001, 128)],
    "low": [(33, 8000, 200), (128, 4000, 2048), (300, 1601, 72)],
    "small": [(40, 20001, 136), (128, 16000, 768), (500, 4001, 1032), (64, 32768, 64)],
    "some": [(64, 40000, 768), (33, 40001, 72), (47, 33001, 776), (64, 70000, 128), (60, 33001, 128)],
    "held": [(137, 131072, 128), (9600, 3549, 64), (10000, 3549, 768), (8400, 4095, 384), (4137, 8155, 136), (385, 90001, 600)],
    "mid": [(100, 40000, 768), (128, 33000, 128), (65, 33001, 24), (100, 33001, 200), (300, 60000, 200), (128, 70001, 1032)],
    "many": [(256, 40000, 64), (200, 60001, 24), (256, 40003, 128), (193, 64001, 800), (600, 17000, 800)],
}


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("kernel,B,L,d", [(k, *s) for k, sizes in CASES.items() for s in sizes])
def test_bits_are_those_of_the_definition(kernel, B, L, d, out_dtype):
    import paper_2409_20156_amd as xc
    g = torch.Generator(device=DEV).manual_seed(B + L + d)
    Z = torch.randn((B, d), device=DEV, generator=g).to(BF16)
    Q = torch.randint(-127, 128, (L, xc.quantized_pitch(d)), dtype=torch.int8, device=DEV, generator=g)
    Q[:, d:] = 0
    s = torch.rand(L, device=DEV, generator=g)
    flat = torch.full((B * L + 128,), 77.0, dtype=out_dtype, device=DEV)
    out = flat[64:B * L + 64].view(B, L)
    xc.scores_quantized(Z, Q, s, out=out)
    torch.cuda.synchronize()
    assert (flat[:64] == 77).all() and (flat[B * L + 64:] == 77).all()
    P, a = xc.quantize_rows(Z)
    P = P.double()
    step = max(1, 40_000_000 // B)
    for l in range(0, L, step):
        sums = P @ Q[l:l + step].double().t()             # whole numbers below 2^53
        want = ((sums.to(F32) * a[:, None]) * s[None, l:l + step]).to(out_dtype)
        assert torch.equal(out[:, l:l + step], want), "labels from %d on" % l


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("B,L,d", [(100000, 384, 64), (65600, 512, 128), (34205, 987, 200), (22521, 1499, 72), (13381, 2523, 384), (7385, 4571, 768),
                                   (3880, 8704, 136), (9517, 3547, 72), (24829, 3547, 24), (9800, 3572, 128), (10161, 8667, 64)])
def test_many_queries_on_few_labels(B, L, d, out_dtype):
    test_bits_are_those_of_the_definition("", B, L, d, out_dtype)
