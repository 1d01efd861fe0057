"""Every kernel that scores_microscaled can take, at sizes that take it, bit for bit against the definition.  Codes are drawn, every block
of a query holds a 4 or a 6 (so that it is laid out as it was drawn) and scales are 2^-1, 1 and 2: products are multiples of 2^-4, and a sum over
up to 4096 elements stays below 4096 * 36 * 4 < 2^20, so that every partial sum is exact in fp32, in any order, and a score is rounded
once, to its own type.  tests/test_microscaled_choice.py checks that the sizes take the kernels they stand under."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32

CASES = {  # kernel -> (queries, labels, elements of a row)
    "online": [(1, 131072, 768), (1, 33, 8), (16, 40007, 128), (16, 3201, 1000), (3, 5000, 2104), (4, 8000, 4096), (1, 64, 3208)],
    "few": [(16, 5001, 4096), (16, 33001, 1032), (9, 64, 1960), (5, 20000, 3976), (13, 3973, 2048)],
    "held": [(4100, 8001, 128), (4097, 8192, 72), (2050, 16000, 256), (4100, 8100, 384), (2112, 16385, 640), (300, 140001, 512), (257, 131072, 768),
             (4100, 8001, 1000), (1000, 33000, 1024), (400, 270000, 136)],
    "small": [(17, 64, 384), (33, 129, 200), (100, 50021, 2048), (256, 30000, 768), (300, 2001, 1032), (20, 500, 4000), (130, 8320, 136)],
    "large": [(2000, 8000, 1288), (4096, 4095, 2048), (1000, 40003, 1160), (2048, 8192, 1408), (700, 20000, 4096)],
}


def _codes(g, n, d):
    """fp32 [n, d]: values of codes, a 4 or a 6 in every block among them, times 2^-1, 1 or 2 block by block."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    v = grid[torch.randint(0, 8, (n, d), device=DEV, generator=g)] * (1 - 2.0 * torch.randint(0, 2, (n, d), device=DEV, generator=g))
    v[:, ::32] = grid[torch.randint(6, 8, (n, (d + 31) // 32), device=DEV, generator=g)]
    e = torch.randint(-1, 2, (n, (d + 31) // 32), device=DEV, generator=g).repeat_interleave(32, 1)[:, :d]
    return torch.ldexp(v, e)


@pytest.mark.parametrize("kernel,B,L,d", [(k, *s) for k, sizes in CASES.items() for s in sizes])
def test_bits_are_those_of_the_definition(kernel, B, L, d):
    import paper_2409_20156_amd as xc
    g = torch.Generator(device=DEV).manual_seed(B + L + d)
    Z, W = _codes(g, B, d), _codes(g, L, d)
    Q, s = xc.microscale_rows(W)
    for out_dtype, in_dtype in ((F32, BF16), (BF16, F32)):
        flat = torch.full((B * L + 128,), 77.0, dtype=out_dtype, device=DEV)
        out = flat[64:B * L + 64].view(B, L)
        xc.scores_microscaled(Z.to(in_dtype), Q, s, out=out)
        torch.cuda.synchronize()
        assert (flat[:64] == 77).all() and (flat[B * L + 64:] == 77).all()
        step = max(1, 40_000_000 // B)
        for l in range(0, L, step):
            want = (Z.double() @ W[l:l + step].double().t().contiguous()).to(out_dtype)
            assert torch.equal(out[:, l:l + step], want), "labels from %d on" % l
        del flat, out
