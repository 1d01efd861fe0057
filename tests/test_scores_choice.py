"""The rule by which a call of scores_quantized takes a kernel (no GPU needed)."""
import pytest

from tests import scores_choice
from tests.test_gpu_scores_kernels import CASES


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    return scores_choice.build(str(tmp_path_factory.mktemp("choice")))


def test_every_kernel_is_run_at_its_own_sizes(choose):
    assert set(CASES) == set(scores_choice.KERNELS)
    for kernel, sizes in CASES.items():
        for s in sizes:
            assert choose(*s) == kernel, s
        # rows of whole stages and others, labels that fill the last tile of any kernel and others
        assert any(d % 128 == 0 or (d + 15) // 16 * 16 % 128 == 0 for _, _, d in sizes), kernel
        assert any((d + 15) // 16 * 16 % 128 != 0 for _, _, d in sizes), kernel
        assert any(L % 2 for _, L, _ in sizes), kernel


def test_every_size_has_a_kernel(choose):
    seen = set()
    for B in (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 192, 193, 256, 257, 384, 385, 1000, 5000, 100000, 2 ** 31 - 1):
        for L in (1, 10, 1000, 8191, 8193, 16385, 33001, 131072, 1300000, 120_000_000, 2 ** 31 - 1):
            for d in (8, 128, 136, 384, 392, 768, 776, 4096, 131072):
                if B * L <= 2 ** 40:
                    seen.add(choose(B, L, d))
    assert seen == set(scores_choice.KERNELS)
