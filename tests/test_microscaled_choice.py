"""The rule by which a call of scores_microscaled takes a kernel (no GPU needed)."""
import pytest

from tests import microscaled_choice
from tests.test_gpu_microscaled_kernels import CASES


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    return microscaled_choice.build(str(tmp_path_factory.mktemp("choice")))


def test_every_kernel_is_run_at_its_own_sizes(choose):
    assert set(CASES) == set(microscaled_choice.KERNELS)
    for kernel, sizes in CASES.items():
        for s in sizes:
            assert choose(*s) == kernel, s
        # rows of whole pairs of units, of a single one at the end, of a part of one; whole and part-filled groups of 64 labels
        units = {(d + 127) // 128 for _, _, d in sizes}
        assert any(u % 2 == 0 for u in units) and any(u % 2 for u in units) and any(d % 128 for _, _, d in sizes), kernel
        assert any(L % 64 == 0 for _, L, _ in sizes) and any(L % 2 for _, L, _ in sizes), kernel
    # short and long places in LDS for few queries; 2, 4, 6 and 8 units held
    assert {(d + 127) // 128 <= 8 for _, _, d in CASES["online"]} == {False, True}
    assert {(d + 255) // 256 for _, _, d in CASES["held"]} == {1, 2, 3, 4}


def test_every_size_has_a_kernel(choose):
    seen = set()
    for B in (1, 2, 4, 15, 16, 17, 64, 128, 129, 256, 257, 1000, 5000, 100000, 2 ** 31 - 1):
        for L in (1, 10, 1000, 3584, 3585, 16385, 131072, 1300000, 120_000_000, 2 ** 31 - 1):
            for d in (8, 128, 136, 768, 1024, 1032, 4096, 4104, 131072):
                if B * L <= 2 ** 40:
                    seen.add(choose(B, L, d))
    assert seen == set(microscaled_choice.KERNELS)


def test_bounds_of_the_rules(choose):
    assert choose(16, 10, 1024) == "online" and choose(16, 10, 1032) == "few" and choose(17, 10, 1024) == "small"
    assert choose(4, 10, 4096) == "online" and choose(5, 10, 4096) == "few" and choose(4, 10, 4104) == "small"
    assert choose(257, 131072, 1024) == "held" and choose(256, 131072, 1024) != "held" and choose(257, 131072, 1032) != "held"
    assert choose(10 ** 6, 3585, 8) == "held" and choose(10 ** 6, 3584, 8) == "large"              # eight tiles of labels, one to an XCD
    assert choose(8192, 4096, 768) == "held" and choose(8128, 4096, 768) != "held"                 # four stages to a compute unit
