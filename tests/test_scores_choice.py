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
            assert choose(*s, 4) == choose(*s, 2) == kernel, s
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
                    seen |= {choose(B, L, d, 4), choose(B, L, d, 2)}
    assert seen == set(scores_choice.KERNELS)


@pytest.mark.parametrize("out", [4, 2])
@pytest.mark.parametrize("B,L,d", [(100000, 384, 768), (65948, 512, 768), (185429, 475, 192), (32972, 1024, 384), (22521, 1499, 768),
                                   (57344, 1536, 192), (20000, 1500, 768), (13381, 2523, 384), (8192, 4500, 768), (7385, 4571, 768),
                                   (19269, 4571, 192), (6600, 5120, 768), (2 ** 31 - 1, 512, 768)])
def test_labels_are_not_held_where_most_compute_units_would_have_none(choose, B, L, d, out):
    """The label-holding kernel gives whole tiles of 512 labels to an XCD: these calls have 1, 2, 3, 5, 9 and 10 of them."""
    assert choose(B, L, d, out) in ("mid", "many")


@pytest.mark.parametrize("B,L,d", [(4096, 8700, 768), (3880, 8704, 768), (5996, 5632, 384), (2001, 16859, 768), (2645, 12763, 192)])
def test_uneven_shares_count_where_the_scores_are_bf16(choose, B, L, d):
    assert choose(B, L, d, 2) == "mid" and choose(B, L, d, 4) == "held"


@pytest.mark.parametrize("out", [4, 2])
@pytest.mark.parametrize("B,L,d", [(4096, 131072, 768), (21697, 4059, 768), (24829, 3547, 192), (10797, 8155, 768), (10161, 8667, 768),
                                   (6901, 12763, 384), (4201, 20955, 768), (1013, 33243, 768), (846, 569976, 192)])
def test_labels_are_held_where_all_have_some(choose, B, L, d, out):
    assert choose(B, L, d, out) == "held"
