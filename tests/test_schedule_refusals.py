"""What a schedule refuses before it allocates, searches or samples anything (no GPU needed)."""
import pytest
import torch

from paper_2409_20156_amd.schedule import Schedule


def _schedule(**kw):
    Z, W, pos = torch.zeros((8, 16)), torch.zeros((40, 16)), torch.zeros((8, 1), dtype=torch.int32)
    return Schedule(Z, W, pos, 4, 2, 4, 0, 2, 0.1, **kw)


@pytest.mark.parametrize("rate", [-0.1, 1.0, float("nan"), float("inf"), 0.9999999, 0.999999, 1 - 2.0 ** -17, 0.9999924])
def test_rates_that_the_kernel_refuses_are_refused_at_once(rate):
    """floor(65536 rate + 1/2) is 65536 from 1 - 2^-17 on: xc_dropout refuses these, and no step may get as far as that."""
    with pytest.raises(ValueError):
        _schedule(dropout=rate)


@pytest.mark.parametrize("rate", [0.0, 1e-6, 0.5, 0.99, 0.99998, 65535 / 65536, 0.99999])
def test_rates_that_the_kernel_takes_are_taken(rate):
    assert _schedule(dropout=rate).dropout == rate


def _state(sch, **kw):
    return {"t": 3, "cur": 0, "built": 0, "had_previous": False, "pending": None, "full_repeats": 0,
            "shortlist": [torch.ones_like(x) for x in sch.shortlist], "W": torch.ones_like(sch.W), **kw}


@pytest.mark.parametrize("rate,saved", [(0.0, {"dropout": 0.1}), (0.1, {"dropout": 0.0}), (0.1, {}), (0.1, {"dropout": 0.2}),
                                        (0.1, {"dropout": 0.1 + 2.0 ** -15})])
def test_a_state_of_another_dropout_rate_is_refused_and_nothing_is_changed(rate, saved):
    sch = _schedule(dropout=rate)
    W, lists = sch.W.clone(), [x.clone() for x in sch.shortlist]
    with pytest.raises(ValueError, match="dropout"):
        sch.load_state_dict(_state(sch, **saved))
    assert torch.equal(sch.W, W) and sch.t == 0 and all(torch.equal(a, b) for a, b in zip(sch.shortlist, lists))
