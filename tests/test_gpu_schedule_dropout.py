"""Alg. 1's outer loop with dropout of the embeddings: losses, returned gradients and the final classifier against the oracle's
own trajectory; a resumed schedule drops the same elements."""
import numpy as np
import pytest
import torch

from oracle import astra_oracle as orc
from oracle import serving_oracle as so
from paper_2409_20156_amd import synth
from tests.parity import TOL, check_rows_close, f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
L, d, B, pool, k_p, k_h, k_r = 4096, 64, 32, 64, 2, 8, 16
TAU_S, TAU_R, LR, RATE = 1, 2, 0.3, 0.2


def _inputs():
    W = synth.make_matrix(12, synth.TAG_W, L, d, torch.float32, DEV)
    Z = synth.make_matrix(12, synth.TAG_Z, pool, d, torch.float32, DEV)
    pos = synth.zipf_positives(12, pool, L, 1.0, "uniform:1:2", k_p)
    return W, synth.add_positive_signal(Z, W, pos), pos


def test_schedule_with_dropout_matches_oracle():
    from paper_2409_20156_amd.schedule import Schedule
    W, Z, pos = _inputs()
    steps = 6
    seeds = [synth.step_seed(synth.BASE_SEED, 9, t) for t in range(steps)]
    W64, Z64 = f64(W), f64(Z)
    sch = Schedule(Z, W, torch.tensor(pos, device=DEV), B, k_h, k_r, TAU_S, TAU_R, LR, dropout=RATE)
    tol = 20 * TOL["f32"]                  # rounding differences compound over the steps
    shortlist = None
    for t in range(steps):
        out = sch.step(seeds[t])
        torch.cuda.synchronize()
        if t >= TAU_S and (t - TAU_S) % TAU_R == 0:
            shortlist, _ = orc.mine_negatives(Z64, W64, k_h)               # on the whole embeddings
            assert (np.sort(sch.shortlist[sch.built].cpu().numpy(), axis=1) == np.sort(shortlist, axis=1)).all()
        lo = t % (pool // B) * B
        neg, logq = orc.sample_negatives(shortlist[lo:lo + B] if shortlist is not None else None, B, k_h, k_r, L, seeds[t])
        keep = so.dropout_kept(B, d, RATE, seeds[t])
        assert 0.1 < 1 - keep.mean() < 0.3
        ref = orc.xc_step(so.dropout(Z64[lo:lo + B], RATE, seeds[t]), W64, pos[lo:lo + B], neg, logq, LR, storage="f32")
        W64[ref["touched"]] = ref["W_rows"]
        loss = float(out["loss"].item())
        assert abs(loss - ref["loss"]) <= tol * abs(ref["loss"]), (t, loss, ref["loss"])
        dZ = out["dZ"].cpu().double().numpy()
        assert (dZ[~keep] == 0).all()
        check_rows_close(dZ, so.dropout(ref["dZ"], RATE, seeds[t]), tol, "dZ of step %d" % t)
    check_rows_close(f64(W), W64, tol, "W after the schedule")


def test_a_resumed_schedule_drops_the_same_elements():
    from paper_2409_20156_amd.schedule import Schedule
    seeds = [synth.step_seed(synth.BASE_SEED, 9, t) for t in range(6)]
    runs = []
    for cut in (None, 3):
        W, Z, pos = _inputs()
        make = lambda w: Schedule(Z, w, torch.tensor(pos, device=DEV), B, k_h, k_r, TAU_S, TAU_R, LR, dropout=RATE)  # noqa: E731
        sch, losses = make(W), []
        for t in range(6):
            if t == cut:
                saved = sch.state_dict()
                W = torch.zeros_like(W)
                sch = make(W)
                sch.load_state_dict(saved)
            losses.append(sch.step(seeds[t])["loss"].item())
        runs.append((losses, W.cpu()))
    assert runs[0][0] == runs[1][0] and torch.equal(runs[0][1], runs[1][1])


def test_dropout_outside_its_range_is_refused():
    from paper_2409_20156_amd.schedule import Schedule
    W, Z, pos = _inputs()
    for rate in (-0.1, 1.0, float("nan")):
        with pytest.raises(ValueError):
            Schedule(Z, W, torch.tensor(pos, device=DEV), B, k_h, k_r, TAU_S, TAU_R, LR, dropout=rate)


@pytest.mark.parametrize("rate", [0.0, RATE])
def test_the_rate_is_saved_and_states_without_one_are_those_of_schedules_without_dropout(rate):
    from paper_2409_20156_amd.schedule import Schedule
    W, Z, pos = _inputs()
    make = lambda r: Schedule(Z, W, torch.tensor(pos, device=DEV), B, k_h, k_r, TAU_S, TAU_R, LR, dropout=r)  # noqa: E731
    sch = make(rate)
    sch.step(5)
    saved = sch.state_dict()
    assert saved["dropout"] == rate
    sch.load_state_dict(saved)
    assert sch.t == 1
    with pytest.raises(ValueError, match="dropout"):
        make(0.5).load_state_dict(saved)
    del saved["dropout"]
    if rate == 0.0:
        sch.load_state_dict(saved)                         # as saved before there was a rate
    else:
        with pytest.raises(ValueError, match="dropout"):
            sch.load_state_dict(saved)
