"""Policy objectives over the whole range of their inputs: chosen actions that are excluded, and rows that are not
finite, in the preference loss; log ratios beyond fp32's exponentials in the clipped loss."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import objective as obj
from tests.gpu_util import log, require_gpu
from tests.test_gpu_objective import E, SEGS_26, TINY, Rows, _bars, _close, _grad_bar, check_pref, run_loss, run_pref

pytestmark = pytest.mark.gpu

# two pairs a wave's tile holds, and long tracks: the preference loss of typed heads in one launch and in three
SHORT, LONG = [2, 1, 3, 2, 1, 4], [130, 90, 1, 70, 65, 80]


def _ptr(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


@pytest.mark.parametrize("smoothing", [0.0, 0.1])
@pytest.mark.parametrize("segs", [SEGS_26, [0, 40], [0, 700], [0, 9001]], ids=lambda s: "%dx%d" % (s[-1], len(s) - 1))
def test_excluded_choice_in_one_track(segs, smoothing):
    """A track with an excluded action that was chosen has ratio -inf: the pair's loss is +inf where the preferred
    track has it (-(1 - s) log sigmoid(-inf) - s log sigmoid(inf)); where the rejected one has it, 0 without
    smoothing and +inf with.  The gradients stay finite."""
    require_gpu()
    for dtype in ("f32", "bf16"):
        for lens in (SHORT, LONG):
            ptr = _ptr(lens)
            for side in (0, 1):
                row = int(ptr[2 + side])

                def edit(z, acts):
                    z[row, acts[row, 0]] = -np.inf
                log("preference loss: %s head=%s tracks of %d, side %d" % (dtype, segs[-1:], lens[0], side))
                R = Rows(dtype, int(ptr[-1]), segs, seed=17, edit=edit)
                lp = obj.row_stats(R.z, segs, R.acts)["logp"]
                ref = (np.where(np.isfinite(lp), lp, -4.0) + 0.3 * R.rng.standard_normal(R.M)).astype(np.float32)
                cfg = dict(beta=0.2, smoothing=smoothing)
                got = run_pref(R, ref, None, ptr, cfg)
                O = check_pref(R, ref, None, ptr, cfg, got)
                assert got[1][2 + side] == -np.inf and np.isfinite(np.delete(got[1], 2 + side)).all()
                assert got[0][0] == (np.inf if side == 0 or smoothing else got[0][1]) and np.isfinite(got[2]).all()
                assert got[0][1] == (np.inf if side == 0 else got[0][1])
                # the excluded action keeps its part of the formula: g_logp (1 - 0)
                want = O["g_logp"][row]
                assert want != 0 or side == 1 and not smoothing
                assert abs(got[2][row, R.acts[row, 0]] - want) <= 2.0 ** (-8 if dtype == "bf16" else -22) * abs(want)


@pytest.mark.parametrize("smoothing", [0.0, 0.1])
@pytest.mark.parametrize("segs", [SEGS_26, [0, 40], [0, 700], [0, 9001]], ids=lambda s: "%dx%d" % (s[-1], len(s) - 1))
def test_pairs_without_a_margin(segs, smoothing):
    """Excluded choices in both tracks, NaN and +inf: the pair has no margin and the loss is NaN, and nothing of it
    reaches the other pairs' ratios and gradients."""
    require_gpu()
    for dtype in ("f32", "bf16"):
        for lens in (SHORT, LONG):
            ptr = _ptr(lens)
            a, b = int(ptr[2]), int(ptr[3])
            for what in ("both", "nan", "inf"):
                def edit(z, acts):
                    for r in (a, b) if what == "both" else (a,):
                        z[r, acts[r, 0]] = {"both": -np.inf, "nan": np.nan, "inf": np.inf}[what]
                R = Rows(dtype, int(ptr[-1]), segs, seed=18, edit=edit)
                cfg = dict(beta=0.2, smoothing=smoothing)
                loss, ratio, dz = run_pref(R, None, None, ptr, cfg)
                assert np.isnan(loss[:3]).all() and np.isfinite(loss[3])
                assert (ratio[2:4] == -np.inf).all() if what == "both" else np.isnan(ratio[2]) and np.isfinite(ratio[3])
                pair = slice(int(ptr[2]), int(ptr[4]))
                assert np.isnan(dz[pair]).all()
                # the other pairs: the same call where the pair's rows are padding
                w = np.ones(R.M, np.float32)
                w[pair] = 0.0
                _, ratio0, dz0 = run_pref(R, None, w, ptr, cfg)
                rest = np.r_[0:pair.start, pair.stop:R.M]
                np.testing.assert_array_equal(dz[rest], dz0[rest])
                np.testing.assert_array_equal(ratio[[0, 1, 4, 5]], ratio0[[0, 1, 4, 5]])


# ------------------------------------------------------------------------------------------------
# the clipped loss: segments, a wave a row, a workgroup a row, rows in chunks
# ------------------------------------------------------------------------------------------------
ROUTES = [(SEGS_26, 130), ([0, 90], 130), ([0, 300], 130), ([0, 4200], 1030), ([0, 9001], 70)]
CFG = dict(clip_low=0.2, clip_high=0.28, w_kl=0.05, w_entropy=0.01)


def _inputs(R, ratios, advs, backs):
    """Every combination of log ratio, advantage and log reference ratio, row after row; weights of 1e-8, some negative."""
    lp = obj.row_stats(R.z, R.segs, R.acts)["logp"]
    i = np.arange(R.M)
    d, a, x = np.array(ratios)[i % len(ratios)], np.array(advs)[i // len(ratios) % len(advs)], np.array(backs)[i // (len(ratios) * len(advs)) % len(backs)]
    w = np.where(i % 11 == 5, -1.0, 1.0) * 1e-8
    f = lambda v: v.astype(np.float32)  # noqa: E731
    return dict(old=f(lp - d), ref=f(lp + x), adv=f(a), w=f(w))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("segs,M", ROUTES, ids=lambda v: str(v) if isinstance(v, int) else "%dx%d" % (v[-1], len(v) - 1))
def test_large_log_ratios(segs, M, dtype):
    """e^89 and more with advantages of 0 and of both signs, and in the KL term: nothing is NaN or infinite that the
    weights leave finite.  A log ratio d of fp32 log-probabilities is off by their rounding, E |logp|, by its own and by
    its product's with log2 e, E |d| each; the exponential and the products by at most 8 E."""
    require_gpu()
    for advs, ratios, backs in (((0.0, 1.3, -0.7), (-100.0, -35.0, 0.1, 35.0, 89.5, 100.0), (-100.0, 0.3, 35.0, 95.0)),
                                ((0.0,), (-100.0, 89.5, 100.0), (0.3,)), ((1.3,), (89.5, 100.0), (-0.2,))):
        log("policy loss: %s M=%d head=%s advantages %s" % (dtype, M, segs[-1:], advs))
        R = Rows(dtype, M, segs, seed=M + 1)
        inp = _inputs(R, ratios, advs, backs)
        c = {k: float(np.float32(v)) for k, v in CFG.items()}
        O = obj.policy_loss(R.z, segs, R.acts, inp["old"], inp["ref"], inp["adv"], inp["w"], **c)
        assert np.isfinite(O["loss"]).all() and np.isfinite(O["dlogits"]).all()
        _, lp_e, H_e = _bars(O["st"], segs)
        w, adv = np.abs(inp["w"].astype(np.float64)), np.abs(inp["adv"].astype(np.float64))
        lp, back = O["logp"], np.exp(inp["ref"] - O["logp"])
        rel = lambda v: lp_e + E * (np.abs(lp) + 2 * np.abs(v) + 8)  # noqa: E731
        # a clipped term does not have the ratio in it
        free = np.minimum(O["ratio"] * inp["adv"], np.clip(O["ratio"], 1 - c["clip_low"], 1 + c["clip_high"]) * inp["adv"]) == O["ratio"] * inp["adv"]
        ds = adv * np.where(free, O["ratio"], 1.3) * rel(lp - inp["old"])
        dk = (back + 1) * rel(inp["ref"] - lp)
        t = [(w * v).sum() + E * abs(x) for v, x in zip((ds, dk, H_e.sum(axis=1) + 4 * E * O["st"]["H"].sum(axis=1)), O["loss"][1:])]
        loss, got_lp, dz = run_loss(R, inp, CFG)
        tol = np.array([t[0] + c["w_kl"] * t[1] + c["w_entropy"] * t[2] + E * abs(O["loss"][0])] + t)
        _close(loss, O["loss"], tol + TINY, "loss")
        _close(got_lp, lp, lp_e + E * np.abs(lp), "logp")
        dg = w * (adv * np.where(free, O["ratio"], 0.0) * rel(lp - inp["old"]) + c["w_kl"] * dk) + 4 * E * np.abs(O["g_logp"])
        _close(dz, O["dlogits"], _grad_bar(O["st"], segs, R.acts, O["g_logp"], O["g_ent"], dg, 2 * E * np.abs(O["g_ent"]),
                                           O["dlogits"], dtype, False), "dlogits")


@pytest.mark.parametrize("segs,M", ROUTES, ids=lambda v: str(v) if isinstance(v, int) else "%dx%d" % (v[-1], len(v) - 1))
def test_advantage_zero_whatever_the_ratio(segs, M):
    """An old log-probability of -inf (the old policy excluded the action) or -1e30: with advantage 0 the row adds
    nothing, as any advantage times 0 would; with another one the loss is infinite."""
    require_gpu()
    for dtype in ("f32", "bf16"):
        R = Rows(dtype, M, segs, seed=M + 2)
        cfg = dict(CFG, w_kl=0.0, w_entropy=0.0)
        inp = _inputs(R, (0.1,), (0.5,), (0.0,))
        inp["w"] = None
        inp["old"][3], inp["old"][4], inp["old"][5] = -np.inf, -1e30, -800.0
        inp["adv"][3:6] = 0.0
        loss, _, dz = run_loss(R, inp, cfg)
        assert np.isfinite(loss).all() and (dz[3:6] == 0).all() and np.isfinite(dz).all()
        rest = dict(inp, old=inp["old"].copy())
        rest["old"][3:6] = rest["old"][0]
        want, _, dz0 = run_loss(R, rest, cfg)
        np.testing.assert_array_equal(loss[[0, 1, 3]], want[[0, 1, 3]])
        # the KL terms, none of them negative, of the three rows are rounded after their weight (E of each), the sums E each
        assert abs(loss[2] - want[2]) <= 3 * E * want[2]
        np.testing.assert_array_equal(dz, dz0)
        inp["adv"][4] = -1.0
        loss, _, dz = run_loss(R, inp, cfg)
        assert loss[0] == np.inf and loss[1] == np.inf and not np.isfinite(dz[4]).all() and np.isfinite(dz[:4]).all()
