"""Policy objectives over the whole range of their inputs: chosen actions that are excluded, and rows that are not
finite, in the preference loss."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import objective as obj
from tests.gpu_util import log, require_gpu
from tests.test_gpu_objective import SEGS_26, Rows, _close, check_pref, run_pref

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
