"""GPU parity of the policy objectives (harl_policy_logp, harl_policy_logp_grad, harl_policy_loss,
harl_preference_loss) against the fp64 oracle (oracle/objective.py).

Bars, with E = 2^-24 (half a step of fp32) and a segment of n columns summed by at least 64 lanes:
  lse    (its second part; the first, the largest logit, is exact) a sum of n rounded terms: n / 64 additions in a lane and at most 40 joining them; every term an
         exponential good to 2 E whose argument d = z - m is rounded twice, and sum p |d| <= log n:
         E (n / 64 + 40 + 4 + 2 log n), beside the output's own rounding, at most E log n
  logp   the segments' lse errors (the difference to z[action] is formed in fp64) and E |logp|
  H      log s - u / s, u = sum e d: lse's error twice (through s in both terms, the second times E1 = sum p |d|),
         u's terms and additions E ((n / 64 + 44) E1 + 4 E2 + 4 E1), E2 = sum p d^2, and E |H|
  dz     g_logp (hot - p) - g_H p (log p + H): p to r = lse's error + E (log n + 3 (|log p| + log n) + 4), the
         gradients' errors (from logp through the objective's derivative), 4 roundings of every product,
         and half a step of the output's type (bf16: 2^-8 of the value)
  sums   of the rows' errors, and E |sum|
Magnitudes below 2^-126 may become 0."""
from __future__ import annotations

import math

import numpy as np
import pytest

from oracle import objective as obj
from tests.gpu_util import log, require_gpu

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
TINY = 2.0 ** -126
SEGS_26 = [0, 17, 20, 23, 26]
GUARD = 7.25  # in every element of the gradient buffer that no row covers


# ------------------------------------------------------------------------------------------------
# bars
# ------------------------------------------------------------------------------------------------
def _bars(st, segs):
    """Errors of lse [M][n], logp [M] (before its rounding) and H [M][n]."""
    lse_e, H_e = np.zeros_like(st["lse"]), np.zeros_like(st["lse"])
    for s in range(len(segs) - 1):
        lo, hi = segs[s], segs[s + 1]
        n = hi - lo
        p, ls = st["p"][:, lo:hi], np.where(st["p"][:, lo:hi] > 0, st["ls"][:, lo:hi], 0.0)
        d = ls - ls.max(axis=1, keepdims=True, where=st["p"][:, lo:hi] > 0, initial=-np.inf)
        d = np.where(st["p"][:, lo:hi] > 0, d, 0.0)
        E1, E2 = (p * -d).sum(axis=1), (p * d * d).sum(axis=1)
        acc = n / 64 + 40
        e = E * (acc + 4 + 2 * math.log(n))
        lse_e[:, s] = e
        H_e[:, s] = e * (1 + E1) + E * ((acc + 4) * E1 + 4 * E2 + 4 * E1) + E * np.abs(st["H"][:, s])
    return lse_e, lse_e.sum(axis=1), H_e


def _grad_bar(st, segs, acts, g, ge, dg, dge, want, dtype, lse_given):
    lse_e, _, H_e = _bars(st, segs)
    tol = np.zeros_like(want)
    for s in range(len(segs) - 1):
        lo, hi = segs[s], segs[s + 1]
        p = st["p"][:, lo:hi]
        ls = np.where(p > 0, st["ls"][:, lo:hi], 0.0)
        H = st["H"][:, s:s + 1]
        e = lse_e[:, s:s + 1] + E * math.log(hi - lo)  # the second part, at most log n, is rounded; the first is exact
        r = e + E * (3 * (np.abs(ls) + math.log(hi - lo)) + 4)  # z - m may be log n beyond log p
        hot = np.zeros_like(p)
        hot[np.arange(p.shape[0]), np.clip(acts[:, s], lo, hi - 1) - lo] = 1.0
        G, GE, DG, DGE = (np.abs(x)[:, None] for x in (g, ge, dg, dge))
        tol[:, lo:hi] = (G * (p * r + 2 * E * (hot + p)) + DG * np.abs(hot - p) + DGE * p * np.abs(ls + H)
                         + GE * p * (np.abs(ls + H) * (r + 4 * E) + e + 2 * E * np.abs(ls) + H_e[:, s:s + 1] + E * np.abs(H))
                         + (G + GE * (1 + np.abs(ls) + np.abs(H))) * TINY)
    half = 2.0 ** -8 if dtype == "bf16" else E
    return tol * (1 + half) + half * np.abs(want) + 2 * TINY


def _without(st, rows):
    """The statistics with zeros in rows that count for nothing (their bars are 0, not 0 times NaN)."""
    return {k: np.where(rows.reshape((-1,) + (1,) * (v.ndim - 1)), np.zeros_like(v), v) for k, v in st.items()}


def _close(got, want, tol, what):
    got = np.asarray(got, np.float64)
    assert (np.isnan(got) == np.isnan(want)).all(), what + ": NaN where the oracle has none, or none where it has"
    fin = np.isfinite(want)
    assert (got[~fin & ~np.isnan(want)] == want[~fin & ~np.isnan(want)]).all(), what + ": infinities"
    err = np.abs(got[fin] - want[fin])
    tol = np.broadcast_to(tol, want.shape)[fin]
    assert (err <= tol).all(), "%s: %d of %d beyond tolerance, worst %.3g times" % (
        what, int((err > tol).sum()), err.size, float((err / np.maximum(tol, 1e-300)).max()))


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
class Rows:
    """M rows of logits on the device, `off` elements into a buffer and `pad` columns apart, and the same
    values in fp64; gradient rows likewise (`in_place`: the same buffer)."""

    def __init__(self, dtype, M, segs, seed, off=0, pad=0, excl=0.0, scale=2.0, off_d=None, pad_d=None, in_place=False,
                 edit=None):
        import torch
        from paper_2211_11172_amd import harl
        self.dtype, self.M, self.segs, self.a = dtype, M, segs, segs[-1]
        rng = self.rng = np.random.default_rng(seed)
        z = (rng.standard_normal((M, self.a)) * scale).astype(np.float32)
        self.acts = np.stack([rng.integers(lo, hi, M) for lo, hi in zip(segs, segs[1:])], axis=1).astype(np.int32)
        if excl:
            drop = rng.random(z.shape) < excl
            np.put_along_axis(drop, self.acts.astype(np.int64), False, axis=1)
            z[drop] = -np.inf
        if edit:
            edit(z, self.acts)
        td = torch.bfloat16 if dtype == "bf16" else torch.float32
        t = torch.from_numpy(z).to(td)
        self.z = t.to(torch.float64).numpy()
        self.ld, self.ld_d = self.a + pad, self.a + (pad if pad_d is None else pad_d)
        off_d = off if off_d is None else off_d

        def buffer(o, ld):
            b = torch.full((o + M * ld + 16,), GUARD, dtype=td, device="cuda")
            return b, b[o:o + M * ld].view(M, ld)[:, :self.a]

        self.buf, self.logits = buffer(off, self.ld)
        self.logits.copy_(t)
        self.off_d = off_d
        self.gbuf, self.grad = (self.buf, self.logits) if in_place else buffer(off_d, self.ld_d)
        if in_place:
            self.ld_d, self.off_d = self.ld, off
        self.head = harl.policy_head(dtype, self.a, segs)
        self.d_acts = self.dev(self.acts)
        self.torch = torch

    def dev(self, x):
        import torch
        return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()

    def f32(self, *shape):
        return self.torch.full(shape, float("nan"), device="cuda")

    def ws(self, n):
        return self.torch.full((n,), 0xA5, dtype=self.torch.uint8, device="cuda"), n

    def take_grad(self):
        """The gradient rows, after a look that nothing around them was written."""
        b = self.gbuf.to(self.torch.float64).cpu().numpy()
        rows = b[self.off_d:self.off_d + self.M * self.ld_d].reshape(self.M, self.ld_d)
        assert (b[:self.off_d] == GUARD).all() and (b[self.off_d + self.M * self.ld_d:] == GUARD).all()
        assert (rows[:, self.a:] == GUARD).all(), "columns behind a row were written"
        return rows[:, :self.a].copy()


def run_logp(R):
    from paper_2211_11172_amd import harl
    n = len(R.segs) - 1
    lp, H, L = R.f32(R.M), R.f32(R.M, n), R.f32(R.M, n, 2)
    ws, wsb = R.ws(harl.harl_policy_logp_workspace_size(R.head, R.M))
    harl.harl_policy_logp(R.head, R.logits, R.ld, R.M, R.d_acts, lp, H, L, ws, wsb)
    R.torch.cuda.synchronize()
    return lp, H, L


def _top_p(st, segs):
    """The largest probability of every segment: e^(largest logit - lse)."""
    return np.stack([st["p"][:, lo:hi].max(axis=1) for lo, hi in zip(segs, segs[1:])], axis=1)


def check_logp(R, got):
    st = obj.row_stats(R.z, R.segs, R.acts)
    lse_e, lp_e, H_e = _bars(st, R.segs)
    lp, H, L = (x.cpu().numpy() for x in got)
    fin = lambda x: np.where(np.isfinite(x), np.abs(x), 0.0)  # noqa: E731
    _close(L[:, :, 0], st["top"], 0.0, "the largest logit")
    n = np.array(R.segs[1:]) - np.array(R.segs[:-1])
    rest = np.where(st["empty"], 0.0, np.where(np.isfinite(st["lse"]), -np.log(np.maximum(_top_p(st, R.segs), 1e-300)), st["lse"]))
    fine = np.isfinite(st["lse"]) | st["empty"]
    assert np.isnan(L[:, :, 1][~fine]).all()
    _close(L[:, :, 1][fine], rest[fine], (lse_e + E * np.log(n))[fine], "log-sum-exp")
    _close(lp, st["logp"], lp_e + E * fin(st["logp"]) + TINY, "logp")
    _close(H, st["H"], H_e + TINY, "entropy")
    return st


def run_loss(R, inp, cfg, grad=True, want_logp=True):
    from paper_2211_11172_amd import harl
    d = {k: R.dev(None if v is None else v.astype(np.float32)) for k, v in inp.items()}
    lp, loss = R.f32(R.M) if want_logp else None, R.f32(4)
    ws, wsb = R.ws(harl.harl_policy_loss_workspace_size(R.head, R.M))
    harl.harl_policy_loss(R.head, harl.policy_loss_config(**cfg), R.logits, R.ld, R.M, R.d_acts, d["old"], d["ref"], d["adv"],
                          d["w"], R.grad if grad else None, R.ld_d if grad else 0, lp, loss, ws, wsb)
    R.torch.cuda.synchronize()
    return (loss.cpu().numpy(), lp.cpu().numpy() if want_logp else None, R.take_grad() if grad else None)


def loss_inputs(R, cfg, weights=None, ref=True, spread=0.4):
    """Old and reference log-probabilities around the true ones, no ratio near a clip border."""
    rng, lp = R.rng, obj.row_stats(R.z, R.segs, R.acts)["logp"]
    lp = np.where(np.isfinite(lp), lp, -3.0)
    x = rng.uniform(-spread, spread, R.M)
    for b in (math.log1p(-cfg["clip_low"]), math.log1p(cfg["clip_high"])):
        x = np.where(np.abs(x - b) < 5e-3, b + 8e-3, x)
    w = None
    if weights == "some":
        w = np.where(rng.random(R.M) < 0.3, 0.0, rng.uniform(0.1, 1.0, R.M) / R.M)
    f = lambda v: None if v is None else v.astype(np.float32)  # noqa: E731
    return dict(old=f(lp - x), ref=f(lp + 0.3 * rng.standard_normal(R.M)) if ref else None, adv=f(rng.standard_normal(R.M)), w=f(w))


def check_loss(R, inp, cfg, got, dtype_grad=True):
    c = {k: float(np.float32(v)) for k, v in cfg.items()}
    O = obj.policy_loss(R.z, R.segs, R.acts, inp["old"], inp["ref"], inp["adv"], inp["w"], **c)
    w = np.full(R.M, float(np.float32(1.0 / R.M))) if inp["w"] is None else inp["w"].astype(np.float64)
    on = w != 0
    st = _without(O["st"], ~on)
    _, lp_e, H_e = _bars(st, R.segs)
    adv = np.where(on, inp["adv"], 0.0).astype(np.float64)
    back = np.zeros(R.M) if inp["ref"] is None else np.where(on, np.exp(np.where(on, inp["ref"], 0.0) - O["logp"]), 0.0)
    w, H_e = np.where(on, np.abs(w), 0.0), np.where(on[:, None], H_e, 0.0)
    # a row's ratio moves by ratio times logp's error, the KL term by |1 - e^x| times it and its derivative by e^x times it
    ds, dk = np.abs(adv) * O["ratio"] * lp_e, np.abs(1 - back) * lp_e + back * lp_e ** 2
    each = [np.abs(adv) * O["ratio"], back + 1, np.abs(st["H"]).sum(axis=1)]
    t = [(w * (e + 4 * E * a)).sum() for e, a in zip((ds, dk, H_e.sum(axis=1)), each)]
    t = [v + E * abs(x) for v, x in zip(t, O["loss"][1:])]
    loss, lp, dz = got
    _close(loss, O["loss"], np.array([t[0] + c["w_kl"] * t[1] + c["w_entropy"] * t[2] + E * abs(O["loss"][0])] + t) + TINY, "loss")
    if lp is not None:
        _close(lp, O["logp"], lp_e + E * np.abs(O["logp"]) + TINY, "logp")
    if dz is not None:
        dg = w * (np.abs(adv) * O["ratio"] + c["w_kl"] * back) * lp_e + 2 * E * np.abs(O["g_logp"])
        _close(dz, O["dlogits"], _grad_bar(st, R.segs, R.acts, O["g_logp"], O["g_ent"], dg, 2 * E * np.abs(O["g_ent"]), O["dlogits"],
                                           R.dtype, False), "dlogits")
        assert (dz[~on] == 0).all()
    return O


CFG = dict(clip_low=0.2, clip_high=0.28, w_kl=0.05, w_entropy=0.01)

# heads: one column, fewer than a wave, around 16-byte vectors, a row in a wave, a workgroup, several
HEADS = [[0, 1], [0, 2], [0, 7], [0, 26], SEGS_26, [0, 1, 2, 3, 64, 127], list(range(0, 33)), [0, 63], [0, 64], [0, 65], [0, 127],
         [0, 300], [0, 511, 514], [0, 513], [0, 1025, 1028, 1031, 1034], [0, 2048], [0, 2049], [0, 4000, 4096], [0, 4095], [0, 5000]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("segs", HEADS, ids=lambda s: "%dx%d" % (s[-1], len(s) - 1))
def test_logp_and_gradient_heads(segs, dtype):
    """Forward and backward over head layouts, ragged row counts, excluded actions."""
    require_gpu()
    import torch
    from paper_2211_11172_amd import harl
    for M, off, pad, excl in ((1, 0, 0, 0.0), (5, 3, 2, 0.3), (133, 0, 0, 0.1)):
        log("logp: %s M=%d head=%s off=%d pad=%d" % (dtype, M, segs[-1:], off, pad))
        R = Rows(dtype, M, segs, seed=M + segs[-1], off=off, pad=pad, excl=excl)
        lp, H, L = run_logp(R)
        st = check_logp(R, (lp, H, L))
        g, ge = R.rng.standard_normal(M).astype(np.float32), R.rng.standard_normal(M).astype(np.float32)
        g[::7], ge[::7] = 0.0, 0.0
        for gent in (ge, None):
            harl.harl_policy_logp_grad(R.head, R.logits, R.ld, M, R.d_acts, L, H if gent is not None else None, R.dev(g),
                                       R.dev(gent), R.grad, R.ld_d)
            torch.cuda.synchronize()
            e = np.zeros(M) if gent is None else gent.astype(np.float64)
            want = obj.logit_grad(st, segs, R.acts, g.astype(np.float64), e)
            zero = np.zeros(M)
            _close(R.take_grad(), want, _grad_bar(st, segs, R.acts, g.astype(np.float64), e, zero, zero, want, dtype, True), "dlogits")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,segs", [(1, [0, 9]), (1, SEGS_26), (70, SEGS_26), (4096, SEGS_26), (65537, SEGS_26), (3, [0, 511, 514]),
                                    (301, [0, 1025, 1028, 1031, 1034]), (2, [0, 4096]), (1, [0, 50001]), (2, [0, 131072]),
                                    (40, [0, 20011]), (300, [0, 4097]), (515, [0, 700]), (2500, [0, 515])],
                         ids=lambda v: str(v) if isinstance(v, int) else "%dx%d" % (v[-1], len(v) - 1))
def test_policy_loss(M, segs, dtype):
    require_gpu()
    for kw, weights, ref, off, pad in ((CFG, "some", True, 0, 0), (dict(CFG, w_kl=0.0, w_entropy=0.0), None, False, 1, 3)):
        if M > 10000 and pad:
            pad = 0
        log("policy loss: %s M=%d head=%s off=%d pad=%d" % (dtype, M, segs[-1:], off, pad))
        R = Rows(dtype, M, segs, seed=M * 3 + segs[-1], off=off, pad=pad, excl=0.05)
        inp = loss_inputs(R, kw, weights, ref)
        check_loss(R, inp, kw, run_loss(R, inp, kw))


@pytest.mark.parametrize("segs,M", [(SEGS_26, 300), ([0, 3001], 9), ([0, 700], 600), ([0, 40001], 3), ([0, 40001], 600)])
def test_policy_loss_outputs_are_optional_and_layouts_agree(segs, M):
    """Without gradient, loss or logp the others are bit-identical; so are the results in place, and with a
    gradient of another alignment than the logits."""
    require_gpu()
    for dtype in ("f32", "bf16"):
        R = Rows(dtype, M, segs, seed=5, off=0, pad=0)
        inp = loss_inputs(R, CFG, "some")
        want = run_loss(R, inp, CFG)
        again = run_loss(R, inp, CFG)
        for x, y in zip(want, again):
            np.testing.assert_array_equal(x, y)
        loss, lp, none = run_loss(R, inp, CFG, grad=False)
        assert none is None
        np.testing.assert_array_equal(loss, want[0])
        np.testing.assert_array_equal(lp, want[1])
        np.testing.assert_array_equal(run_loss(R, inp, CFG, want_logp=False)[2], want[2])
        # other alignments sum in another order: the oracle's bars, not the bits
        for kw in (dict(off=1, pad=1, off_d=0, pad_d=0), dict(off=3, pad=5, off_d=2, pad_d=3), dict(off=1, pad=2, in_place=True)):
            R2 = Rows(dtype, M, segs, seed=5, **kw)
            check_loss(R2, inp, CFG, run_loss(R2, inp, CFG))
        R3 = Rows(dtype, M, segs, seed=5, in_place=True)
        for x, y in zip(want, run_loss(R3, inp, CFG)):
            np.testing.assert_array_equal(x, y)


@pytest.mark.parametrize("segs,M", [(SEGS_26, 40), ([0, 300], 40), ([0, 9001], 40), ([0, 9001], 2000)])
def test_padding_rows_are_not_read(segs, M):
    """NaN in every value of rows of weight 0."""
    require_gpu()
    for dtype in ("f32", "bf16"):
        def edit(z, acts):
            z[::3] = np.nan
        R = Rows(dtype, M, segs, seed=8, edit=edit)
        inp = loss_inputs(R, CFG)
        w = R.rng.uniform(0.1, 1.0, M).astype(np.float32)
        w[::3] = 0.0
        inp["w"] = w
        for k in ("old", "ref", "adv"):
            inp[k][::3] = np.nan
        got = run_loss(R, inp, CFG)
        assert np.isfinite(got[0]).all() and np.isfinite(got[1]).all() and np.isfinite(got[2]).all()
        check_loss(R, inp, CFG, got)


def test_all_rows_padding():
    require_gpu()
    for segs in (SEGS_26, [0, 40001]):
        R = Rows("bf16", 5, segs, seed=2, edit=lambda z, a: z.fill(np.nan))
        inp = dict(old=np.full(5, np.nan, np.float32), ref=None, adv=np.full(5, np.nan, np.float32), w=np.zeros(5, np.float32))
        loss, lp, dz = run_loss(R, inp, dict(CFG, w_kl=0.0))
        assert (loss == 0).all() and (lp == 0).all() and (dz == 0).all()


@pytest.mark.parametrize("segs", [SEGS_26, [0, 26], [0, 3, 700], [0, 9000], [0, 70001]], ids=lambda s: "%dx%d" % (s[-1], len(s) - 1))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_infinities_and_nan(segs, dtype):
    """Empty segments, one action left, the type's lowest value as a mask, logits far from 0, NaN, +inf, an
    excluded action that was chosen, actions outside their segment."""
    require_gpu()
    low = float(np.finfo(np.float32).min) if dtype == "f32" else -3.3895313892515355e38
    a0, a1 = segs[0], segs[1]

    def edit(z, acts):
        z[0] = -np.inf                               # every segment empty
        z[1, a0:a1] = -np.inf                        # the first one empty
        z[2, a0:a1] = -np.inf                        # one action left, and chosen
        z[2, a0] = 1.5
        acts[2, 0] = a0
        z[3, a0:a1:2] = low                          # masked by the lowest value
        z[4] = low                                   # wholly so: uniform
        z[5] += 3000.0
        z[6] -= 20000.0
        z[7, (a0 + a1) // 2] = np.nan
        z[8, a1 - 1] = np.inf
        if a1 - a0 > 1:
            z[9, a0] = -np.inf                       # excluded and chosen
            acts[9, 0] = a0
        acts[10], acts[11] = -5, 1 << 30             # clamped
        z[12] = 0.0
    R = Rows(dtype, 16, segs, seed=11, edit=edit)
    got = run_logp(R)
    st = check_logp(R, got)
    assert got[0][0].item() == 0 and (got[1][0] == 0).all()
    assert (got[2][0, :, 0] == -np.inf).all() and (got[2][0, :, 1] == 0).all()
    clamped = np.clip(R.acts, np.array(segs[:-1]), np.array(segs[1:]) - 1)
    keep = np.ones(16, bool)
    keep[[7, 8, 9]] = False                          # rows whose results are not finite
    for w_kl in (0.0, 0.05):
        kw = dict(CFG, w_kl=w_kl)
        inp = loss_inputs(R, kw)
        inp["w"] = np.where(keep, 0.25, 0.0).astype(np.float32)
        check_loss(R, inp, kw, run_loss(R, inp, kw))
        # the rows that are not finite, each alone: they make the loss what the formula says
        for r in (7, 8, 9):
            w = np.zeros(16, np.float32)
            w[r] = 1.0
            inp["w"] = w
            loss, lp, dz = run_loss(R, inp, kw)
            rest = np.arange(16) != r
            assert (dz[rest] == 0).all() and (lp[rest] == 0).all()
            if r < 9 or a1 - a0 == 1:
                continue
            adv = float(inp["adv"][9])  # ratio 0: -min(0 A, (1 - clip_low) A)
            assert lp[9] == -np.inf and loss[2] == np.inf
            assert abs(loss[1] - max(0.0, -(1 - float(np.float32(0.2))) * adv)) <= 4 * E * abs(adv)
            assert loss[0] == np.inf if w_kl else np.isfinite(loss[0])
    nan = np.isnan(st["logp"])
    assert nan[7] and nan[8] and nan.sum() == 2
    assert (clamped[10] == np.array(segs[:-1])).all()


# ------------------------------------------------------------------------------------------------
# preference loss
# ------------------------------------------------------------------------------------------------
def run_pref(R, ref, w, ptr, cfg, grad=True):
    from paper_2211_11172_amd import harl
    P = (len(ptr) - 1) // 2
    ratio, loss = R.f32(2 * P), R.f32(4)
    ws, wsb = R.ws(harl.harl_preference_loss_workspace_size(R.head, R.M, P))
    d_ptr = R.dev(np.asarray(ptr, np.int32))
    harl.harl_preference_loss(R.head, harl.preference_config(**cfg), R.logits, R.ld, R.M, R.d_acts, R.dev(ref), R.dev(w), d_ptr, P,
                              R.grad if grad else None, R.ld_d if grad else 0, ratio, loss, ws, wsb)
    R.torch.cuda.synchronize()
    return loss.cpu().numpy(), ratio.cpu().numpy(), R.take_grad() if grad else None


def check_pref(R, ref, w, ptr, cfg, got):
    c = {k: float(np.float32(v)) for k, v in cfg.items()}
    O = obj.preference_loss(R.z, R.segs, R.acts, ref, w, ptr, **c)
    P = (len(ptr) - 1) // 2
    wt = np.ones(R.M) if w is None else np.abs(w.astype(np.float64))
    st = _without(O["st"], wt == 0)
    _, lp_e, _ = _bars(st, R.segs)
    row_e = np.where(wt != 0, wt * lp_e, 0.0)
    R_e = np.array([row_e[ptr[q]:ptr[q + 1]].sum() for q in range(2 * P)])
    h_e = c["beta"] * (R_e[0::2] + R_e[1::2]) + 1e-13
    assert (np.abs(O["h"]) > h_e)[O["h"] != 0].all()  # whether h > 0 is not in doubt
    loss, ratio, dz = got
    _close(ratio, O["ratio"], R_e + E * np.abs(O["ratio"]) + TINY, "ratio")
    _close(loss, O["loss"], np.array([h_e.mean()] * 3 + [0.0]) + E * np.abs(O["loss"]) + TINY, "loss")
    if dz is None:
        return O
    dg = np.zeros(R.M)
    for q in range(2 * P):
        dg[ptr[q]:ptr[q + 1]] = c["beta"] / (4 * P) * h_e[q // 2]
    dg = wt * dg + 2 * E * np.abs(O["g_logp"])
    zero = np.zeros(R.M)
    tol = _grad_bar(st, R.segs, R.acts, O["g_logp"], zero, dg, zero, O["dlogits"], R.dtype, False)
    ins = O["inside"]
    _close(dz[ins], O["dlogits"][ins], tol[ins], "dlogits")
    return O


def _ptr(rng, P, longest, before=0, empties=True):
    n = rng.integers(0 if empties else 1, longest + 1, 2 * P)
    return np.concatenate([[before], before + np.cumsum(n)]).astype(np.int64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("segs,P,longest", [(SEGS_26, 1, 1), (SEGS_26, 300, 20), ([0, 5], 3, 700), ([0, 700], 9, 40), ([0, 1025, 1034], 5, 30),
                                            ([0, 4097], 2, 100), ([0, 32768], 2, 16), ([0, 20011], 16, 33), ([0, 131072], 1, 3),
                                            ([0, 9001], 30, 60)], ids=lambda v: str(v) if isinstance(v, int) else "%dx%d" % (v[-1], len(v) - 1))
def test_preference_loss(segs, P, longest, dtype):
    require_gpu()
    for before, behind, weights, smoothing, off, pad in ((0, 0, False, 0.0, 0, 0), (3, 5, True, 0.1, 1, 1)):
        rng = np.random.default_rng(P * longest + before)
        ptr = _ptr(rng, P, longest, before, empties=P > 1)
        N = int(ptr[-1]) + behind
        log("preference loss: %s pairs=%d rows=%d head=%s" % (dtype, P, N, segs[-1:]))
        R = Rows(dtype, max(N, 1), segs, seed=N, off=off, pad=pad, excl=0.02)
        lp = obj.row_stats(R.z, segs, R.acts)["logp"]
        ref = (lp + 0.4 * rng.standard_normal(R.M)).astype(np.float32)
        w = np.where(rng.random(R.M) < 0.3, 0.0, rng.uniform(0.5, 1.5, R.M)).astype(np.float32) if weights else None
        before_rows = R.gbuf.clone()
        cfg = dict(beta=0.3, smoothing=smoothing)
        O = check_pref(R, ref, w, ptr, cfg, run_pref(R, ref, w, ptr, cfg))
        # rows outside every track keep their bytes
        g = R.gbuf[R.off_d:R.off_d + R.M * R.ld_d].view(R.M, R.ld_d)
        old = before_rows[R.off_d:R.off_d + R.M * R.ld_d].view(R.M, R.ld_d)
        out = R.dev(~O["inside"])
        assert R.torch.equal(g[out], old[out])


def test_preference_loss_edges():
    """No rows at all, only empty tracks, every row padding with NaN, missing reference, extreme margins, and
    results that do not depend on the gradient being asked for."""
    require_gpu()
    import torch
    from paper_2211_11172_amd import harl
    for segs in (SEGS_26, [0, 9001]):
        head = harl.policy_head("f32", segs[-1], segs)
        loss, ratio = torch.full((4,), 9.0, device="cuda"), torch.full((6,), 9.0, device="cuda")
        ptr = torch.zeros(7, dtype=torch.int32, device="cuda")
        wsb = harl.harl_preference_loss_workspace_size(head, 0, 3)
        ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
        harl.harl_preference_loss(head, harl.preference_config(0.1), None, 0, 0, None, None, None, ptr, 3, None, 0, ratio, loss, ws, wsb)
        np.testing.assert_allclose(loss.cpu().numpy(), [math.log(2), math.log(2), 0, 0], rtol=2 * E)
        assert (ratio == 0).all()
        R = Rows("bf16", 7, segs, seed=1)
        cfg = dict(beta=0.5, smoothing=0.0)
        ptr = [2, 2, 2, 5, 5]                                     # a pair of empty tracks, a track against nothing
        got = run_pref(R, None, None, ptr, cfg)
        check_pref(R, None, None, ptr, cfg, got)
        bare = run_pref(R, None, None, ptr, cfg, grad=False)
        np.testing.assert_array_equal(bare[0], got[0])
        np.testing.assert_array_equal(bare[1], got[1])
        N = Rows("f32", 6, segs, seed=1, edit=lambda z, a: z.fill(np.nan))
        w = np.zeros(6, np.float32)
        loss, ratio, dz = run_pref(N, np.full(6, np.nan, np.float32), w, [0, 2, 3, 3, 6], cfg)
        assert (ratio == 0).all() and (dz == 0).all()
        np.testing.assert_allclose(loss, [math.log(2), math.log(2), 0, 0], rtol=2 * E)
        X = Rows("f32", 4, segs, seed=3)
        lp = obj.row_stats(X.z, segs, X.acts)["logp"]
        ref = (lp + np.array([-2000.0, 2000.0, 2000.0, -2000.0])).astype(np.float32)
        for cfg in (dict(beta=1.0, smoothing=0.0), dict(beta=1.0, smoothing=0.2)):
            check_pref(X, ref, None, [0, 1, 2, 3, 4], cfg, run_pref(X, ref, None, [0, 1, 2, 3, 4], cfg))


def test_preference_loss_in_place_and_misaligned():
    require_gpu()
    for segs in (SEGS_26, [0, 5003]):
        for dtype in ("f32", "bf16"):
            for kw in (dict(in_place=True), dict(off=1, pad=1, off_d=2, pad_d=5), dict(off=5, pad=3, in_place=True)):
                R = Rows(dtype, 50, segs, seed=4, **kw)
                ptr = [0, 7, 19, 20, 50]
                check_pref(R, None, None, ptr, dict(beta=0.2, smoothing=0.05), run_pref(R, None, None, ptr, dict(beta=0.2, smoothing=0.05)))


# ------------------------------------------------------------------------------------------------
# offsets beyond 32 bits, broken device data, streams, graphs
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("segs", [SEGS_26, [0, 3001], [0, 70001]], ids=lambda s: "%dx%d" % (s[-1], len(s) - 1))
def test_rows_beyond_32_bits(segs):
    """The last of 4 rows starts 4.8e9 elements into the buffer."""
    require_gpu()
    import torch
    R = Rows("bf16", 4, segs, seed=21)
    ld = 1_600_000_003
    big = torch.empty(3 * ld + segs[-1] + 8, dtype=torch.bfloat16, device="cuda")
    rows = torch.as_strided(big, (4, segs[-1]), (ld, 1))
    rows.copy_(R.logits)
    inp = loss_inputs(R, CFG)
    from paper_2211_11172_amd import harl
    d = {k: R.dev(v) for k, v in inp.items()}
    lp, loss = R.f32(4), R.f32(4)
    ws, wsb = R.ws(harl.harl_policy_loss_workspace_size(R.head, 4))
    harl.harl_policy_loss(R.head, harl.policy_loss_config(**CFG), rows, ld, 4, R.d_acts, d["old"], d["ref"], d["adv"], None, rows, ld,
                          lp, loss, ws, wsb)
    torch.cuda.synchronize()
    check_loss(R, inp, CFG, (loss.cpu().numpy(), lp.cpu().numpy(), rows.double().cpu().numpy()))


@pytest.mark.parametrize("segs", [SEGS_26, [0, 5003]])
def test_track_bounds_out_of_order_stay_inside(segs):
    """Bounds that break the precondition give wrong numbers at most: nothing outside the rows is written
    (the bounds are clamped on the device), and the call after it is right."""
    require_gpu()
    R = Rows("f32", 12, segs, seed=6, off=4, pad=2)
    for ptr in ([0, 20, -3, 7, 100], [9, 4, 2, 1, 0], [-8, -7, -6, -5, -4], [50, 60, 70, 80, 90]):
        run_pref(R, None, None, np.array(ptr), dict(beta=0.1, smoothing=0.0))
    ptr = [0, 3, 6, 6, 12]
    check_pref(R, None, None, ptr, dict(beta=0.1, smoothing=0.0), run_pref(R, None, None, ptr, dict(beta=0.1, smoothing=0.0)))


def _session(torch, M=2048, seed=7):
    """The calls as a session makes them: the actor's logits, sampled actions, their log-probabilities, the
    tracks' advantages, the clipped loss, and a preference between tracks."""
    from paper_2211_11172_amd import harl
    from synth import gen_policy, gen_states, gen_track_step, get_config
    cfg = get_config("standard").with_(pol_a=26, n_prog=M)
    s = dict(M=M, a=26, segs=np.array(SEGS_26, np.int32), pol=harl.harl_policy_create(gen_policy(cfg)))
    d = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    s["states"] = d(gen_states(cfg).astype(np.float32))
    s["track"] = {k: d(v) for k, v in gen_track_step(cfg, n=M).items()}
    f = lambda *n: torch.zeros(*n, device="cuda")  # noqa: E731
    s.update(action=torch.zeros(M, dtype=torch.int32, device="cuda"), value=f(M), logits=f(M, 26), old=f(M), entropy=f(M, 4), lse=f(M, 4, 2),
             pick=torch.zeros(M, 4, dtype=torch.int32, device="cuda"), pick_logp=f(M, 4), reward=f(M), adv=f(M), dz=f(M, 26),
             new=f(M), loss=f(4), dz2=f(M, 26), ratio=f(2 * (M // 40)), ploss=f(4))
    s["ptr"] = d(np.arange(0, M // 40 * 40 + 1, 20).astype(np.int32))
    s["head"] = harl.policy_head("f32", 26, SEGS_26)
    s["cfg"], s["pcfg"] = harl.policy_loss_config(0.2, 0.2, 0.0, 0.01), harl.preference_config(0.1)
    n = max(harl.harl_policy_logp_workspace_size(s["head"], M), harl.harl_policy_loss_workspace_size(s["head"], M),
            harl.harl_preference_loss_workspace_size(s["head"], M, M // 40))
    s["ws"], s["wsb"] = torch.empty(n, dtype=torch.uint8, device="cuda"), n
    s["outs"] = [s[k] for k in ("logits", "pick", "old", "entropy", "lse", "adv", "dz", "new", "loss", "dz2", "ratio", "ploss")]

    def run(stream=None):
        t, ws = s["track"], (s["ws"], s["wsb"])
        harl.harl_policy_step(s["pol"], s["states"], M, s["action"], s["value"], None, s["logits"], stream)
        harl.harl_policy_select(s["logits"], M, 26, s["segs"], harl.HARL_SELECT_SAMPLE, 11, seed, s["pick"], s["pick_logp"], None, stream)
        harl.harl_policy_logp(s["head"], s["logits"], 26, M, s["pick"], s["old"], s["entropy"], s["lse"], *ws, stream)
        harl.harl_track_advantage(t["c_prev"], t["c_next"], t["v_prev"], t["v_next"], M, 0.9, 1e-6, s["reward"], s["adv"], stream)
        harl.harl_policy_loss(s["head"], s["cfg"], s["logits"], 26, M, s["pick"], s["old"], None, s["adv"], None, s["dz"], 26, s["new"],
                              s["loss"], *ws, stream)
        harl.harl_preference_loss(s["head"], s["pcfg"], s["logits"], 26, M, s["pick"], None, None, s["ptr"], M // 40, s["dz2"], 26,
                                  s["ratio"], s["ploss"], *ws, stream)
    s["run"] = run
    return s


def test_session_of_calls():
    """The calls together: the log-probabilities are the selection's, the losses the oracle's, and with
    ratio 1 the clipped loss is harl_ppo_update's surrogate and entropy on the same network."""
    require_gpu()
    import torch
    s = _session(torch)
    s["run"]()
    torch.cuda.synchronize()
    z, acts = s["logits"].cpu().numpy().astype(np.float64), s["pick"].cpu().numpy()
    old = s["old"].cpu().numpy()
    np.testing.assert_allclose(old, s["pick_logp"].sum(1).cpu().numpy(), atol=4e-6)
    adv = s["adv"].cpu().numpy()
    f = lambda x: float(np.float32(x))  # noqa: E731
    O = obj.policy_loss(z, SEGS_26, acts, old, None, adv, None, f(0.2), f(0.2), 0.0, f(0.01))
    np.testing.assert_allclose(s["loss"].cpu().numpy(), O["loss"], rtol=1e-5, atol=1e-7)
    np.testing.assert_allclose(s["dz"].cpu().numpy(), O["dlogits"], atol=1e-6 * np.abs(O["dlogits"]).max())
    np.testing.assert_array_equal(s["new"].cpu().numpy(), old)
    P = obj.preference_loss(z, SEGS_26, acts, None, None, s["ptr"].cpu().numpy(), f(0.1))
    np.testing.assert_allclose(s["ploss"].cpu().numpy(), P["loss"], rtol=1e-5, atol=1e-6)
    n = s["ptr"].numel() // 2 * 40
    np.testing.assert_allclose(s["dz2"].cpu().numpy()[:n], P["dlogits"][:n], atol=1e-6 * np.abs(P["dlogits"]).max())
    assert (s["dz2"][n:] == 0).all()  # as it was
    s["pol"].close()


def test_matches_the_ppo_update_of_the_librarys_network():
    """harl_ppo_update's loss terms on its own network equal harl_policy_loss's on that network's logits."""
    require_gpu()
    import torch
    from oracle import ppo
    from paper_2211_11172_amd import harl
    from tests.test_gpu_ppo import SEGS, _gpu_update, _setup
    dims, M = (64, 256, 256, 26), 1000
    flat, batch = _setup(M, dims, seed=3)
    up = _gpu_update(flat, batch, dims, SEGS)[0]
    L = ppo.loss(ppo.unpack(flat.astype(np.float64), *dims), batch, SEGS)
    R = Rows("f32", M, SEGS, seed=0, edit=lambda z, a: (np.copyto(z, L["fwd"]["logits"]), np.copyto(a, batch["actions"])))
    cfg = dict(clip_low=0.2, clip_high=0.2, w_kl=0.0, w_entropy=0.01)
    loss, _, _ = run_loss(R, dict(old=batch["logp_old"], ref=None, adv=batch["adv"], w=None), cfg)
    np.testing.assert_allclose(loss[[1, 3]], up["loss"][[1, 3]], rtol=1e-4, atol=1e-6)


@pytest.mark.parametrize("wide", [False, True])
def test_graph_replay_and_side_stream(wide):
    """Captured calls replay to the eager results, replay after replay, and give them on another stream."""
    require_gpu()
    import torch
    if wide:
        from paper_2211_11172_amd import harl
        R = Rows("bf16", 6, [0, 70001], seed=3)
        inp = {k: R.dev(v) for k, v in loss_inputs(R, CFG).items()}
        lp, loss, lp2, H, L = R.f32(6), R.f32(4), R.f32(6), R.f32(6), R.f32(6, 2)
        ratio, ploss, g2 = R.f32(2), R.f32(4), torch.zeros_like(R.grad).contiguous()
        ptr = R.dev(np.array([0, 2, 6], np.int32))
        n = max(harl.harl_policy_loss_workspace_size(R.head, 6), harl.harl_policy_logp_workspace_size(R.head, 6),
                harl.harl_preference_loss_workspace_size(R.head, 6, 1))
        ws, wsb = R.ws(n)
        outs = [lp, loss, lp2, H, L, ratio, ploss, g2, R.gbuf]

        def run(stream=None):
            harl.harl_policy_logp(R.head, R.logits, R.ld, 6, R.d_acts, lp2, H, L, ws, wsb, stream)
            harl.harl_policy_loss(R.head, harl.policy_loss_config(**CFG), R.logits, R.ld, 6, R.d_acts, inp["old"], inp["ref"], inp["adv"],
                                  None, R.grad, R.ld_d, lp, loss, ws, wsb, stream)
            harl.harl_preference_loss(R.head, harl.preference_config(0.1), R.logits, R.ld, 6, R.d_acts, inp["ref"], None, ptr, 1, g2,
                                      R.a, ratio, ploss, ws, wsb, stream)
    else:
        s = _session(torch)
        run, outs = s["run"], s["outs"]
    run()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    for o in outs:
        o.zero_()
    torch.cuda.synchronize()
    run(side)
    side.synchronize()
    first = [o.clone() for o in outs]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for rep in range(4):
        for o in outs:
            o.zero_()
        junk = torch.randn(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for i, (o, w) in enumerate(zip(outs, first)):
            assert torch.equal(o.view(torch.uint8), w.view(torch.uint8)), "replay %d differs in output %d" % (rep, i)
        del junk
    for i, (o, w) in enumerate(zip(first, want)):  # bytes that no call writes were 0 in one and not in the other
        if o is not (R.gbuf if wide else None) and not (wide and i == len(outs) - 1):
            assert torch.equal(o.view(torch.uint8), w.view(torch.uint8)), "the side stream differs in output %d" % i
