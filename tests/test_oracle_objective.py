"""Pins of the fp64 oracle of the policy objectives (oracle/objective.py): closed forms, central
differences of every objective at every logit, and the PPO oracle's surrogate and entropy terms."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import objective as obj
from oracle import ppo

SEGS = [0, 5, 8, 9]


def _rows(seed, M=7, segs=SEGS, excl=0.0):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((M, segs[-1])) * 1.5
    acts = np.stack([rng.integers(a, b, M) for a, b in zip(segs, segs[1:])], axis=1)
    if excl:
        drop = rng.random(z.shape) < excl
        np.put_along_axis(drop, acts, False, axis=1)
        z[drop] = -np.inf
    return rng, z, acts


def _central(f, z, h=1e-6):
    d = np.zeros_like(z)
    for i in np.ndindex(z.shape):
        if not np.isfinite(z[i]):
            continue
        p, m = z.copy(), z.copy()
        p[i] += h
        m[i] -= h
        d[i] = (f(p) - f(m)) / (2 * h)
    return d


def test_uniform_rows_and_closed_forms():
    z = np.zeros((3, 9))
    st = obj.row_stats(z, SEGS, np.array([[0, 5, 8]] * 3))
    np.testing.assert_allclose(st["logp"], -np.log(5) - np.log(3), rtol=1e-14)
    np.testing.assert_allclose(st["H"], [[np.log(5), np.log(3), 0.0]] * 3, atol=1e-15)
    # ratio 1: the surrogate is the mean advantage, the KL term 0; x = log 2 gives 2 - log 2 - 1
    adv = np.array([1.0, -2.0, 4.0])
    L = obj.policy_loss(z, SEGS, [[0, 5, 8]] * 3, st["logp"], st["logp"] + np.log(2), adv, w_kl=1.0)
    np.testing.assert_allclose(L["loss"], [-1.0 + 1 - np.log(2), -1.0, 1 - np.log(2), np.log(15)], rtol=1e-14)
    # equal tracks: log 2, and the gradient of h is -beta/2 a pair
    P = obj.preference_loss(z[:2], SEGS, [[0, 5, 8]] * 2, None, None, [0, 1, 2], beta=0.3)
    np.testing.assert_allclose(P["loss"], [np.log(2), np.log(2), 0.0, 0.0], rtol=1e-14)
    np.testing.assert_allclose(P["g_logp"], [-0.15, 0.15], rtol=1e-14)


def test_empty_and_excluded():
    rng, z, acts = _rows(1, excl=0.4)
    z[0, 0:5] = -np.inf
    st = obj.row_stats(z, SEGS, acts)
    assert np.isfinite(st["logp"]).all() and st["H"][0, 0] == 0 and st["lse"][0, 0] == -np.inf
    d = obj.logit_grad(st, SEGS, acts, np.ones(7), np.ones(7))
    assert (d[~np.isfinite(z)] == 0).all() and np.isfinite(d).all()
    for a, b in zip(SEGS, SEGS[1:]):  # a segment's gradient sums to 0
        np.testing.assert_allclose(d[:, a:b].sum(axis=1), 0.0, atol=1e-14)


@pytest.mark.parametrize("excl", [0.0, 0.3])
@pytest.mark.parametrize("w_kl,w_ent,weights", [(0.0, 0.0, False), (0.3, 0.0, True), (0.2, 0.05, True)])
def test_policy_loss_gradient_is_the_central_difference(excl, w_kl, w_ent, weights):
    rng, z, acts = _rows(2, excl=excl)
    lp = obj.row_stats(z, SEGS, acts)["logp"]
    old, ref, adv = lp + rng.uniform(-0.5, 0.5, 7), lp + rng.uniform(-1, 1, 7), rng.standard_normal(7)
    w = np.array([0.0, 0.1, 0.3, 0.0, 0.2, 0.2, 0.2]) if weights else None
    kw = dict(clip_low=0.2, clip_high=0.3, w_kl=w_kl, w_entropy=w_ent)
    L = obj.policy_loss(z, SEGS, acts, old, ref, adv, w, **kw)
    assert (np.abs(L["ratio"] - 0.8) > 1e-4).all() and (np.abs(L["ratio"] - 1.3) > 1e-4).all()
    f = lambda x: obj.policy_loss(x, SEGS, acts, old, ref, adv, w, **kw)["loss"][0]  # noqa: E731
    np.testing.assert_allclose(L["dlogits"], _central(f, z), atol=2e-9)


@pytest.mark.parametrize("smoothing", [0.0, 0.1])
def test_preference_gradient_is_the_central_difference(smoothing):
    rng, z, acts = _rows(3, M=11, excl=0.2)
    ptr = [1, 4, 4, 5, 9]  # an empty track; rows before the first and behind the last
    ref, w = rng.standard_normal(11) * 0.3 - 3, np.array([1, 1, 0, 2, 1, 1, 0.5, 1, 1, 1, 1])
    kw = dict(beta=0.4, smoothing=smoothing)
    L = obj.preference_loss(z, SEGS, acts, ref, w, ptr, **kw)
    f = lambda x: obj.preference_loss(x, SEGS, acts, ref, w, ptr, **kw)["loss"][0]  # noqa: E731
    np.testing.assert_allclose(L["dlogits"], _central(f, z), atol=2e-9)
    assert (L["dlogits"][[0, 2, 9, 10]] == 0).all()


def test_logp_gradient_is_the_central_difference():
    rng, z, acts = _rows(4, excl=0.2)
    gl, ge = rng.standard_normal(7), rng.standard_normal(7)

    def f(x):
        st = obj.row_stats(x, SEGS, acts)
        return (gl * st["logp"]).sum() + (ge * st["H"].sum(axis=1)).sum()

    np.testing.assert_allclose(obj.logit_grad(obj.row_stats(z, SEGS, acts), SEGS, acts, gl, ge), _central(f, z), atol=2e-8)


def test_surrogate_and_entropy_agree_with_the_ppo_oracle():
    """With weights 1/M and no KL term the loss is the PPO oracle's without its value term, and the
    gradient at the logits chains to its actor-head gradient."""
    rng = np.random.default_rng(5)
    dims, segs, M = (4, 6, 5, 9), SEGS, 13
    p = {k: rng.standard_normal(s) * 0.5 for k, s in ppo.param_shapes(*dims).items()}
    acts = np.stack([rng.integers(a, b, M) for a, b in zip(segs, segs[1:])], axis=1)
    batch = dict(states=rng.standard_normal((M, 4)), actions=acts, logp_old=rng.uniform(-4, -2, M),
                 adv=rng.standard_normal(M), ret=rng.standard_normal(M))
    g, L = ppo.grads(p, batch, segs, w_v=0.0)
    O = obj.policy_loss(L["fwd"]["logits"], segs, acts, batch["logp_old"], None, batch["adv"], w_entropy=0.01)
    np.testing.assert_allclose([O["loss"][0], O["loss"][1], O["loss"][3]], [L["total"], L["clip"], L["entropy"]], rtol=1e-12)
    np.testing.assert_allclose(O["dlogits"].T @ L["fwd"]["h2"], g["wa"], atol=1e-14)


@pytest.mark.parametrize("mistake", ["sign_kl", "no_weight", "other_track", "open_clip"])
def test_differences_would_show_a_mistake(mistake):
    """The central differences above are far from a gradient with one of these mistakes."""
    rng, z, acts = _rows(6)
    lp = obj.row_stats(z, SEGS, acts)["logp"]
    old, ref, adv, w = lp - 0.4, lp + 0.7, np.abs(rng.standard_normal(7)), rng.uniform(0.1, 1, 7)
    if mistake == "other_track":
        L = obj.preference_loss(z[:4], SEGS, acts[:4], None, None, [0, 2, 4], beta=0.5)
        f = lambda x: obj.preference_loss(x, SEGS, acts[:4], None, None, [0, 2, 4], beta=0.5)["loss"][0]  # noqa: E731
        bad = obj.logit_grad(L["st"], SEGS, acts[:4], -L["g_logp"], np.zeros(4))
        assert np.abs(bad - _central(f, z[:4])).max() > 1e-3
        return
    kw = dict(w_kl=0.2, w_entropy=0.0)
    L = obj.policy_loss(z, SEGS, acts, old, ref, adv, w, **kw)
    g = {"sign_kl": w * (-adv * L["ratio"] * 0 + 0.2 * np.expm1(ref - lp)), "no_weight": L["g_logp"] / w,
         "open_clip": w * (-adv * L["ratio"] - 0.2 * np.expm1(ref - lp))}[mistake]
    f = lambda x: obj.policy_loss(x, SEGS, acts, old, ref, adv, w, **kw)["loss"][0]  # noqa: E731
    assert np.abs(obj.logit_grad(L["st"], SEGS, acts, g, np.zeros(7)) - _central(f, z)).max() > 1e-3
