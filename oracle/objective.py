"""TEST INFRASTRUCTURE: the fp64 oracle of the policy objectives on an actor's logits.

Log-probabilities of chosen actions over segments (modification types), the clipped policy loss of
Schulman et al., "Proximal Policy Optimization Algorithms" (2017), with an entropy bonus and a KL
term to a reference policy (the estimator e^x - x - 1, x = logp_ref - logp, which is unbiased under
the policy's own samples and never negative), and the preference loss of paired log ratios of
Rafailov et al., "Direct Preference Optimization" (NeurIPS'23), with label smoothing.  Conventions:

  - a logit of -inf is an excluded action (probability 0, gradient 0 unless it was chosen); a segment of
    nothing but -inf adds 0 to log-probability and entropy and has gradient 0;
  - a row of weight 0 is padding: none of its values counts, its gradient is 0;
  - min passes the gradient to the unclipped term on equality, clip inside its closed range.

Only tests/ uses this module.
"""
from __future__ import annotations

import numpy as np


def row_stats(z, segs, actions) -> dict:
    """Joint log-probability [M], entropies, log-sum-exps and largest logits [M][n_seg], probabilities and log-softmax."""
    z = np.asarray(z, np.float64)
    M, n = z.shape[0], len(segs) - 1
    logp, H, L = np.zeros(M), np.zeros((M, n)), np.zeros((M, n))
    P, S, T = np.zeros_like(z), np.zeros_like(z), np.zeros((M, n))
    empty = np.zeros((M, n), bool)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        for s in range(n):
            lo, hi = segs[s], segs[s + 1]
            x = z[:, lo:hi]
            act = np.clip(np.asarray(actions)[:, s], lo, hi - 1)
            top = x.max(axis=1, keepdims=True)
            none = (top == -np.inf)[:, 0]
            shifted = x - np.where(top == -np.inf, 0.0, top)
            e = np.exp(shifted)
            tot = e.sum(axis=1, keepdims=True)
            lse = np.where(none[:, None], -np.inf, top + np.log(tot))
            ls = np.where(none[:, None], -np.inf, shifted - np.log(tot))
            p = np.where(none[:, None], 0.0, e / tot)
            H[:, s] = -np.where(p == 0, 0.0, p * ls).sum(axis=1)
            P[:, lo:hi], S[:, lo:hi], L[:, s], T[:, s], empty[:, s] = p, ls, lse[:, 0], top[:, 0], none
            logp += np.where(none, 0.0, ls[np.arange(M), act - lo])
    return dict(logp=logp, H=H, lse=L, top=T, p=P, ls=S, empty=empty)


def logit_grad(st, segs, actions, g_logp, g_ent):
    """g_logp (onehot - p) - g_ent p (log p + H), rows of zero gradients exactly 0."""
    M = st["p"].shape[0]
    g_logp, g_ent = np.asarray(g_logp, np.float64), np.asarray(g_ent, np.float64)
    d = np.zeros_like(st["p"])
    with np.errstate(invalid="ignore"):
        for s in range(len(segs) - 1):
            lo, hi = segs[s], segs[s + 1]
            act = np.clip(np.asarray(actions)[:, s], lo, hi - 1)
            p = st["p"][:, lo:hi]
            hot = np.zeros_like(p)
            hot[np.arange(M), act - lo] = 1.0
            plogp = np.where(p == 0, 0.0, p * st["ls"][:, lo:hi])
            ent = np.where((g_ent != 0)[:, None], g_ent[:, None] * (plogp + p * st["H"][:, s:s + 1]), 0.0)
            v = g_logp[:, None] * (hot - p) - ent
            zero = st["empty"][:, s] | ((g_logp == 0) & (g_ent == 0))
            d[:, lo:hi] = np.where(zero[:, None], 0.0, v)
    return d


def policy_loss(z, segs, actions, logp_old, logp_ref, adv, weight=None, clip_low=0.2, clip_high=0.2, w_kl=0.0,
                w_entropy=0.0) -> dict:
    st = row_stats(z, segs, actions)
    M = st["logp"].size
    w = np.full(M, 1.0 / M) if weight is None else np.asarray(weight, np.float64)
    on = w != 0
    lp = np.where(on, st["logp"], 0.0)
    f = lambda x: np.where(on, np.asarray(x, np.float64), 0.0)  # noqa: E731
    adv, old = f(adv), f(logp_old)
    with np.errstate(invalid="ignore", over="ignore"):
        ratio = np.exp(lp - old)
        s1, s2 = ratio * adv, np.clip(ratio, 1 - clip_low, 1 + clip_high) * adv
        if logp_ref is None:
            kl, dkl = np.zeros(M), np.zeros(M)
        else:
            x = f(logp_ref) - lp
            kl, dkl = np.where(x == np.inf, np.inf, np.expm1(x) - x), -np.expm1(x)
        inside = (ratio >= 1 - clip_low) & (ratio <= 1 + clip_high)
        d = np.where((s2 < s1) & ~inside, 0.0, -adv * ratio)
        g = np.where(on, w * (d + (w_kl * dkl if w_kl else 0.0)), 0.0)
        H = np.where(on, st["H"].sum(axis=1), 0.0)
        t = [np.where(on, w * v, 0.0).sum() for v in (-np.minimum(s1, s2), kl, H)]
    ge = np.where(on, -w * w_entropy, 0.0)
    total = t[0] + (w_kl * t[1] if w_kl else 0.0) - (w_entropy * t[2] if w_entropy else 0.0)
    return dict(loss=np.array([total] + t), logp=lp, g_logp=g, g_ent=ge, ratio=ratio, st=st,
                dlogits=logit_grad(st, segs, actions, g, ge))


def preference_loss(z, segs, actions, logp_ref, weight, seq_ptr, beta=0.1, smoothing=0.0) -> dict:
    st = row_stats(z, segs, actions)
    N = st["logp"].size
    w = np.ones(N) if weight is None else np.asarray(weight, np.float64)
    ref = np.zeros(N) if logp_ref is None else np.asarray(logp_ref, np.float64)
    diff = np.where(w != 0, w * (np.where(w != 0, st["logp"], 0.0) - np.where(w != 0, ref, 0.0)), 0.0)
    P = (len(seq_ptr) - 1) // 2
    R = np.array([diff[seq_ptr[q]:seq_ptr[q + 1]].sum() for q in range(2 * P)])
    h = beta * (R[0::2] - R[1::2])
    lose = np.logaddexp(0.0, -h)
    win = np.logaddexp(0.0, h)
    each = (1 - smoothing) * lose + (smoothing * win if smoothing else 0.0)
    sig = 0.5 * (1.0 + np.tanh(0.5 * h))
    gh = beta / P * (smoothing * sig - (1 - smoothing) * (1.0 - sig))
    g, inside = np.zeros(N), np.zeros(N, bool)
    for q in range(2 * P):
        rows = slice(seq_ptr[q], seq_ptr[q + 1])
        g[rows] = np.where(w[rows] != 0, w[rows] * (gh[q // 2] if q % 2 == 0 else -gh[q // 2]), 0.0)
        inside[rows] = True
    return dict(loss=np.array([each.mean(), lose.mean(), h.mean(), (h > 0).mean()]), ratio=R, h=h, g_logp=g, inside=inside,
                st=st, dlogits=logit_grad(st, segs, actions, g, np.zeros(N)))
