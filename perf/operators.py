"""Performance cases of the policy objectives: log-probabilities of chosen actions with their
gradient, the clipped policy loss with a KL term and the pairwise preference loss, through their public
entry points.

An actor's logits are rows of `a` columns, cut into one segment per modification type (one segment: a
token head, as wide as a vocabulary).  Rows are transitions or tokens; some are padding (weight 0), and
some actions are excluded (logit -inf).  The kinds of cases:

  logp   harl_policy_logp, and with `grad` harl_policy_logp_grad after it: log-probability and entropy
         of every row, and the logits' gradient from the gradients of both
  loss   harl_policy_loss: clipped surrogate, KL term to a reference and entropy bonus, with the
         logits' gradient
  pref   harl_preference_loss: paired log ratios of preferred and rejected tracks of unequal lengths,
         with the logits' gradient

Where `own` is false, run() computes the same from elementary torch operations in 32 bits; exact()
does in 64 bits.  Sizes are those of the framework's own actor (26 logits in 4 types, 4,096 and 65,536
transitions, windows of 20 steps) and of generic token heads of 2^9 to 2^17 columns.
"""
import math

import torch

DEV = "cuda"
own = False


# ------------------------------------------------------------------------------------------------
# the cases: M rows of `a` columns in `types` segments (the first holds a - 3 (types - 1) actions, the
# others 3 each), `pad` unused columns behind a row, a share `excl` of excluded actions and `empty` of
# padding rows
# ------------------------------------------------------------------------------------------------
def listed():
    return [
        # one decoding step of one sequence: latency
        dict(name="logp_step", kind="logp", dtype="bf16", M=1, a=50001, types=1, pad=7, excl=0.0, empty=0.0, grad=False),
        # log-probabilities of a large rollout of the framework's own actor
        dict(name="logp_rollout", kind="logp", dtype="f32", M=65521, a=26, types=4, pad=0, excl=0.1, empty=0.0, grad=False),
        # a user's own loss on the tokens of a micro-batch: forward and backward
        dict(name="logp_grad_tokens", kind="logp", dtype="bf16", M=2048, a=32768, types=1, pad=0, excl=0.0, empty=0.0, grad=True),
        # a PPO mini-batch of the framework's own actor, invalid modifications excluded
        dict(name="loss_minibatch", kind="loss", dtype="f32", M=4096, a=26, types=4, pad=0, excl=0.1, empty=0.0, w_kl=0.0, w_entropy=0.01),
        # an actor with 32 x 32 + 1 tile-size actions and three more types
        dict(name="loss_tiles", kind="loss", dtype="f32", M=8192, a=1034, types=4, pad=0, excl=0.2, empty=0.1, w_kl=0.05, w_entropy=0.01),
        # the last few tokens of a batch, an odd vocabulary with padded rows
        dict(name="loss_few_tokens", kind="loss", dtype="bf16", M=7, a=100003, types=1, pad=5, excl=0.01, empty=0.0, w_kl=0.04, w_entropy=0.0),
        # the tokens of a micro-batch over a large vocabulary
        dict(name="loss_tokens", kind="loss", dtype="bf16", M=4096, a=131072, types=1, pad=0, excl=0.0, empty=0.15, w_kl=0.04, w_entropy=0.001),
        # the same in fp32 at an odd width (rows of every alignment)
        dict(name="loss_tokens_f32", kind="loss", dtype="f32", M=1024, a=65521, types=1, pad=0, excl=0.0, empty=0.1, w_kl=0.04, w_entropy=0.0),
        # pairs of schedule tracks of up to 20 steps
        dict(name="pref_tracks", kind="pref", dtype="f32", pairs=256, longest=20, a=26, types=4, pad=0, excl=0.1, empty=0.0),
        # a few pairs of short answers
        dict(name="pref_short", kind="pref", dtype="bf16", pairs=2, longest=16, a=32768, types=1, pad=0, excl=0.0, empty=0.2),
        # an odd vocabulary in fp32
        dict(name="pref_odd_f32", kind="pref", dtype="f32", pairs=16, longest=33, a=20011, types=1, pad=2, excl=0.01, empty=0.2),
        # a micro-batch of pairs of long answers, a fifth of the tokens prompts
        dict(name="pref_long", kind="pref", dtype="bf16", pairs=8, longest=512, a=65536, types=1, pad=0, excl=0.0, empty=0.2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logp", "loss", "loss", "pref", "pref"])
    case = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), excl=rng.choice([0.0, 0.01, 0.1, 0.3]))
    if rng.random() < 0.4:  # an actor with modification types
        case.update(types=rng.randint(2, 6), pad=rng.choice([0, 0, 1, 6]))
        case["a"] = _log_int(rng, 4, 1030) + 3 * (case["types"] - 1)
        most = min(65536, (1 << 28) // case["a"])
    else:  # a token head
        case.update(types=1, a=_log_int(rng, 512, 131072), pad=rng.choice([0, 0, 1, 8, 13]))
        if rng.random() < 0.5:
            case["a"] -= case["a"] % 64
        most = min(16384, (1 << 28) // case["a"])
    rows = _log_int(rng, 1, most)
    if kind == "pref":
        case["longest"] = _log_int(rng, 1, max(1, min(1024, rows // 2)))
        case.update(pairs=max(1, rows // (case["longest"] + 1)), empty=rng.choice([0.0, 0.2, 0.4]))
    else:
        case.update(M=rows, empty=rng.choice([0.0, 0.0, 0.15]) if kind == "loss" else 0.0)
    if kind == "logp":
        case["grad"] = rng.random() < 0.6
    if kind == "loss":
        case.update(w_kl=rng.choice([0.0, 0.04, 0.2]), w_entropy=rng.choice([0.0, 0.0, 0.01]))
    return case


CLIP_LOW, CLIP_HIGH, BETA, SMOOTHING = 0.2, 0.28, 0.1, 0.05


def _segments(case):
    first = case["a"] - 3 * (case["types"] - 1)
    return [0] + [first + 3 * t for t in range(case["types"])]


def _lengths(case):
    """Rows of the 2 `pairs` sequences: 1 .. longest, the same for every seed."""
    return [1 + (q * 7919 + 13) % case["longest"] for q in range(2 * case["pairs"])]


def _rows(case):
    return sum(_lengths(case)) if case["kind"] == "pref" else case["M"]


def _live(case):
    """Rows that are no padding."""
    return _rows(case) - int(case["empty"] * _rows(case))


# ------------------------------------------------------------------------------------------------
# inputs, drawn from the seed alone
# ------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    M, a, segs, n = _rows(case), case["a"], _segments(case), case["types"]
    normal = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    full = normal(M, a + case["pad"]) * 2.0
    if case["excl"]:
        full = torch.where(torch.rand(M, a + case["pad"], generator=g, device=DEV) < case["excl"], -math.inf, full)
    full = full.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
    logits = full[:, :a]
    acts = []
    for lo, hi in zip(segs, segs[1:]):  # every action is drawn from its segment's softmax
        u = torch.rand(M, hi - lo, generator=g, device=DEV).clamp_(1e-7, 1 - 1e-7)
        acts.append((logits[:, lo:hi].float() - torch.log(-torch.log(u))).argmax(1).to(torch.int32) + lo)
        del u
    live = torch.ones(M, device=DEV)
    live[torch.randperm(M, generator=g, device=DEV)[: M - _live(case)]] = 0.0
    s = dict(case=case, M=M, a=a, segs=segs, ld=full.stride(0), full=full, logits=logits, live=live,
             actions=torch.stack(acts, 1).contiguous())
    if n > 1:  # the plain forms' view of a row: [types][longest type], short types padded
        longest = max(hi - lo for lo, hi in zip(segs, segs[1:]))
        index = torch.tensor(segs[:-1], device=DEV)[:, None] + torch.arange(longest, device=DEV)
        s["valid"] = index < torch.tensor(segs[1:], device=DEV)[:, None]
        s["index"] = index.clamp(max=a - 1)
    f32 = dict(dtype=torch.float32, device=DEV)
    s["out_logp"] = torch.zeros(M, **f32)
    if case["kind"] == "logp":
        s["out_entropy"], s["out_lse"] = torch.zeros(M, n, **f32), torch.zeros(M, n, 2, **f32)
        if case["grad"]:
            s["g_logp"], s["g_entropy"] = normal(M) / M, normal(M) * (0.01 / M)
    else:
        logp = _row_stats(s, s)[0].float()
        s["logp_ref"] = logp + 0.2 * normal(M)
        s["out_loss"] = torch.zeros(4, **f32)
    if case["kind"] == "loss":
        # log ratios up to 0.4 either way, none within 1e-3 of a clip border
        x = (torch.rand(M, generator=g, device=DEV) - 0.5) * 0.8
        near = ((x - math.log1p(-CLIP_LOW)).abs() < 1e-3) | ((x - math.log1p(CLIP_HIGH)).abs() < 1e-3)
        s["logp_old"] = logp - torch.where(near, x + 5e-3, x)
        s["adv"], s["weight"] = normal(M), live / max(1, _live(case))
    if case["kind"] == "pref":
        lens = _lengths(case)
        order = torch.randperm(len(lens), generator=g, device=DEV)
        lens = torch.tensor(lens, device=DEV)[order]
        s["seq_ptr"] = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), lens.cumsum(0)]).to(torch.int32)
        s["seq_of_row"] = torch.repeat_interleave(torch.arange(len(order), device=DEV), lens)
        s["out_ratio"] = torch.zeros(2 * case["pairs"], **f32)
    if case["kind"] != "logp" or case["grad"]:
        s["out_grad"] = torch.zeros_like(full)
    return s


# ------------------------------------------------------------------------------------------------
# the plain forms
# ------------------------------------------------------------------------------------------------
def _by_type(s, logits):
    """fp32 logits as [M][types][longest type], -inf where a type has no such action."""
    if s["case"]["types"] == 1:
        return logits.float().unsqueeze(1)
    return torch.where(s["valid"], logits.float()[:, s["index"]], -math.inf)


def _row_stats(s, inp):
    """Joint log-probability, per-type entropy, per-type log-sum-exp (maximum, rest), and the log-softmax's parts."""
    z = _by_type(s, inp["logits"])
    top = z.amax(2, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(z - top)
    total = e.sum(2, keepdim=True, dtype=torch.float64)
    some = total > 0
    # in 64 bits: a track's log ratio is a long sum of small differences of these
    lse = top.double() + torch.log(total)
    p = torch.where(some, e / total.float(), 0.0)
    logs = torch.where(e > 0, (z - top) - torch.log(total).float(), 0.0)
    entropy = -(p * logs).sum(2)
    chosen = torch.gather(inp["logits"].double(), 1, inp["actions"].long())
    logp = torch.where(some[:, :, 0], chosen - lse[:, :, 0], 0.0).sum(1)
    parts = torch.stack([torch.where(some, top.double(), -math.inf), torch.where(some, torch.log(total), 0.0)], 3)
    return logp, entropy, parts[:, :, 0], p, logs, some


def _logit_grad(s, p, logs, entropy, some, g_logp, g_entropy):
    """g_logp (onehot - p) - g_entropy p (log p + H), rounded once to the logits' type."""
    g = -g_logp[:, None, None] * p
    if g_entropy is not None:
        g = g - g_entropy[:, None, None] * p * (logs + entropy[:, :, None])
    if s["case"]["types"] == 1:
        d = g[:, 0]
    else:
        d = torch.zeros(s["M"], s["a"], device=DEV)
        d[:, s["index"][s["valid"]]] = g[:, s["valid"]]
    d = d.scatter_add(1, s["actions"].long(), torch.where(some[:, :, 0], g_logp[:, None], 0.0))
    return d.to(s["logits"].dtype)


def _plain_logp(s):
    logp, entropy, lse, p, logs, some = _row_stats(s, s)
    out = dict(logp=logp.float(), entropy=entropy, lse=lse.float())
    if s["case"]["grad"]:
        out["dlogits"] = _logit_grad(s, p, logs, entropy, some, s["g_logp"], s["g_entropy"])
    return out


def _plain_loss(s):
    case, w, adv = s["case"], s["weight"], s["adv"]
    logp, entropy, _, p, logs, some = _row_stats(s, s)
    logp = torch.where(w != 0, logp, 0.0)
    ratio = torch.exp((logp - s["logp_old"]).float())
    s1, s2 = ratio * adv, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * adv
    x = s["logp_ref"] - logp
    kl = torch.expm1(x) - x
    sums = [(w.double() * t).sum() for t in (-torch.minimum(s1, s2), kl, entropy.sum(1))]
    total = sums[0] + case["w_kl"] * sums[1] - case["w_entropy"] * sums[2]
    inside = (ratio >= 1 - CLIP_LOW) & (ratio <= 1 + CLIP_HIGH)
    g = w * (case["w_kl"] * -torch.expm1(x).float() - adv * ratio * ((s1 <= s2) | inside))
    ge = -w * case["w_entropy"] if case["w_entropy"] else None
    return dict(loss=torch.stack([total] + sums).float(), logp=logp.float(), dlogits=_logit_grad(s, p, logs, entropy, some, g, ge))


def _plain_pref(s):
    pairs = s["case"]["pairs"]
    logp, entropy, _, p, logs, some = _row_stats(s, s)
    diff = torch.where(s["live"] != 0, logp - s["logp_ref"], 0.0)
    ratio = torch.zeros(2 * pairs, dtype=torch.float64, device=DEV).index_add(0, s["seq_of_row"], diff)
    h = BETA * (ratio[0::2] - ratio[1::2])
    lose = torch.log1p(torch.exp(-h.abs())) + torch.clamp(-h, min=0.0)  # -log sigmoid(h)
    losses = lose + SMOOTHING * h
    g_h = (torch.sigmoid(h) - (1 - SMOOTHING)) * (BETA / pairs)
    g = torch.stack([g_h, -g_h], 1).reshape(-1)[s["seq_of_row"]].float() * s["live"]
    loss = torch.stack([losses.mean(), lose.mean(), h.mean(), (h > 0).double().mean()]).float()
    return dict(loss=loss, ratio=ratio.float(), dlogits=_logit_grad(s, p, logs, entropy, some, g, None))


# ------------------------------------------------------------------------------------------------
# the framework's calls
# ------------------------------------------------------------------------------------------------
def _workspace(s, nbytes):
    if "ws" not in s:
        s["ws"] = torch.empty(max(256, nbytes), dtype=torch.uint8, device=DEV)
    return s["ws"], s["ws"].numel()


def _own(s):
    from paper_2211_11172_amd import harl
    case, M, ld = s["case"], s["M"], s["ld"]
    if "head" not in s:
        s["head"] = harl.policy_head(case["dtype"], s["a"], s["segs"])
    head = s["head"]
    if case["kind"] == "logp":
        ws, wsb = _workspace(s, harl.harl_policy_logp_workspace_size(head, M))
        harl.harl_policy_logp(head, s["logits"], ld, M, s["actions"], s["out_logp"], s["out_entropy"], s["out_lse"], ws, wsb)
        out = dict(logp=s["out_logp"], entropy=s["out_entropy"], lse=s["out_lse"])
        if case["grad"]:
            harl.harl_policy_logp_grad(head, s["logits"], ld, M, s["actions"], s["out_lse"], s["out_entropy"], s["g_logp"],
                                       s["g_entropy"], s["out_grad"], ld)
            out["dlogits"] = s["out_grad"][:, :s["a"]]
        return out
    if case["kind"] == "loss":
        if "cfg" not in s:
            s["cfg"] = harl.policy_loss_config(CLIP_LOW, CLIP_HIGH, case["w_kl"], case["w_entropy"])
        ws, wsb = _workspace(s, harl.harl_policy_loss_workspace_size(head, M))
        harl.harl_policy_loss(head, s["cfg"], s["logits"], ld, M, s["actions"], s["logp_old"], s["logp_ref"], s["adv"],
                              s["weight"], s["out_grad"], ld, s["out_logp"], s["out_loss"], ws, wsb)
        return dict(loss=s["out_loss"], logp=s["out_logp"], dlogits=s["out_grad"][:, :s["a"]])
    if "cfg" not in s:
        s["cfg"] = harl.preference_config(BETA, SMOOTHING)
    ws, wsb = _workspace(s, harl.harl_preference_loss_workspace_size(head, M, case["pairs"]))
    harl.harl_preference_loss(head, s["cfg"], s["logits"], ld, M, s["actions"], s["logp_ref"], s["live"], s["seq_ptr"],
                              case["pairs"], s["out_grad"], ld, s["out_ratio"], s["out_loss"], ws, wsb)
    return dict(loss=s["out_loss"], ratio=s["out_ratio"], dlogits=s["out_grad"][:, :s["a"]])


def run(state):
    if own:
        return _own(state)
    return dict(logp=_plain_logp, loss=_plain_loss, pref=_plain_pref)[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without: the logits of every row that counts read once, the gradient written once
# (zeros for padding rows, which need no logits), per-row values and parameters
# ------------------------------------------------------------------------------------------------
def work(case):
    M, live, a, n = _rows(case), _live(case), case["a"], case["types"]
    es = 2 if case["dtype"] == "bf16" else 4
    grad = case["kind"] != "logp" or case["grad"]
    per_row = {"logp": 4 * n + 4 + 12 * n + (8 + 12 * n if grad else 0), "loss": 4 * n + 20, "pref": 4 * n + 8}[case["kind"]]
    # maximum, difference, exponential, sum, entropy's product and sum; gradient: difference, exponential, product
    return {"bytes": es * a * (live + (M if grad else 0)) + per_row * M, "flops": a * live * (6 + (4 if grad else 0))}


# ------------------------------------------------------------------------------------------------
# the definition in 64 bits, a block of rows and a type at a time
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    M, a, segs = s["M"], s["a"], s["segs"]
    f64 = dict(dtype=torch.float64, device=DEV)
    pairs_of = list(zip(segs, segs[1:]))
    blocks = [slice(i, min(M, i + max(1, (1 << 26) // a))) for i in range(0, M, max(1, (1 << 26) // a))]
    logp, H, L, top = torch.zeros(M, **f64), *(torch.zeros(M, len(pairs_of), **f64) for _ in range(3))
    for b in blocks:
        z = s["logits"][b].double()
        for t, (lo, hi) in enumerate(pairs_of):
            lse = torch.logsumexp(z[:, lo:hi], 1)
            ls = z[:, lo:hi] - lse[:, None]
            pl = torch.where(ls > -1e300, ls.exp() * ls, 0.0)
            chosen = z.gather(1, s["actions"][b, t:t + 1].long())[:, 0]
            none = torch.isinf(lse)
            logp[b] += torch.where(none, 0.0, chosen - lse)
            H[b, t], L[b, t] = torch.where(none, 0.0, -pl.nan_to_num(0.0).sum(1)), lse
            top[b, t] = z[:, lo:hi].amax(1)
    one = lambda k: s[k].double()  # noqa: E731
    f = lambda v: float(torch.tensor(v, dtype=torch.float32))  # the calls take their parameters as fp32  # noqa: E731
    if case["kind"] == "logp":
        out = dict(logp=logp, entropy=H, lse=torch.stack([top, torch.where(torch.isinf(L), 0.0, L - top)], 2))
        if not case["grad"]:
            return out
        g, ge = one("g_logp"), one("g_entropy")
    elif case["kind"] == "loss":
        w, adv, wk, we = one("weight"), one("adv"), f(case["w_kl"]), f(case["w_entropy"])
        lo, hi = 1 - f(CLIP_LOW), 1 + f(CLIP_HIGH)
        logp = torch.where(w == 0, torch.zeros_like(logp), logp)
        ratio, back = torch.exp(logp - one("logp_old")), torch.exp(one("logp_ref") - logp)
        sur = torch.minimum(ratio * adv, torch.clamp(ratio, lo, hi) * adv)
        kl = back - 1 - (one("logp_ref") - logp)
        parts = [-(w * sur).sum(), (w * kl).sum(), (w * H.sum(1)).sum()]
        out = dict(loss=torch.stack([parts[0] + wk * parts[1] - we * parts[2]] + parts), logp=logp)
        flat = ((ratio > hi) & (adv > 0)) | ((ratio < lo) & (adv < 0))
        g, ge = w * (torch.where(flat, 0.0, -adv * ratio) + wk * (1 - back)), -we * w
    else:
        n, beta, ls = case["pairs"], f(BETA), f(SMOOTHING)
        ptr, live = s["seq_ptr"].long(), one("live")
        diff = torch.where(live == 0, torch.zeros_like(logp), logp - one("logp_ref"))
        run_sum = torch.cat([torch.zeros(1, **f64), diff.cumsum(0)])
        ratio = run_sum[ptr[1:]] - run_sum[ptr[:-1]]
        h = beta * (ratio[0::2] - ratio[1::2])
        lose = torch.nn.functional.softplus(-h, threshold=700.0)
        win = torch.nn.functional.softplus(h, threshold=700.0)
        each = (1 - ls) * lose + ls * win
        out = dict(loss=torch.stack([each.mean(), lose.mean(), h.mean(), (h > 0).double().mean()]), ratio=ratio)
        gh = beta / n * (ls / (1 + torch.exp(-h)) - (1 - ls) / (1 + torch.exp(h)))
        seq = torch.searchsorted(ptr[1:].contiguous(), torch.arange(M, device=DEV), right=True)
        g, ge = torch.where(seq % 2 == 0, 1.0, -1.0) * gh[seq // 2] * live, torch.zeros(M, **f64)
    d = torch.zeros(M, a, **f64)
    for b in blocks:
        z = s["logits"][b].double()
        for t, (lo, hi) in enumerate(pairs_of):
            none = torch.isinf(L[b, t])[:, None]
            ls = torch.where(none, -math.inf, z[:, lo:hi] - L[b, t][:, None])
            p = ls.exp()
            d[b, lo:hi] = -g[b, None] * p - ge[b, None] * p * (torch.where(p > 0, ls, 0.0) + H[b, t][:, None])
            hit = torch.where(none[:, 0], 0.0, g[b])
            d[b] = d[b].scatter_add(1, s["actions"][b, t:t + 1].long(), hit[:, None])
    out["dlogits"] = d
    return out
