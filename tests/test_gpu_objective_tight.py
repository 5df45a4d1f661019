"""Policy objectives with bars that a single lost column, or a correction left out, is beyond.  The bars of
tests/test_gpu_objective.py count every rounding that a row of n columns may meet, and grow with n.

Rows of which every 64th column holds one value c and the others c - 300 (whose exponential is 0 in fp32): the sum is
the number of those columns, k, without a rounding (2^0 = 1), so that log s = log k to the logarithm's own error; 64 rows
with the columns of every remainder see each column once.  With E = 2^-24: the hardware's log2 is mended by s 2^-(log2 s) - 1
(an exponential, 2 E, and a rounding), ln 2 and the product are rounded (E log k each): 2 E log k + 4 E.  A lost column moves
log k by 1 / k, 40 times that at 2^20 columns."""
from __future__ import annotations

import math

import numpy as np
import pytest

from tests.gpu_util import log, require_gpu

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
STEP = 64


def _rows(torch, dtype, M, a, off, pad, step):
    """Logits in a buffer `off` elements in and `pad` columns apart; c a row; the number of columns of value c."""
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    buf = torch.full((off + M * (a + pad) + 16,), 9.0, dtype=td, device="cuda")
    z = buf[off:off + M * (a + pad)].view(M, a + pad)[:, :a]
    r = torch.arange(M, device="cuda")
    c = (r % 5 - 2).float()
    for i in range(0, M, 128):
        s = slice(i, i + 128)
        on = (torch.arange(a, device="cuda")[None, :] - r[s, None]) % step == 0
        z[s] = torch.where(on, c[s, None], c[s, None] - 300.0).to(td)
    k = (a - r % step + step - 1) // step
    act = (r % step + step * (r * 7919 % k)).to(torch.int32)[:, None].contiguous()  # one of the k, another one a row
    return buf, z, c, k.double(), act


# rows that a workgroup of 16 waves reads, chunks, a wave a row, workgroups of 4, 8 and 16 waves, rows beyond the registers
SHAPES = [("f32", 64, 65540, 0, 0), ("bf16", 64, 131072, 0, 0), ("bf16", 64, 139003, 1, 3), ("f32", 64, 1 << 20, 0, 0), ("bf16", 64, 1 << 20, 3, 1),
          ("f32", 1100, 513, 1, 2), ("bf16", 1100, 3999, 0, 1), ("f32", 1100, 7001, 2, 0), ("bf16", 1100, 30011, 5, 2), ("bf16", 1100, 60032, 0, 0),
          ("f32", 1100, 33001, 0, 3), ("bf16", 1100, 131072, 0, 0), ("f32", 1100, 66001, 1, 2), ("bf16", 1100, 139003, 7, 6),
          ("f32", 1100, 127, 0, 0), ("bf16", 1100, 511, 0, 1)]


@pytest.mark.parametrize("dtype,M,a,off,pad", SHAPES)
def test_every_column_counts(dtype, M, a, off, pad):
    require_gpu()
    import torch
    from paper_2211_11172_amd import harl
    head, ld = harl.policy_head(dtype, a), a + pad
    f = lambda *n: torch.full(n, float("nan"), device="cuda")  # noqa: E731
    n = max(harl.harl_policy_logp_workspace_size(head, M), harl.harl_policy_loss_workspace_size(head, M),
            harl.harl_preference_loss_workspace_size(head, M, M // 2))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    for step in (STEP, 1):
        log("every column: %s %d x %d, every %d" % (dtype, M, a, step))
        buf, z, c, k, act = _rows(torch, dtype, M, a, off, pad, step)
        want = torch.log(k)
        bar = 2 * E * want + 4 * E
        lp, H, L = f(M), f(M, 1), f(M, 1, 2)
        harl.harl_policy_logp(head, z, ld, M, act, lp, H, L, ws, n)
        assert (L[:, 0, 0] == c).all()
        assert ((L[:, 0, 1].double() - want).abs() <= bar).all()
        assert ((lp.double() + want).abs() <= bar + E * want).all()
        assert ((H[:, 0].double() - want).abs() <= bar + E * want).all()
        # the gradient: 1 / k where the value is c, to the errors of 1 / s and of one product more, and 0 elsewhere
        g = torch.full((M,), -1.0, device="cuda")
        gbuf = torch.zeros_like(buf)
        dz = gbuf[off:off + M * ld].view(M, ld)[:, :a]
        half = 2.0 ** -8 if dtype == "bf16" else E

        def check_grad(scale, rel):
            for i in range(0, M, 128):
                s = slice(i, min(i + 128, M))
                on = z[s].float() == c[s, None]
                p = torch.where(on, (scale[s] / k[s])[:, None], torch.zeros((), dtype=torch.float64, device="cuda"))
                p.scatter_add_(1, act[s].long(), -scale[s][:, None])
                assert ((dz[s].double() - p).abs() <= p.abs() * (rel + half) + E * scale[s].abs()[:, None] * on).all()
        harl.harl_policy_logp_grad(head, z, ld, M, act, L, None, g, None, dz, ld)
        # e^-(log s) from the saved log s: its error and its rounding, the product with log2 e, an exponential
        check_grad(torch.ones(M, dtype=torch.float64, device="cuda"), float((bar + 3 * E * want).max()) + 4 * E)
        # the clipped loss with ratio 1 and advantage 1: gradient -(1 - 1 / k) / M at the action
        old, adv, loss, new = (-want).float(), torch.ones(M, device="cuda"), f(4), f(M)
        dz.zero_()
        harl.harl_policy_loss(head, harl.policy_loss_config(0.2, 0.2, 0.0, 0.0), z, ld, M, act, old, None, adv, None, dz, ld, new, loss, ws, n)
        assert ((new.double() + want).abs() <= bar + E * want).all()
        # the ratio is 1 but for the errors of logp and of logp_old
        r = float((bar + 2 * E * want).max()) + 4 * E
        check_grad(torch.full((M,), 1.0 / M, dtype=torch.float64, device="cuda"), r + 4 * E)
        assert abs(loss[1].item() + 1.0) <= r and loss[2] == 0
        assert abs(loss[3].item() - want.mean().item()) <= float((bar + 2 * E * want).max())
        # the preference loss, a track a row: the sum of the row in parts, its log-probability in 64 bits
        ptr = torch.arange(M + 1, dtype=torch.int32, device="cuda")
        ratio, dz_ = f(M), dz.zero_()
        harl.harl_preference_loss(head, harl.preference_config(1.0), z, ld, M, act, old, None, ptr, M // 2, dz_, ld, ratio, loss, ws, n)
        torch.cuda.synchronize()
        if a > 512:  # (the short heads' logarithm is the mended one)
            bar = 4 * E * torch.ones_like(want)
        assert ((ratio.double() - (-want - old.double())).abs() <= bar + E * 1e-5).all()
        assert abs(loss[1].item() - math.log(2.0)) <= 4 * E * (1 + float(want.max()))
        sign = torch.where(torch.arange(M, device="cuda") % 2 == 0, 1.0, -1.0).double() / (M // 2) * 0.5
        check_grad(sign, 8 * E + float(bar.max()))
        del buf, gbuf, z, dz


@pytest.mark.parametrize("dtype,M,a", [("bf16", 1030, 131072), ("f32", 1030, 65521), ("bf16", 1030, 139003), ("bf16", 40, 131072), ("f32", 3, 1 << 20)])
def test_random_rows_by_their_depth(dtype, M, a):
    """The error of log s by the additions that a lane makes (and at most 16 more for edges and whole vectors), and 40
    that join lanes and chunks: E (lane + 56), and E (4 + 2 log n) for the exponentials and the logarithm.  From 1,024 rows
    on harl_policy_logp has 256 lanes a row and harl_policy_loss 1,024; fewer rows have 1,024 lanes up to 16,384
    vectors and else, as in the clipped loss, 256 a chunk of the row, of which there are enough for 1,024 items, 64 at most;
    the preference loss has 256 a chunk of 2,048 vectors, or 64 chunks."""
    require_gpu()
    import torch
    from paper_2211_11172_amd import harl
    head = harl.policy_head(dtype, a)
    g = torch.Generator(device="cuda")
    g.manual_seed(a)
    z = torch.empty(M, a, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    for i in range(0, M, 128):
        z[i:i + 128] = (torch.randn(min(128, M - i), a, generator=g, device="cuda") * 2).to(z.dtype)
    act = torch.randint(0, a, (M, 1), generator=g, device="cuda", dtype=torch.int32)
    f = lambda *n: torch.full(n, float("nan"), device="cuda")  # noqa: E731
    n = max(harl.harl_policy_logp_workspace_size(head, M), harl.harl_policy_loss_workspace_size(head, M),
            harl.harl_preference_loss_workspace_size(head, M, M // 2))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    lp, H, L, new, ratio = f(M), f(M, 1), f(M, 1, 2), f(M), f(M // 2 * 2)
    harl.harl_policy_logp(head, z, a, M, act, lp, H, L, ws, n)
    lse = torch.cat([torch.logsumexp(z[i:i + 64].double(), 1) for i in range(0, M, 64)])
    want = torch.gather(z, 1, act.long())[:, 0].double() - lse
    harl.harl_policy_loss(head, harl.policy_loss_config(), z, a, M, act, lp, None, lp, None, None, 0, new, None, ws, n)
    ptr = torch.arange(M // 2 * 2 + 1, dtype=torch.int32, device="cuda")
    ref = want.float()
    harl.harl_preference_loss(head, harl.preference_config(1.0), z, a, M, act, ref, None, ptr, M // 2, None, 0, ratio, None, ws, n)
    torch.cuda.synchronize()
    vec = 8 if dtype == "bf16" else 4
    cut = min(64, -(-1024 // M), a // vec // 512)
    lanes = dict(logp=256 if M >= 1024 else 1024 if a <= 16384 * vec else 256 * cut, loss=1024 if M >= 1024 else 256 * cut,
                 pref=256 * min(64, max(cut, a // vec // 2048)))
    e = {k: E * (a / v + 16 + 40 + 4 + 2 * math.log(a)) for k, v in lanes.items()}
    errors = dict(logp=L[:, 0, 1].double() + L[:, 0, 0].double() - lse, loss=new.double() - want,
                  pref=ratio.double() - (want - ref.double())[:ratio.numel()])
    for k, v in errors.items():
        log("%s: bar %.2g, largest error %.2g" % (k, e[k], v.abs().max().item()))
    # the outputs' rounding, and in fp32 those of z - m and of the logarithm; the preference loss has them in 64 bits
    out = 2 * E * want.abs() + 2 * E * math.log(a)
    assert (errors["logp"].abs() <= e["logp"] + E * math.log(a)).all()
    assert ((lp.double() - want).abs() <= e["logp"] + out).all()
    assert (errors["loss"].abs() <= e["loss"] + out).all()
    assert (errors["pref"].abs() <= e["pref"] + E * 1e-5).all()


def test_track_ratios_do_not_have_the_exponents_roundings():
    """What the exponents y = (z - m) log2 e of a wide row are rounded by does not show in a track's log ratio.

    2,048 rows of five bf16 values each, the largest of them in every lane's first vector, so that every exponent is
    relative to it, and no more than four others in a lane (the rest is excluded), so that a lane's sums round little:
    R = round(sum 2^fl(y)) - round(sum 2^y), in 64 bits, is what those roundings do to log s.  The errors of
    the rows' log ratios, against the reference to the last bit so that they come out unrounded, are regressed on R: the
    slope is -1 where the roundings stay in the sum and 0 where they are taken out.  What else the errors hold (the
    exponential's, of at most 2 E = 1.2e-7 a value) does not know R: with the spreads as they come it moves the slope by
    (errors' / R's) / sqrt(2,048), which has to be a third of the 0.5 between the two at most."""
    require_gpu()
    import torch
    from paper_2211_11172_amd import harl
    M, a = 2048, 16384
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    top = (6.0 + torch.rand(M, 1, generator=g, device="cuda")).bfloat16().float()
    values = (top - 0.5 - 3.0 * torch.rand(M, 4, generator=g, device="cuda")).bfloat16()
    z = torch.gather(values, 1, torch.randint(0, 4, (M, a), generator=g, device="cuda"))
    z[:, (torch.arange(a, device="cuda") // 8 % 2 == 0) | (torch.arange(a, device="cuda") % 8 != 3)] = -math.inf
    z[:, :2048:8] = top.bfloat16()
    act = torch.zeros(M, 1, dtype=torch.int32, device="cuda")
    d = z.float() - top                                              # exact: both are bf16 and near each other
    assert torch.equal(d.double(), z.double() - top.double()) and (d <= 0).all()
    log2e = torch.tensor(1.44269504088896340736, dtype=torch.float32, device="cuda")
    lse, R = torch.empty(M, dtype=torch.float64, device="cuda"), torch.empty(M, dtype=torch.float64, device="cuda")
    for i in range(0, M, 256):
        s = slice(i, i + 256)
        lse[s] = torch.log(torch.exp(d[s].double()).sum(1))
        R[s] = torch.log(torch.exp2((d[s] * log2e).double()).sum(1)) - torch.log(torch.exp2(d[s].double() * log2e.double()).sum(1))
    ref = (-lse).float()
    head = harl.policy_head("bf16", a)
    n = harl.harl_preference_loss_workspace_size(head, M, M // 2)
    ws, ratio = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(M, device="cuda")
    ptr = torch.arange(M + 1, dtype=torch.int32, device="cuda")
    harl.harl_preference_loss(head, harl.preference_config(1.0), z, a, M, act, ref, None, ptr, M // 2, None, 0, ratio, None, ws, n)
    torch.cuda.synchronize()
    err = ratio.double() - (-lse - ref.double())
    R, err = (R - R.mean()).cpu().numpy(), (err - err.mean()).cpu().numpy()
    slope = float((R * err).sum() / (R * R).sum())
    log("spread of the roundings' part %.2g, of the errors %.2g, slope %.3f" % (R.std(), err.std(), slope))
    assert err.std() / R.std() / M ** 0.5 < 0.5 / 3
    assert abs(slope) < 0.5
