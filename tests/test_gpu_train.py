"""The losses on logits with their gradients (space_sar_loss_grad, space_policy_loss, space_preference_loss) and the gradient norm
with clipping (space_grad_norm, space_grad_clip) against the formulas in 64 bits, through the C ABI.  Tolerances: train_common."""
import ctypes as C
import itertools

import numpy as np
import pytest

from tests import gpu_common as gc
from tests import train_common as tc

pytestmark = pytest.mark.gpu
U = tc.U


def _loss_tol(terms, term_tol):
    """A sum of 32-bit terms in 64 bits, rounded once: every term's tolerance and rounding, then the sum's."""
    return float((term_tol + terms.abs() * U).sum() + terms.sum().abs() * U) + 2.0 ** -125


# rows shorter than a vector, than a wave, a workgroup; odd ones; around the sizes at which a row no longer fits what a
# workgroup holds (fp32 and bf16)
SIZES = [(1, 3), (2, 5), (3, 70), (7, 1), (64, 9), (65, 33), (255, 4), (1000, 200), (1027, 7), (4095, 3), (4096, 3), (4099, 6), (8191, 3), (8200, 5),
         (16384, 4), (16389, 3), (32000, 36), (32003, 3), (40001, 5), (65536, 2), (65543, 3), (131072, 2), (131079, 2), (262147, 2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,rows", SIZES)
def test_sar_loss_and_gradient(V, rows, dtype):
    torch = gc.require_gpu()
    gm = tc.head_model(V)
    x, labels = tc.make_logits(np.random.default_rng(V + rows), rows, V, dtype)
    ref = tc.Rows64(x, labels)
    n = int(ref.keep.sum())
    for mean, scale in ((False, None), (True, 0.25)):
        out = tc.fresh_out(gm, rows, dtype)
        gs = None if scale is None else torch.tensor([scale], device="cuda")
        gm.sar_loss_grad(x, labels, out, mean=mean, grad_scale=gs)
        torch.cuda.synchronize()
        ref.check_logp(out.row_logp)
        ref.check_logp(out.row_loss, -1.0)
        assert int(out.n_terms) == n
        w = 1.0 / max(n, 1) if mean else 1.0
        assert abs(float(out.loss) + float(ref.logp.sum()) * w) <= _loss_tol(ref.logp, ref.logp_tol) * w + abs(float(ref.logp.sum())) * w * U
        c = torch.full_like(ref.logp, w * (scale or 1.0))
        ref.check_gradient(out.dlogits, -c, c * 2 * U, dtype)
    assert gm.device_faults() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,xs,ds,xo,do", [(1000, 1000, 1000, 1, 0), (1000, 1008, 1003, 0, 3), (4097, 4100, 4097, 2, 1), (32000, 32001, 32000, 0, 1),
                                           (777, 777, 778, 5, 7)])
def test_strides_and_alignments_and_what_lies_between_rows(V, xs, ds, xo, do, dtype):
    """Strides of logits and gradient that differ, starts on any element: the same bits as from dense rows, and nothing written
    in front of, between or behind the rows."""
    torch = gc.require_gpu()
    rows, t = 6, tc.torch_type(dtype)
    gm = tc.head_model(V)
    x, labels = tc.make_logits(np.random.default_rng(V), rows, V, dtype)
    dense = tc.fresh_out(gm, rows, dtype)
    gm.sar_loss_grad(x, labels, dense)
    xb = torch.full((xo + rows * xs + 8,), float("nan"), dtype=t, device="cuda")
    xv = xb[xo:xo + rows * xs].view(rows, xs)[:, :V]
    xv.copy_(x)
    db = torch.full((do + rows * ds + 8,), 5.0, dtype=t, device="cuda")
    dv = db[do:do + rows * ds].view(rows, ds)[:, :V]
    out = tc.fresh_out(gm, rows, dlogits=dv)
    gm.sar_loss_grad(xv, labels, out)
    torch.cuda.synchronize()
    tc.Rows64(x, labels).check_gradient(dv, -torch.ones(rows, device="cuda", dtype=torch.float64), torch.zeros(rows, device="cuda", dtype=torch.float64), dtype)
    assert torch.equal(dv, dense.dlogits) and torch.equal(out.row_loss, dense.row_loss) and torch.equal(out.loss, dense.loss)
    dv.fill_(5.0)
    assert bool((db == 5.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1000, 32000, 131079])
def test_gradient_in_the_place_of_the_logits_and_beside_them(V, dtype):
    torch = gc.require_gpu()
    rows = 9
    gm = tc.head_model(V)
    x, labels = tc.make_logits(np.random.default_rng(V), rows, V, dtype)
    for call in ("sar", "pref"):
        def go(logits, out):
            if call == "sar":
                gm.sar_loss_grad(logits, labels, out)
            else:
                gm.preference_loss(logits, labels, torch.tensor([0, 4, 9], dtype=torch.int32, device="cuda"), out)
        out = tc.fresh_out(gm, rows, dtype, pairs=1)
        go(x, out)
        y = x.clone()
        place = tc.fresh_out(gm, rows, dlogits=y, pairs=1)
        go(y, place)
        wide = torch.full((rows, 2 * V + 1), 3.0, dtype=x.dtype, device="cuda")
        wide[:, :V] = x
        side = tc.fresh_out(gm, rows, dlogits=wide[:, V + 1:], pairs=1)
        go(wide[:, :V], side)
        torch.cuda.synchronize()
        assert torch.equal(y, out.dlogits) and torch.equal(wide[:, V + 1:], out.dlogits)
        assert torch.equal(wide[:, :V], x) and bool((wide[:, V] == 3.0).all())
        assert torch.equal(place.loss, out.loss) and torch.equal(side.loss, out.loss)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 1000, 32000, 131079])
def test_masked_and_infinite_logits(V, dtype):
    """-inf everywhere but at the label and at one other token, in front, behind, at the label itself; the type's lowest value as a mask;
    a row of nothing but -inf, NaN, +inf; the same in rows that do not count."""
    torch = gc.require_gpu()
    t = tc.torch_type(dtype)
    rng = np.random.default_rng(V)
    x, _ = tc.make_logits(rng, 13, V, dtype, lift=False)
    labels = torch.full((13,), V // 2, dtype=torch.int32, device="cuda")
    inf = float("inf")
    x[0, : V // 2] = -inf
    x[1, V // 2 + 1:] = -inf
    x[2, :] = -inf; x[2, V // 2] = 1.5                      # the label alone: loss 0, gradient 0
    x[3, V // 2] = -inf                                     # the label masked: infinite loss, gradient p - 1
    x[4, :] = torch.finfo(t).min; x[4, V // 2] = 0.25; x[4, V - 1] = 0.25
    x[5, :] = torch.finfo(t).min                            # nothing but the lowest value: uniform
    x[6, ::2] = -inf; x[6, V // 2] = 0.0
    x[7, :] = -inf; x[8, 1] = float("nan"); x[9, 2] = inf
    x[10, :] = -inf; x[11, 3] = float("nan"); x[12, 0] = inf
    labels[10:] = -1
    out = tc.fresh_out(tc.head_model(V), 13, dtype)
    gm = tc.head_model(V)
    gm.sar_loss_grad(x, labels, out)
    torch.cuda.synchronize()
    fine = [0, 1, 2, 4, 5, 6]
    ref = tc.Rows64(x[fine], labels[fine])
    ref.check_logp(out.row_logp[fine])
    one = torch.ones(len(fine), dtype=torch.float64, device="cuda")
    # x - top of the lowest value overflows to -inf: exponential 0, as in 64 bits
    ref.check_gradient(out.dlogits[fine], -one, 0 * one, dtype)
    assert float(out.row_loss[2]) == 0.0 and bool((out.dlogits[2] == 0).all())
    assert float(out.row_loss[3]) == inf and float(out.dlogits[3, V // 2]) == -1.0 and bool(torch.isfinite(out.dlogits[3]).all())
    assert abs(float(out.dlogits[3].double().sum())) < 1e-2
    for r in (7, 8, 9):
        assert np.isnan(float(out.row_loss[r])) and bool(torch.isnan(out.dlogits[r]).any()), r
    assert bool((out.dlogits[10:] == 0).all()) and bool((out.row_loss[10:] == 0).all())
    assert gm.device_faults() == 0


def test_labels_behind_the_vocabulary_and_no_row_that_counts():
    torch = gc.require_gpu()
    V, rows = 1000, 5
    gm = tc.head_model(V)
    x, _ = tc.make_logits(np.random.default_rng(0), rows, V, "f32")
    for labels, faults in (([-1] * 5, 0), ([V, 5, -3, 2 ** 31 - 1, -2 ** 31], 2)):
        lab = torch.tensor(labels, dtype=torch.int32, device="cuda")
        keep = torch.tensor([0 <= v < V for v in labels], device="cuda")
        out = tc.fresh_out(gm, rows, "f32", pairs=1)
        gm.sar_loss_grad(x, lab, out, mean=True)
        torch.cuda.synchronize()
        assert int(out.n_terms) == int(keep.sum()) and bool((out.dlogits[~keep] == 0).all()) and bool((out.row_loss[~keep] == 0).all())
        assert np.isfinite(float(out.loss)) and (faults or float(out.loss) == 0.0)
        assert gm.device_faults() == faults
        out = tc.fresh_out(gm, rows, "f32")
        gm.policy_loss(x, lab, torch.full((rows,), float("nan"), device="cuda") * torch.where(keep, 0.0, 1.0) if not faults else torch.ones(rows, device="cuda"), out)
        assert bool((out.dlogits[~keep] == 0).all()) and int(out.n_terms) == int(keep.sum())
        assert gm.device_faults() == faults
        out = tc.fresh_out(gm, rows, "f32", pairs=1)
        gm.preference_loss(x, lab, torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda"), out)
        assert bool((out.dlogits[~keep] == 0).all()) and int(out.n_terms) == int(keep.sum())
        assert abs(float(out.loss) - np.log1p(np.exp(-0.1 * float(out.seq_logp[0] - out.seq_logp[1])))) < 1e-5
        assert gm.device_faults() == faults


POLICY = list(itertools.product([1000, 4099, 32000], ["f32", "bf16"], [0.0, 0.3], [False, True]))


@pytest.mark.parametrize("V,dtype,kl,plain", POLICY)
def test_policy_loss_and_gradient(V, dtype, kl, plain):
    """plain: without old_logp and row weights, summed; else the full form, mean and scaled.  Advantages of both signs and 0, ratios on
    both sides of the clamp."""
    torch = gc.require_gpu()
    rows = 41
    rng = np.random.default_rng(V)
    gm = tc.head_model(V)
    x, labels = tc.make_logits(rng, rows, V, dtype)
    ref = tc.Rows64(x, labels)
    f = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()
    adv = f(rng.standard_normal(rows)); adv[3] = 0.0
    old = None if plain else ref.logp.float() + f(rng.standard_normal(rows) * 0.4)
    refp = ref.logp.float() + f(rng.standard_normal(rows) * 0.5)
    weight = None if plain else f(rng.uniform(0, 2, rows))
    scale = None if plain else torch.tensor([0.5], device="cuda")
    out = tc.fresh_out(gm, rows, dtype)
    gm.policy_loss(x, labels, adv, out, old_logp=old, ref_logp=refp, clip_low=0.2, clip_high=0.3, kl_coef=kl, row_weight=weight, mean=not plain,
                   grad_scale=scale)
    torch.cuda.synchronize()
    ref.check_logp(out.row_logp)
    A = adv.double()
    q = torch.ones_like(ref.logp) if plain else torch.exp(ref.logp - old.double())
    lo, hi = float(np.float32(1) - np.float32(0.2)), float(np.float32(1) + np.float32(0.3))
    u, c = q * A, q.clamp(lo, hi) * A
    clipped = ref.keep & (u > c)
    gap = refp.double() - ref.logp
    k = float(np.float32(kl))
    w = torch.ones_like(u) if plain else weight.double()
    term = w * (-torch.minimum(u, c) + k * (torch.expm1(gap) - gap))
    slope = -w * (torch.where(clipped, 0 * u, u) + k * torch.expm1(gap))
    # logp is off by logp_tol; the terms' and the slopes' derivatives in it
    t = ref.logp_tol + 4 * U
    term_tol = w * (u.abs() + k * (torch.expm1(gap).abs() + 1) * (1 + t)) * t + term.abs() * U
    slope_tol = w * (u.abs() + k * torch.exp(gap)) * (t + 2 * U)
    zero = torch.zeros_like(term)
    term, term_tol = torch.where(ref.keep, term, zero), torch.where(ref.keep, term_tol, zero)
    err = (out.row_loss.double() - term).abs()
    assert bool((err <= term_tol).all()), float((err - term_tol).max())
    kl_err = (out.row_kl.double() - torch.where(ref.keep, torch.expm1(gap) - gap, zero)).abs()
    assert bool((kl_err <= torch.expm1(gap).abs() * t + (torch.expm1(gap) - gap).abs() * 2 * U + t * t).all())
    n = int(ref.keep.sum())
    assert int(out.n_terms) == n and int(out.n_clipped) == int(clipped.sum())
    assert plain or 0 < int(clipped.sum()) < n
    norm = 1.0 if plain else 1.0 / n
    assert abs(float(out.loss) - float(term.sum()) * norm) <= _loss_tol(term, term_tol) * norm
    g = norm * (1.0 if plain else 0.5)
    ref.check_gradient(out.dlogits, slope * g, slope_tol * g + slope.abs() * g * 3 * U, dtype)
    assert gm.device_faults() == 0


def test_policy_without_ratio_is_weighted_likelihood_and_at_the_clamp_the_gradient_stays():
    """old_logp NULL: the gradient of -advantage * logp.  A ratio of exactly 1 with clip 0 / 0 sits on both borders: not clipped."""
    torch = gc.require_gpu()
    V, rows = 500, 8
    gm = tc.head_model(V)
    x, labels = tc.make_logits(np.random.default_rng(4), rows, V, "f32")
    adv = torch.linspace(-2, 2, rows, device="cuda")
    out = tc.fresh_out(gm, rows, "f32")
    gm.policy_loss(x, labels, adv, out, clip_low=0.0, clip_high=0.0, mean=False)
    ref = tc.Rows64(x, labels)
    ref.check_gradient(out.dlogits, -adv.double(), adv.double().abs() * 2 * U, "f32")
    assert int(out.n_clipped) == 0 and bool((out.row_loss[ref.keep] == -adv[ref.keep]).all()) and bool((out.row_kl == 0).all())


def test_ratios_that_overflow_or_vanish():
    """A token that the old model gave (nearly) no chance: the ratio is infinite in 32 bits, not in the clamp."""
    torch = gc.require_gpu()
    V = 64
    gm = tc.head_model(V)
    x, _ = tc.make_logits(np.random.default_rng(4), 4, V, "f32")
    labels = torch.zeros(4, dtype=torch.int32, device="cuda")
    adv = torch.tensor([1.0, -1.0, 1.0, -1.0], device="cuda")
    old = torch.tensor([-200.0, 0.0, 300.0, -30.0], device="cuda")
    out = tc.fresh_out(gm, 4, "f32")
    gm.policy_loss(x, labels, adv, out, old_logp=old, mean=False)
    lp = tc.Rows64(x, labels).logp
    q = torch.exp(lp - old.double())
    want = -torch.minimum(q * adv, q.clamp(0.8, 1.2) * adv)
    assert bool(((out.row_loss.double() - want).abs() <= want.abs() * 1e-4 + 1e-7).all())
    assert bool((out.dlogits[0] == 0).all()) and bool(torch.isfinite(out.dlogits).all())


def test_policy_loss_of_tokens_that_one_of_the_models_masks():
    """-inf as this model's, the old one's or the reference's log probability: limits of the formulas, not differences of infinities."""
    torch = gc.require_gpu()
    V, inf = 64, float("inf")
    gm = tc.head_model(V)
    x, _ = tc.make_logits(np.random.default_rng(4), 4, V, "f32")
    labels = torch.full((4,), 9, dtype=torch.int32, device="cuda")
    x[0, 9] = -inf                                                     # ratio 0, KL infinite
    adv = torch.tensor([1.0, 1.0, 1.0, -1.0], device="cuda")
    old = torch.tensor([-2.0, -inf, -2.0, -2.0], device="cuda")        # ratio infinite: clipped
    ref = torch.tensor([-1.0, -1.0, -inf, -1.0], device="cuda")        # KL infinite, its slope the coefficient
    out = tc.fresh_out(gm, 4, "f32")
    gm.policy_loss(x, labels, adv, out, old_logp=old, ref_logp=ref, mean=False)
    lp = tc.Rows64(x, labels).logp
    assert float(out.row_logp[0]) == -inf and float(out.row_loss[0]) == 0.0 and bool((out.dlogits[0] == 0).all()) and float(out.row_kl[0]) == inf
    assert float(out.row_loss[1]) == -float(np.float32(1) + np.float32(0.2)) and bool((out.dlogits[1] == 0).all()) and int(out.n_clipped) >= 1
    assert float(out.row_kl[2]) == inf and bool(torch.isfinite(out.row_loss[1:]).all()) and bool(torch.isfinite(out.dlogits).all())
    gm.policy_loss(x, labels, adv, out, old_logp=torch.where(old == -inf, -2.0, old), ref_logp=ref, kl_coef=0.5, mean=False)
    q = torch.exp(lp[2] + 2.0)
    want = -float(q * adv[2]) * (1.0 if float(q) <= 1.2 else 0.0) + 0.5
    assert float(out.row_loss[0]) == inf and float(out.row_loss[2]) == inf
    assert abs(float(out.dlogits[2, 9]) - want * (1 - float(torch.exp(lp[2])))) <= 1e-5 * abs(want)


PREF = [  # V, sequence lengths, rows in front, rows behind
    (1000, [1, 1], 0, 0), (1000, [0, 5], 0, 0), (1000, [0, 0, 3, 4], 2, 3), (32000, [24, 19], 0, 2),
    (4099, [7, 130, 64, 1, 33, 65, 2, 0], 1, 0), (50, list(np.arange(66) % 9), 0, 5), (131079, [3, 2], 0, 0),
    # on both sides of what one launch does for the pairs as well: rows, pairs; every width of the launch behind it
    (1000, [130, 120], 3, 3), (1000, [130, 121], 3, 3), (1000, [700, 600], 0, 3), (300, [5] * 16, 0, 1), (300, [5] * 18, 0, 1), (4100, [600, 700], 1, 2), (20000, [530, 511], 0, 0),
    (40, [0] * 40 + [3] * 100, 0, 0)]


@pytest.mark.parametrize("average,smoothing,with_ref,mean", [(False, 0.0, True, True), (True, 0.2, False, False)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,lens,front,behind", PREF)
def test_preference_loss_and_gradient(V, lens, front, behind, dtype, average, smoothing, with_ref, mean):
    torch = gc.require_gpu()
    rng = np.random.default_rng(V + len(lens))
    rows, S, P = front + int(sum(lens)) + behind, len(lens), len(lens) // 2
    gm = tc.head_model(V)
    x, labels = tc.make_logits(rng, rows, V, dtype)
    ref = tc.Rows64(x, labels)
    start = front + np.concatenate([[0], np.cumsum(lens)])
    seq_ref = torch.from_numpy((rng.standard_normal(S) * 4 - 10).astype(np.float32)).cuda() if with_ref else None
    scale = torch.tensor([1.5], device="cuda") if mean else None
    beta, margin = 0.3, 0.4
    out = tc.fresh_out(gm, rows, dtype, pairs=P)
    gm.preference_loss(x, labels, torch.from_numpy(start.astype(np.int32)).cuda(), out, ref_logp=seq_ref, beta=beta, margin=margin, smoothing=smoothing,
                       average=average, mean=mean, grad_scale=scale)
    torch.cuda.synchronize()
    ref.check_logp(out.row_logp)
    d = lambda v: float(np.float32(v))
    tot, tol, cnt = (torch.zeros(S, dtype=torch.float64, device="cuda") for _ in range(3))
    for s in range(S):
        r = slice(int(start[s]), int(start[s + 1]))
        tot[s], cnt[s] = ref.logp[r].sum(), ref.keep[r].sum()
        tol[s] = ((ref.logp_tol + ref.logp.abs() * U) * ref.keep)[r].sum()
    if average:
        tot, tol = tot / cnt.clamp(min=1), tol / cnt.clamp(min=1)
    err = (out.seq_logp.double() - tot).abs()
    assert bool((err <= tol + tot.abs() * 2 * U).all())
    ratio = tot - (seq_ref.double() if with_ref else 0.0)
    z = d(beta) * (ratio[0::2] - ratio[1::2]) - d(margin)
    z_tol = d(beta) * (tol[0::2] + tol[1::2]) + 1e-12
    eps = d(smoothing)
    sp = torch.nn.functional.softplus
    term = (1 - eps) * sp(-z, threshold=50) + eps * sp(z, threshold=50)
    assert bool(((out.pair_loss.double() - term).abs() <= z_tol + term * 2 * U).all())
    w = 1.0 / P if mean else 1.0
    assert abs(float(out.loss) - float(term.sum()) * w) <= _loss_tol(term, z_tol + term * U) * w
    assert int(out.n_terms) == int(cnt.sum())
    slope = d(beta) * (eps * torch.sigmoid(z) - (1 - eps) * torch.sigmoid(-z)) * w * (1.5 if mean else 1.0)
    slope_tol = d(beta) * z_tol * w * 1.5 + slope.abs() * 4 * U
    c, c_tol = (torch.zeros(rows, dtype=torch.float64, device="cuda") for _ in range(2))
    for s in range(S):
        r = slice(int(start[s]), int(start[s + 1]))
        share = 1.0 / max(float(cnt[s]), 1.0) if average else 1.0
        c[r], c_tol[r] = (slope[s // 2] if s % 2 == 0 else -slope[s // 2]) * share, slope_tol[s // 2] * share
    ref.check_gradient(out.dlogits, c, c_tol, dtype)
    outside = torch.ones(rows, dtype=torch.bool, device="cuda")
    outside[int(start[0]):int(start[-1])] = False
    assert bool((out.dlogits[outside] == 0).all())
    assert gm.device_faults() == 0


def test_preference_with_far_margins_and_bad_offsets():
    """Pairs far apart (the sigmoid saturates on either side) and offsets out of range or falling: clamped, counted, nothing else hurt."""
    torch = gc.require_gpu()
    V, rows = 300, 12
    gm = tc.head_model(V)
    x, _ = tc.make_logits(np.random.default_rng(1), rows, V, "f32")
    labels = torch.arange(rows, dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 3, 6, 9, 12], dtype=torch.int32, device="cuda")
    far = torch.tensor([-5e4, 0.0, 5e4, 0.0], device="cuda")
    out = tc.fresh_out(gm, rows, "f32", pairs=2)
    gm.preference_loss(x, labels, start, out, ref_logp=far, beta=1.0, mean=False)
    assert float(out.pair_loss[0]) == 0.0 and abs(float(out.pair_loss[1]) - 5e4) < 100
    assert bool((out.dlogits[:6] == 0).all()) and bool(torch.isfinite(out.dlogits).all())
    ref = tc.Rows64(x, labels)
    c = torch.tensor([0.0] * 6 + [-1.0] * 3 + [1.0] * 3, dtype=torch.float64, device="cuda")
    ref.check_gradient(out.dlogits, c, c.abs() * 4 * U, "f32")
    for bad in ([-4, 3, 6, 9, 12], [0, 3, 6, 9, 400], [0, 3, 6, 2, 12], [2 ** 31 - 1] * 5, [-2 ** 31] * 5):
        gm.preference_loss(x, labels, torch.tensor(bad, dtype=torch.int32, device="cuda"), out)
        assert gm.device_faults() > 0, bad
        assert bool(torch.isfinite(out.dlogits).all())
    gm.preference_loss(x, labels, start, out)
    assert gm.device_faults() == 0


@pytest.mark.parametrize("kind", ["sar", "policy", "pref"])
def test_gradient_against_differences(kind):
    """(L(x + h d) - L(x - h d)) / 2h along random directions, L from the library's own 32-bit terms summed in 64 bits: what a loss of rounding
    2 (|L| + 100) u allows at h, and h^2 of the third derivative."""
    torch = gc.require_gpu()
    V, rows = 200, 12
    rng = np.random.default_rng(3)
    gm = tc.head_model(V)
    x, labels = tc.make_logits(rng, rows, V, "f32")
    adv = torch.from_numpy(rng.standard_normal(rows).astype(np.float32)).cuda()
    lp = tc.Rows64(x, labels).logp.float()
    start = torch.tensor([0, 5, 9, 10, 12], dtype=torch.int32, device="cuda")

    def loss(v, out):
        if kind == "sar":
            gm.sar_loss_grad(v, labels, out)
        elif kind == "policy":
            gm.policy_loss(v, labels, adv, out, old_logp=lp - 0.05, ref_logp=lp + 0.3, kl_coef=0.2, mean=False)
        else:
            gm.preference_loss(v, labels, start, out, mean=False, beta=0.5)
        return float((out.pair_loss if kind == "pref" else out.row_loss).double().sum())

    out = tc.fresh_out(gm, rows, "f32", pairs=2)
    loss(x, out)
    grad = out.dlogits.double().clone()
    ev = tc.fresh_out(gm, rows, pairs=2)  # no gradient asked for: the loss alone
    h = 2.0 ** -6
    for i in range(6):
        d = torch.from_numpy(rng.standard_normal((rows, V)).astype(np.float32)).cuda()
        num = (loss(x + h * d, ev) - loss(x - h * d, ev)) / (2 * h)
        want = float((grad * d).sum())
        assert abs(num - want) <= 12 * 300 * U / h + 40 * h * h, (i, num, want)


@pytest.mark.parametrize("V,rows", [(32000, 40), (1000, 700), (131079, 3)])
def test_same_bits_twice_and_on_another_stream_and_in_a_graph(V, rows):
    """Each loss and the clipping: eager twice, on a side stream, and captured and replayed with inputs that change between the replays."""
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    rng = np.random.default_rng(8)
    gm = tc.head_model(V)
    data = [tc.make_logits(rng, rows, V, "bf16") for _ in range(3)]
    x, labels = data[0][0].clone(), data[0][1].clone()
    adv = torch.from_numpy(rng.standard_normal(rows).astype(np.float32)).cuda()
    start = torch.tensor([0, rows // 4, rows // 2, rows - 1, rows], dtype=torch.int32, device="cuda")
    head = torch.zeros(V, 3, device="cuda")

    def calls(outs, gset):
        gm.sar_loss_grad(x, labels, outs[0], mean=True)
        gm.policy_loss(x, labels, adv, outs[1])
        gm.preference_loss(x, labels, start, outs[2])
        gm.grad_clip(gset, 0.01)

    def make():
        outs = [tc.fresh_out(gm, rows, "bf16", pairs=2) for _ in range(3)]
        return outs, binding.GradSet(gm, [o.dlogits for o in outs], [torch.empty(rows, V, device="cuda") for _ in outs])

    def values(outs, gset):
        torch.cuda.synchronize()
        return [t.clone() for o in outs for t in (o.loss, o.dlogits, o.row_logp)] + [gset.norm.clone()] + [o.clone() for o in gset.outs]

    def same(a, b):
        return all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(a, b))

    eager, again, side, graphed = make(), make(), make(), make()
    calls(*eager), calls(*again)
    want = values(*eager)
    assert same(want, values(*again))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        calls(*side)
    stream.synchronize()
    assert same(want, values(*side))
    with torch.cuda.stream(stream):
        calls(*graphed)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls(*graphed)
    for i in (1, 2, 0, 1):
        x.copy_(data[i][0]); labels.copy_(data[i][1])
        for o in graphed[0]:
            tc.spoil(o.dlogits), tc.spoil(o.loss), tc.spoil(o.work[4:])
        tc.spoil(graphed[1].norm)
        g.replay()
        calls(*eager)
        assert same(values(*eager), values(*graphed)), i
        head.zero_()


def test_two_calls_at_once_and_two_graphs_in_turn_with_buffers_of_their_own():
    """Two streams with a LossOut each, many times over, and two captured graphs replayed on them: the bits of a call by itself."""
    torch = gc.require_gpu()
    V, rows = 32000, 40
    gm = tc.head_model(V)
    rng = np.random.default_rng(21)
    data = [tc.make_logits(rng, rows, V, "f32") for _ in range(2)]
    adv = torch.from_numpy(rng.standard_normal(rows).astype(np.float32)).cuda()
    start = torch.tensor([0, 9, 20, 31, 40], dtype=torch.int32, device="cuda")

    def call(i, out, kind):
        x, labels = data[i]
        if kind == "sar":
            gm.sar_loss_grad(x, labels, out, mean=True)
        elif kind == "policy":
            gm.policy_loss(x, labels, adv, out)
        else:
            gm.preference_loss(x, labels, start, out)

    def bits(out):
        return [t.clone().view(torch.uint8) for t in (out.loss, out.row_logp, out.dlogits, out.n_terms)]

    for kind in ("sar", "policy", "pref"):
        want = []
        for i in range(2):
            out = tc.fresh_out(gm, rows, "f32", pairs=2)
            call(i, out, kind)
            torch.cuda.synchronize()
            want.append(bits(out))
        outs = [tc.fresh_out(gm, rows, "f32", pairs=2) for _ in range(2)]
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(20):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    call(i, outs[i], kind)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for i in range(2) for a, b in zip(want[i], bits(outs[i]))), kind
        graphs = []
        for i in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                call(i, outs[i], kind)
            graphs.append(g)
        for _ in range(3):
            for o in outs:
                tc.spoil(o.dlogits), tc.spoil(o.loss)
            torch.cuda.synchronize()
            for _ in range(5):
                for i in range(2):
                    with torch.cuda.stream(streams[i]):
                        graphs[i].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for i in range(2) for a, b in zip(want[i], bits(outs[i]))), kind


def test_one_set_of_buffers_for_calls_of_every_kind():
    """A LossOut that goes from call to call, loss to loss and back, with and without the mean: what a fresh one gives, bit for bit."""
    torch = gc.require_gpu()
    V = 1000
    gm = tc.head_model(V)
    rng = np.random.default_rng(5)
    for rows in (30, 400):  # added up by the rows themselves, and by a launch behind them
        x, labels = tc.make_logits(rng, rows, V, "bf16")
        adv = torch.from_numpy(rng.standard_normal(rows).astype(np.float32)).cuda()
        start = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device="cuda")
        calls = [lambda o: gm.sar_loss_grad(x, labels, o, mean=True), lambda o: gm.preference_loss(x, labels, start, o),
                 lambda o: gm.policy_loss(x, labels, adv, o, mean=False), lambda o: gm.sar_loss_grad(x, labels, o), lambda o: gm.policy_loss(x, labels, adv, o)]
        one = tc.fresh_out(gm, rows, "bf16", pairs=1)
        for i in (0, 1, 2, 3, 4, 1, 0, 4, 4):
            new = tc.fresh_out(gm, rows, "bf16", pairs=1)
            calls[i](one), calls[i](new)
            torch.cuda.synchronize()
            assert all(torch.equal(getattr(one, n), getattr(new, n)) for n in ("loss", "n_terms", "row_logp", "dlogits")), (rows, i)
            assert bool((one.work[:4] == 0).all()), "the arrival count"


@pytest.mark.parametrize("V,rows", [(1000, 1), (1000, 30), (1000, 900), (32000, 200), (131079, 3)])
def test_loss_without_gradient_and_without_what_may_be_left_out(V, rows):
    """dlogits NULL: the loss, terms and counts of the call with a gradient, bit for bit.  row_kl, n_clipped and seq_logp NULL: the rest as it was."""
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    gm = tc.head_model(V)
    rng = np.random.default_rng(rows)
    x, labels = tc.make_logits(rng, rows, V, "f32")
    adv = torch.from_numpy(rng.standard_normal(rows).astype(np.float32)).cuda()
    start = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device="cuda")
    full, bare = tc.fresh_out(gm, rows, "f32", pairs=1), tc.fresh_out(gm, rows, pairs=1)
    for mean in (False, True):
        for call, names in ((lambda o: gm.sar_loss_grad(x, labels, o, mean=mean), ("loss", "n_terms", "row_loss", "row_logp")),
                            (lambda o: gm.policy_loss(x, labels, adv, o, old_logp=adv - 7, ref_logp=adv - 8, kl_coef=0.1, mean=mean),
                             ("loss", "n_terms", "row_loss", "row_logp", "row_kl", "n_clipped")),
                            (lambda o: gm.preference_loss(x, labels, start, o, mean=mean), ("loss", "n_terms", "row_logp", "pair_loss", "seq_logp"))):
            call(full), call(bare)
            torch.cuda.synchronize()
            for n in names:
                assert torch.equal(getattr(full, n), getattr(bare, n)), n
    grad = full.dlogits.clone()
    tc.spoil(full.dlogits)
    io = gm._loss_io(x, labels, full, None, True)
    p = binding.SpacePreferenceParams(start.data_ptr(), None, full.pair_loss.data_ptr(), None, 1, 0, 0.1, 0.0, 0.0)
    assert gm.lib.space_preference_loss(gm.ctx, C.byref(io), C.byref(p), binding._stream()) == 0
    torch.cuda.synchronize()
    assert torch.equal(full.dlogits, grad) and torch.equal(full.loss, bare.loss)
    gm.policy_loss(x, labels, adv, bare)
    p = binding.SpacePolicyParams(adv.data_ptr(), None, None, None, None, None, 0.2, 0.2, 0.0)
    assert gm.lib.space_policy_loss(gm.ctx, C.byref(io), C.byref(p), binding._stream()) == 0
    torch.cuda.synchronize()
    assert torch.equal(full.loss, bare.loss) and torch.equal(full.row_loss, bare.row_loss)


def test_rows_and_gradients_beyond_32_bit_offsets():
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    V, rows, stride = 1001, 70, (1 << 26) + 3  # 4.7 G elements from the first row to the last
    gm = tc.head_model(V)
    x, labels = tc.make_logits(np.random.default_rng(9), rows, V, "bf16")
    dense = tc.fresh_out(gm, rows, "bf16", pairs=1)
    big = torch.zeros(rows * stride, dtype=torch.bfloat16, device="cuda")
    far = big.view(rows, stride)[:, 17:17 + V]
    start = torch.tensor([0, 30, 70], dtype=torch.int32, device="cuda")
    out = tc.fresh_out(gm, rows, dlogits=far, pairs=1)
    for call in (lambda a, o: gm.sar_loss_grad(a, labels, o), lambda a, o: gm.preference_loss(a, labels, start, o)):
        far.copy_(x)
        call(x, dense)
        call(far, out)  # in place
        torch.cuda.synchronize()
        assert torch.equal(far, dense.dlogits) and torch.equal(out.loss, dense.loss)
    del out, far, big
    g = torch.ones((1 << 32) + 7, dtype=torch.bfloat16, device="cuda")
    gs = binding.GradSet(gm, [g])
    want = float((1 << 32) + 7) ** 0.5
    assert abs(float(gm.grad_norm(gs)) - want) <= want * U * 1.001
    gm.grad_clip(gs, 1.0, norm=torch.tensor([4.0], device="cuda"))
    for part in g.split(1 << 30):
        assert bool((part == 0.25).all())


# ------------------------------------------------------------------------------- norm and clipping

def _norm64(grads):
    return float(sum((g.double() ** 2).sum() for g in grads)) ** 0.5


def _make_grads(rng, sizes, types, std=1.0):
    import torch
    return [torch.from_numpy((rng.standard_normal(n) * std).astype(np.float32)).cuda().to(tc.torch_type(types[i % len(types)])) for i, n in enumerate(sizes)]


@pytest.mark.parametrize("types", [["f32"], ["bf16"], ["f32", "bf16"]])
@pytest.mark.parametrize("sizes", [[1], [0, 5, 0], [1, 2, 3, 4, 5, 6, 7, 8, 9], [8191, 8192, 8193], [100003, 1, 16384], list(range(300)), [0],
                                   [(1 << 22) + 5, 64, (1 << 20) + 1], [40000] * 230])
def test_gradient_norm_and_clipping(sizes, types):
    """Lengths around a chunk, none, many tensors (several launches); clipped into outputs of either type, in place, and not clipped.
    norm: one rounding to 32 bits (u) of a 64-bit sum; scale: the quotient's rounding and the norm's; product: one more; output rounding."""
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    gm = tc.head_model(40)
    grads = _make_grads(np.random.default_rng(len(sizes)), sizes, types)
    want = _norm64(grads)
    for out_types, max_norm in ((["bf16", "f32"], 0.37), (["f32"], 1e9), (None, 0.37), (None, 1e9)):
        src = [g.clone() for g in grads]
        outs = None if out_types is None else [tc.spoil(torch.empty_like(g, dtype=tc.torch_type(out_types[i % len(out_types)]))) for i, g in enumerate(src)]
        gs = binding.GradSet(gm, src, outs)
        tc.spoil(gs.norm), tc.spoil(gs.work[2:])
        norm = float(gm.grad_clip(gs, max_norm))
        assert abs(norm - want) <= want * U * 1.001
        limit = float(np.float32(max_norm))
        scale = limit / want if want > limit else 1.0
        for g, o in zip(grads, gs.outs):
            step = tc.HALF_STEP["f32" if o.dtype == torch.float32 else "bf16"]
            err = (o.double() - g.double() * scale).abs()
            tol = g.double().abs() * scale * ((4 * U + step * (1 + 2.0 ** -6)) if scale != 1.0 else (0.0 if o.dtype == g.dtype or o.dtype == torch.float32 else step))
            assert bool((err <= tol).all())
        if outs is not None:
            assert all(torch.equal(a, b) for a, b in zip(src, grads)), "the gradients themselves were written"


def test_more_gradients_than_the_cache_holds_over_several_launches():
    """A set beyond the memory-side cache, whose border lies within one of its lists: every element is scaled once, in place and not, and the norm
    has them all.  Gradients of ones, halves and quarters: squares and sums are exact, the scale 1 / 2^k too."""
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    gm = tc.head_model(40)
    sizes = [(5 << 17) + 3 * i for i in range(190)]
    for types, value in ((["f32"], 0.5), (["f32", "bf16"], 1.0), (["bf16"], 0.25)):
        grads = [torch.full((n,), value, dtype=tc.torch_type(types[i % len(types)]), device="cuda") for i, n in enumerate(sizes)]
        want = value * sum(sizes) ** 0.5
        outs = [torch.zeros_like(g) for g in grads]
        gs = binding.GradSet(gm, grads, outs)
        assert abs(float(gm.grad_norm(gs)) - want) <= want * U * 1.001
        gm.grad_clip(gs, 1.0, norm=torch.tensor([4.0], device="cuda"))
        assert all(bool((o == value / 4).all()) for o in outs) and all(bool((g == value).all()) for g in grads)
        gm.grad_clip(binding.GradSet(gm, grads), 1.0, norm=torch.tensor([2.0], device="cuda"))
        assert all(bool((g == value / 2).all()) for g in grads)


def test_norm_neither_overflows_nor_vanishes_and_what_is_not_finite_is_left():
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    gm = tc.head_model(40)
    for scale in (1e30, 1e-30):
        g = torch.full((10000,), scale, device="cuda")
        want = 100 * float(np.float32(scale))
        assert abs(float(gm.grad_norm(binding.GradSet(gm, [g]))) - want) <= want * U * 1.001
    g = torch.full((10,), 3e38, device="cuda")  # the norm itself is beyond 32 bits
    gs = binding.GradSet(gm, [g])
    assert float(gm.grad_clip(gs, 1.0)) == float("inf") and bool((g == 3e38).all())
    for bad in (float("nan"), float("inf")):
        a, b = torch.ones(5000, device="cuda"), torch.ones(77, device="cuda", dtype=torch.bfloat16)
        a[4321] = bad
        keep = a.clone()
        n = float(gm.grad_clip(binding.GradSet(gm, [b, a]), 0.5))
        assert not np.isfinite(n) and torch.equal(a.view(torch.int32), keep.view(torch.int32)) and bool((b == 1).all())
    # a norm of the caller's (summed over processes), and a limit of 0
    a = torch.ones(100, device="cuda")
    gs = binding.GradSet(gm, [a])
    gm.grad_clip(gs, 1.0, norm=torch.tensor([4.0], device="cuda"))
    assert bool((a == 0.25).all())
    gm.grad_clip(gs, 0.0)
    assert bool((a == 0).all())
    assert float(gm.grad_norm(binding.GradSet(gm, []))) == 0.0


def test_gradients_at_any_alignment_and_order_of_dimensions_with_nothing_written_around_them():
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    gm = tc.head_model(40)
    for t, off_g, off_o in itertools.product((torch.float32, torch.bfloat16), (0, 1, 3), (0, 1, 2)):
        buf, dst = torch.full((9000,), 2.0, dtype=t, device="cuda"), torch.full((9000,), 9.0, dtype=t, device="cuda")
        g, o = buf[off_g:off_g + 8500].view(85, 100).t(), dst[off_o:off_o + 8500].view(85, 100).t()
        gm.grad_clip(binding.GradSet(gm, [g], [o]), 1.0)
        torch.cuda.synchronize()
        want = 2.0 / (2.0 * 8500 ** 0.5)
        assert bool(((o.double() - want).abs() <= want * (4 * U + (U if t == torch.float32 else 2.0 ** -8))).all())
        o.fill_(9.0)
        assert bool((dst == 9.0).all()) and bool((buf == 2.0).all())
    with pytest.raises(AssertionError):
        binding.GradSet(gm, [torch.ones(4, 6, device="cuda")[:, :3]])
    with pytest.raises(AssertionError):
        binding.GradSet(gm, [torch.ones(4, 6, device="cuda")], [torch.ones(6, 4, device="cuda").t()])


# ------------------------------------------------------------------------------- refusals

def _io(gm, rows=4, V=100):
    import torch
    from paper_2402_11809_amd import binding
    x = torch.zeros(rows, V, device="cuda")
    labels = torch.zeros(rows, dtype=torch.int32, device="cuda")
    out = binding.LossOut(gm, rows, grad_dtype=torch.float32, pairs=2)
    return gm._loss_io(x, labels, out, None, True), (x, labels, out)


def test_refusals_of_the_losses():
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    E = binding.SPACE_EINVAL
    gm = tc.head_model(100)
    f = torch.zeros(8, device="cuda")
    start = torch.zeros(5, dtype=torch.int32, device="cuda")
    pol = lambda **kw: binding.SpacePolicyParams(**dict(dict(advantages=f.data_ptr(), clip_low=0.2, clip_high=0.2), **kw))
    prf = lambda **kw: binding.SpacePreferenceParams(**dict(dict(seq_start=start.data_ptr(), pair_loss=f.data_ptr(), pairs=2, beta=0.1), **kw))

    def rc(io, which=("sar", "policy", "pref"), p=None):
        codes = set()
        if "sar" in which:
            codes.add(gm.lib.space_sar_loss_grad(gm.ctx, io, None))
        if "policy" in which:
            codes.add(gm.lib.space_policy_loss(gm.ctx, io, C.byref(p or pol()), None))
        if "pref" in which:
            codes.add(gm.lib.space_preference_loss(gm.ctx, io, C.byref(p or prf()), None))
        assert len(codes) == 1, codes
        return codes.pop()

    io, keep = _io(gm)
    assert rc(C.byref(io)) == 0 and rc(None) == E
    for field, value in [("logits", None), ("labels", None), ("loss", None), ("n_terms", None), ("row_logp", None), ("work", None), ("rows", 0), ("rows", -1),
                         ("logits_stride", 99), ("dlogits_stride", 99), ("logits_stride", 1 << 62), ("dlogits_stride", 1 << 62), ("dtype", 2), ("dtype", -1),
                         ("logits", lambda io: io.logits + 2), ("dlogits", lambda io: io.dlogits + 1), ("work", lambda io: io.work + 4),
                         ("dlogits", lambda io: io.logits + 4), ("dlogits", lambda io: io.logits + 400), ("dlogits_stride", 101)]:
        io, keep = _io(gm)
        setattr(io, field, value(io) if callable(value) else value)
        if (field, value) == ("dlogits_stride", 101):
            io.dlogits = io.logits
        assert rc(C.byref(io)) == E, (field, value)
        assert gm.lib.space_last_error(gm.ctx)
    for field in ("labels", "loss", "n_terms", "row_logp", "row_loss", "grad_scale"):  # on 4 bytes
        io, keep = _io(gm)
        setattr(io, field, (getattr(io, field) or f.data_ptr()) + 2)
        assert rc(C.byref(io)) == E, field
    io, keep = _io(gm)
    io.rows = 1 << 22
    assert rc(C.byref(io)) == binding.SPACE_ESHAPE
    io, keep = _io(gm)
    assert rc(C.byref(io), ("policy",), pol(old_logp=f.data_ptr() + 1)) == E and rc(C.byref(io), ("pref",), prf(seq_start=start.data_ptr() + 2)) == E
    assert rc(C.byref(io), ("pref",), prf(pairs=1 << 22)) == binding.SPACE_ESHAPE
    io, keep = _io(gm)
    io.row_loss = None
    assert rc(C.byref(io), ("sar", "policy")) == E and rc(C.byref(io), ("pref",)) == 0
    io, keep = _io(gm)
    nan, inf = float("nan"), float("inf")
    for bad in (dict(advantages=None), dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_low=nan), dict(clip_high=-0.1), dict(clip_high=inf), dict(clip_high=nan),
                dict(kl_coef=-1.0, ref_logp=f.data_ptr()), dict(kl_coef=nan, ref_logp=f.data_ptr()), dict(kl_coef=0.1)):
        assert rc(C.byref(io), ("policy",), pol(**bad)) == E, bad
    for bad in (dict(seq_start=None), dict(pair_loss=None), dict(pairs=0), dict(pairs=-3), dict(beta=0.0), dict(beta=nan), dict(beta=inf), dict(margin=inf),
                dict(margin=nan), dict(smoothing=-0.1), dict(smoothing=1.5), dict(smoothing=nan)):
        assert rc(C.byref(io), ("pref",), prf(**bad)) == E, bad
    assert gm.lib.space_policy_loss(gm.ctx, C.byref(io), None, None) == E and gm.lib.space_preference_loss(gm.ctx, C.byref(io), None, None) == E
    assert gm.lib.space_sar_loss_grad(None, C.byref(io), None) == E
    x, labels, out = keep
    for bad in (lambda: gm.sar_loss_grad(x.half(), labels, out), lambda: gm.sar_loss_grad(x[:, :50], labels, out), lambda: gm.sar_loss_grad(x, labels.long(), out),
                lambda: gm.sar_loss_grad(x.bfloat16(), labels, out), lambda: gm.sar_loss_grad(x.cpu(), labels, out), lambda: gm.policy_loss(x, labels, f, out),
                lambda: gm.preference_loss(x, labels, start[:3], out), lambda: gm.sar_loss_grad(x, labels, out, grad_scale=f)):
        with pytest.raises(AssertionError):
            bad()
    torch.cuda.synchronize()
    assert gm.device_faults() == 0


def test_refusals_of_the_gradient_list():
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    E = binding.SPACE_EINVAL
    gm = tc.head_model(40)
    buf = torch.ones(1000, device="cuda")
    norm, work = torch.zeros(1, device="cuda"), torch.zeros(binding.SPACE_GRAD_WORK, dtype=torch.float64, device="cuda")
    p = buf.data_ptr()

    def rc(entries, max_norm=1.0, n=None):
        arr = (binding.SpaceGradTensor * max(len(entries), 1))(*[binding.SpaceGradTensor(*e) for e in entries])
        n = len(entries) if n is None else n
        return (gm.lib.space_grad_norm(gm.ctx, arr, n, norm.data_ptr(), work.data_ptr(), None),
                gm.lib.space_grad_clip(gm.ctx, arr, n, norm.data_ptr(), max_norm, None))

    assert rc([(p, p, 10, 0, 0), (p + 40, p + 40, 10, 0, 0), (None, None, 0, 0, 0)]) == (0, 0)
    assert rc([]) == (0, 0) and rc([], n=-1) == (E, E)
    for bad in ([(None, p, 5, 0, 0)], [(p, p, -1, 0, 0)], [(p, p, 5, 2, 0)], [(p + 2, p + 400, 5, 0, 0)], [(p + 1, p + 400, 5, 1, 0)], [(p, p, 1 << 62, 0, 0)]):
        assert rc(bad) == (E, E), bad
    for bad in ([(p, None, 5, 0, 0)], [(p, p + 402, 5, 0, 0)], [(p, p + 400, 5, 0, 3)],
                [(p, p, 10, 0, 0), (p, p, 10, 0, 0)],               # the same gradient twice
                [(p, p, 10, 0, 0), (p + 36, p + 36, 10, 0, 0)],     # tensors that share an element
                [(p, p + 4, 10, 0, 0)], [(p, p, 10, 0, 1)], [(p, p, 10, 1, 0)],  # an output on a part of its gradient
                [(p, p + 400, 10, 0, 0), (p + 404, p + 800, 1, 0, 0)]):          # an output on another gradient
        assert rc(bad) == (0, E), bad
    assert rc([(p, p + 400, 10, 0, 0), (p, p + 800, 10, 0, 1)]) == (0, 0)        # one gradient read twice
    for limit in (-1.0, float("nan")):
        assert rc([(p, p, 10, 0, 0)], limit)[1] == E
    one = (binding.SpaceGradTensor * 1)(binding.SpaceGradTensor(p, p, 10, 0, 0))
    for call in ((gm.lib.space_grad_norm, (gm.ctx, one, 1, None, work.data_ptr(), None)), (gm.lib.space_grad_norm, (gm.ctx, one, 1, norm.data_ptr(), None, None)),
                 (gm.lib.space_grad_norm, (None, one, 1, norm.data_ptr(), work.data_ptr(), None)), (gm.lib.space_grad_clip, (gm.ctx, one, 1, None, 1.0, None)),
                 (gm.lib.space_grad_norm, (gm.ctx, None, 1, norm.data_ptr(), work.data_ptr(), None)), (gm.lib.space_grad_clip, (gm.ctx, None, 1, norm.data_ptr(), 1.0, None))):
        assert call[0](*call[1]) == E
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------- together

def test_loss_of_a_step_then_policy_gradient_on_its_logits():
    """A block is decoded by Model.step; its logits go through the finetuning loss (the same terms as space_sar_loss, to rounding) and the policy loss."""
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding, layout as lo
    from space_inputs import SHAPES, all_weights
    shape = SHAPES["tiny"]
    gm = gc.make_gpu_model(shape, all_weights(shape, seed=0), max_batch=1, max_rows=36)
    k, spec = 5, lo.paper_layout(5)
    kv = gm.kv_cache(1, 64)
    out = binding.StepOut(gm, 1, spec.n_rows, k)
    toks = torch.randint(0, shape.vocab, (1, spec.n_rows), dtype=torch.int32, device="cuda")
    gm.step(toks, gm.layout(spec), kv, out)
    logits, labels = out.logits[0], out.argmax[0].clone()
    labels[1::6] = -1
    plain = torch.empty(spec.n_rows, device="cuda")
    loss, n = gm.sar_loss(logits, labels, plain)
    lg = tc.fresh_out(gm, spec.n_rows, "f32")
    gm.sar_loss_grad(logits, labels, lg)
    ref = tc.Rows64(logits, labels)
    ref.check_logp(lg.row_logp)
    assert int(n) == int(lg.n_terms) and bool(((plain - lg.row_loss).abs().double() <= 2 * ref.logp_tol).all())
    one = torch.ones(spec.n_rows, dtype=torch.float64, device="cuda")
    ref.check_gradient(lg.dlogits, -one, 0 * one, "f32")
    pl = tc.fresh_out(gm, spec.n_rows, "f32")
    gm.policy_loss(logits, labels, -torch.ones(spec.n_rows, device="cuda"), pl, old_logp=lg.row_logp, mean=False)
    ref.check_gradient(pl.dlogits, one, 4 * U * one + 2 * ref.logp_tol, "f32")
    assert gm.device_faults() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_training_step_of_the_head(dtype):
    """Hidden states -> logits -> loss with gradient -> gradients of the head and of the hidden states (the caller's products) -> norm and
    clipping, for each loss, against the same in 64 bits.  The products are torch's in 32 bits on what the kernels returned, so what is
    compared behind them is bounded by the gradient's own rounding: each product's error by its absolute values."""
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    V, d, rows = 1003, 64, 24
    t = tc.torch_type(dtype)
    rng = np.random.default_rng(11)
    gm = tc.head_model(V)
    f = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()
    h, W = f(rng.standard_normal((rows, d))), f(rng.standard_normal((V, d)) * 0.3)
    labels = torch.from_numpy(rng.integers(0, V, rows).astype(np.int32)).cuda()
    labels[:3] = -1
    adv, start = f(rng.standard_normal(rows)), torch.tensor([0, 6, 12, 18, 24], dtype=torch.int32, device="cuda")
    logits = (h.double() @ W.double().t()).to(t)  # what the losses are given; the 64-bit form starts from the same
    out = tc.fresh_out(gm, rows, dtype, pairs=2)
    for kind in ("sar", "policy", "pref"):
        x = logits.double().requires_grad_(True)
        keep = labels >= 0
        lp = torch.log_softmax(x, 1).gather(1, labels.long().clamp(min=0)[:, None])[:, 0] * keep
        if kind == "sar":
            gm.sar_loss_grad(logits, labels, out, mean=True)
            loss = -lp.sum() / keep.sum()
        elif kind == "policy":
            gm.policy_loss(logits, labels, adv, out)
            loss = -(torch.exp(lp - lp.detach()) * adv.double() * keep).sum() / keep.sum()
        else:
            gm.preference_loss(logits, labels, start, out)
            s = torch.stack([lp[int(a):int(b)].sum() for a, b in zip(start[:-1], start[1:])])
            loss = torch.nn.functional.softplus(-float(np.float32(0.1)) * (s[0::2] - s[1::2])).mean()
        loss.backward()
        assert abs(float(out.loss) - float(loss.detach())) <= 300 * U * max(1.0, abs(float(loss.detach())))
        dW, dh = out.dlogits.float().t() @ h, out.dlogits.float() @ W
        wantW, wanth = x.grad.t() @ h.double(), x.grad @ W.double()
        # relative error of every gradient element, and of a 32-bit product of at most 1003 terms
        rel = tc.HALF_STEP[dtype] * 1.02 + 400 * U + 1003 * U
        assert bool(((dW - wantW).abs() <= rel * (x.grad.abs().t() @ h.double().abs()) + 1e-12).all())
        assert bool(((dh - wanth).abs() <= rel * (x.grad.abs() @ W.double().abs()) + 1e-12).all())
        gs = binding.GradSet(gm, [dW, dh])
        a, b = dW.clone(), dh.clone()
        norm = float(gm.grad_clip(gs, 0.05))
        want = _norm64([a, b])
        assert abs(norm - want) <= want * U * 1.001
        scale = min(1.0, float(np.float32(0.05)) / want)
        for got, was in ((dW, a), (dh, b)):
            assert bool(((got.double() - was.double() * scale).abs() <= was.double().abs() * 4 * U).all())
        assert abs(_norm64([dW, dh]) - min(want, float(np.float32(0.05)))) <= want * 4 * U
    assert gm.device_faults() == 0


def test_lowest_value_as_a_mask_in_the_loss_without_gradient():
    """space_sar_loss on logits masked with the lowest 32-bit number: the terms of the same logits masked with -inf, bit for bit."""
    torch = gc.require_gpu()
    V, rows = 3000, 6
    gm = tc.head_model(V)
    x, labels = tc.make_logits(np.random.default_rng(2), rows, V, "f32")
    labels.fill_(7)
    mask = torch.rand(rows, V, device="cuda") < 0.5
    mask[:, 7] = False
    got = [torch.empty(rows, device="cuda") for _ in range(2)]
    for value, t in zip((float("-inf"), torch.finfo(torch.float32).min), got):
        gm.sar_loss(x.masked_fill(mask, value), labels, t)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(got[0]).all()) and torch.equal(*got)


# ------------------------------------------------------------------------------- what may not overlap

def test_outputs_of_a_loss_on_its_inputs_or_on_each_other_are_refused():
    """Values of an earlier call go in as a copy: a call that gets its own outputs as inputs (whose values it would have spoiled) is refused,
    and so are two outputs, or the scratch, on the same bytes."""
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    V, rows = 100, 4
    gm = tc.head_model(V)
    x, labels = tc.make_logits(np.random.default_rng(6), rows, V, "f32")
    labels.fill_(3)
    adv = torch.tensor([1.0, -1.0, 0.5, -0.5], device="cuda")
    start = torch.tensor([0, 1, 2, 3, 4], dtype=torch.int32, device="cuda")
    out = tc.fresh_out(gm, rows, "f32", pairs=2)
    refused = lambda call: pytest.raises(binding.SpaceError, call)

    gm.policy_loss(x, labels, adv, out)
    old, ref = out.row_logp.clone(), out.row_logp - 0.5
    for kw in (dict(old_logp=out.row_logp), dict(ref_logp=out.row_logp, kl_coef=0.1), dict(old_logp=out.row_loss), dict(row_weight=out.row_kl),
               dict(old_logp=out.work[4:8]), dict(grad_scale=out.loss), dict(ref_logp=out.dlogits[1, :4])):
        refused(lambda: gm.policy_loss(x, labels, adv, out, **kw))
    refused(lambda: gm.policy_loss(x, labels, out.row_logp, out))
    refused(lambda: gm.sar_loss_grad(x, out.row_logp.view(torch.int32), out))
    refused(lambda: gm.sar_loss_grad(x, labels, out, grad_scale=out.row_loss[:1]))
    refused(lambda: gm.sar_loss_grad(out.dlogits, labels, out, grad_scale=out.dlogits[3, 99:]))
    refused(lambda: gm.preference_loss(x, labels, start, out, ref_logp=out.seq_logp))
    refused(lambda: gm.preference_loss(x, labels, start, out, ref_logp=out.row_logp))
    refused(lambda: gm.preference_loss(x, labels, start, out, grad_scale=out.pair_loss[1:]))
    for a, b in itertools.permutations(("loss", "n_terms", "row_logp", "row_loss", "work"), 2):
        io = gm._loss_io(x, labels, out, None, True)
        was = getattr(io, a)
        setattr(io, a, getattr(io, b))
        assert gm.lib.space_sar_loss_grad(gm.ctx, C.byref(io), None) == binding.SPACE_EINVAL, (a, b)
        setattr(io, a, was)
    for name in ("loss", "row_logp", "row_loss", "work"):  # an output on the logits, and on the gradient
        for place in (x, out.dlogits):
            io = gm._loss_io(x, labels, out, None, True)
            was = getattr(io, name)
            setattr(io, name, place[rows - 1, V - 4:].data_ptr())
            assert gm.lib.space_sar_loss_grad(gm.ctx, C.byref(io), None) == binding.SPACE_EINVAL, name
            setattr(io, name, was)
    assert "overlaps" in gm.lib.space_last_error(gm.ctx).decode()
    # the same with copies, or between the rows of a wider buffer, is what it was
    gm.policy_loss(x, labels, adv, out, old_logp=old - 1.0, ref_logp=ref, kl_coef=0.1)
    want = [t.clone() for t in (out.loss, out.row_loss, out.row_kl, out.dlogits)]
    assert int(out.n_clipped) == 2 and bool((out.row_kl > 0).all())
    wide = torch.zeros(rows, V + 8, device="cuda")
    wide[0, V:V + 4] = old - 1.0
    between = tc.fresh_out(gm, rows, dlogits=wide[:, :V], pairs=2)
    gm.policy_loss(x, labels, adv, between, old_logp=wide[0, V:V + 4], ref_logp=ref, kl_coef=0.1)
    assert all(torch.equal(a, b) for a, b in zip(want, (between.loss, between.row_loss, between.row_kl, between.dlogits)))
    gm.preference_loss(x, labels, start, out, ref_logp=out.seq_logp.clone())
    torch.cuda.synchronize()
    assert gm.device_faults() == 0


def test_a_norm_inside_a_clipped_gradient_is_refused():
    """Every workgroup reads the norm: an output over it would change the scale of what is clipped later.  Beside an output it may stand, and
    within a gradient that is only read."""
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    gm = tc.head_model(40)
    flat = torch.full((20001,), 2.0, device="cuda")  # a norm, then the gradients
    flat[0] = 8.0
    dst = torch.full((20001,), 3.0, device="cuda")
    for norm, grads, outs in ((flat[5:6], [flat[1:]], None), (flat[20000:], [flat[1:9000], flat[9000:]], None), (dst[7:8], [flat[1:]], [dst[1:]])):
        with pytest.raises(binding.SpaceError):
            gm.grad_clip(binding.GradSet(gm, grads, outs), 1.0, norm=norm)
    torch.cuda.synchronize()
    assert bool((flat[1:] == 2.0).all()) and bool((dst == 3.0).all())
    gm.grad_clip(binding.GradSet(gm, [flat], [dst]), 4.0, norm=flat[:1])
    assert float(dst[0]) == 4.0 and bool((dst[1:] == 1.0).all()) and float(flat[0]) == 8.0
    gm.grad_clip(binding.GradSet(gm, [flat[1:]]), 2.0, norm=flat[:1])
    assert bool((flat[1:] == 0.5).all()) and float(flat[0]) == 8.0


def test_a_norm_or_scratch_on_a_gradient_or_on_each_other_is_refused():
    """The norm inside the scratch would stay in the arrival count, the scratch inside a gradient would be read as one."""
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    gm = tc.head_model(40)
    W = binding.SPACE_GRAD_WORK
    buf = torch.zeros(3 * W, dtype=torch.float64, device="cuda")  # [gradient | scratch | norm]
    g, work, norm = buf.data_ptr(), buf[W:].data_ptr(), buf[2 * W:].data_ptr()
    buf[:W].view(torch.float32).fill_(0.5)
    one = lambda n, dtype=0: (binding.SpaceGradTensor * 2)(binding.SpaceGradTensor(g, None, n, dtype, 0), binding.SpaceGradTensor(work, None, 0, 0, 0))
    rc = lambda t, norm, work: gm.lib.space_grad_norm(gm.ctx, t, 2, norm, work, binding._stream())
    for t, a, b in ((one(2 * W), work, work), (one(2 * W), work + 8 * W - 4, work), (one(2 * W), g + 8, work), (one(2 * W + 1), norm, work),
                    (one(2 * W), norm, g + 8 * W - 8), (one(4 * W + 1, 1), norm, work), (one(4 * W + 1), work + 8 * W, work)):
        assert rc(t, a, b) == binding.SPACE_EINVAL
    torch.cuda.synchronize()
    assert bool((buf[:W].view(torch.float32) == 0.5).all()) and bool((buf[W:] == 0).all())
    for _ in range(2):
        assert rc(one(2 * W), norm, work) == 0
        torch.cuda.synchronize()
        want = 0.5 * (2 * W) ** 0.5
        assert abs(float(buf[2 * W:].view(torch.float32)[0]) - want) <= want * U * 1.001 and bool((buf[W:W + 2] == 0).all())
        assert bool((buf[:W].view(torch.float32) == 0.5).all())


# ------------------------------------------------------------------------------- what is no number, and what counts nothing

@pytest.mark.parametrize("V,rows", [(40, 7), (1000, 300), (32000, 7), (40001, 210), (131079, 7)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_are_no_number_make_all_their_terms_and_gradient_nan(V, rows, dtype):
    """Nothing but -inf, a NaN, a +inf, at the label or beside it: term, KL term, log probability and the whole gradient of the row, in the policy loss
    also where the ratio is 1 by definition and where advantage or weight is 0.  Other rows are what they are without these."""
    torch = gc.require_gpu()
    gm = tc.head_model(V)
    x, _ = tc.make_logits(np.random.default_rng(V), rows, V, dtype, lift=False)
    labels = torch.full((rows,), V // 2, dtype=torch.int32, device="cuda")
    clean = x.clone()
    x[0, :] = float("-inf"); x[1, 1] = float("nan"); x[2, V - 1] = float("inf"); x[3, V // 2] = float("nan"); x[4, V // 2] = float("inf")
    bad = torch.arange(rows, device="cuda") < 5
    ones = torch.ones(rows, device="cuda")
    zeros = torch.zeros(rows, device="cuda")
    for call, names in ((lambda a, o: gm.sar_loss_grad(a, labels, o), ("row_loss", "row_logp")),
                        (lambda a, o: gm.policy_loss(a, labels, ones, o), ("row_loss", "row_logp")),
                        (lambda a, o: gm.policy_loss(a, labels, -ones, o, old_logp=-ones, ref_logp=-ones, kl_coef=0.1, mean=False), ("row_loss", "row_logp", "row_kl")),
                        (lambda a, o: gm.policy_loss(a, labels, zeros, o, row_weight=zeros), ("row_loss", "row_logp"))):
        out, ref = tc.fresh_out(gm, rows, dtype), tc.fresh_out(gm, rows, dtype)
        call(x, out), call(clean, ref)
        torch.cuda.synchronize()
        for n in names:
            assert bool(torch.isnan(getattr(out, n)[bad]).all()), n
            assert torch.equal(getattr(out, n)[~bad], getattr(ref, n)[~bad]), n
        assert bool(torch.isnan(out.dlogits[bad]).all()) and torch.equal(out.dlogits[~bad], ref.dlogits[~bad])
        assert np.isnan(float(out.loss)) and int(out.n_terms) == rows
        bare = tc.fresh_out(gm, rows)
        call(x, bare)
        torch.cuda.synchronize()
        assert bool(torch.isnan(bare.row_loss[bad]).all()) and np.isnan(float(bare.loss))


@pytest.mark.parametrize("rows", [12, 300])  # added up by the rows, and by a launch behind them
def test_an_advantage_or_weight_of_zero_takes_infinite_factors_away(rows):
    """Ratios that are infinite (a token that the old model gave no chance, as -inf or as the lowest number) with an advantage of 0, KL terms that are
    infinite (masked now, or by the reference) with a weight of 0: nothing is contributed, as for every finite factor."""
    torch = gc.require_gpu()
    V, inf, low = 64, float("inf"), torch.finfo(torch.float32).min
    gm = tc.head_model(V)
    x, _ = tc.make_logits(np.random.default_rng(4), rows, V, "f32")
    labels = torch.full((rows,), 9, dtype=torch.int32, device="cuda")
    f = lambda *v: torch.tensor(list(v) + [1.0] * (rows - len(v)), device="cuda")
    x[4, 9] = -inf
    #      0     1    2     3     4     5     6
    adv = f(0.0, 0.0, -0.0, 1.0, 1.0, -1.0, 0.0)
    wgt = f(1.0, 1.0, 1.0, 0.0, 0.0, 0.0, 1.0)
    old = f(-inf, low, -800.0, -2.0, -2.0, -inf, -inf)
    ref = f(-2.0, -2.0, -2.0, -inf, -2.0, -2.0, -2.0)
    old[7:], ref[7:] = -2.0, -2.0
    out = tc.fresh_out(gm, rows, "f32")
    gm.policy_loss(x, labels, adv, out, old_logp=old, ref_logp=ref, row_weight=wgt, mean=False)
    torch.cuda.synchronize()
    assert bool((out.row_loss[:7] == 0).all()) and bool((out.dlogits[:7] == 0).all())
    lp = tc.Rows64(x[7:], labels[7:]).logp
    q = torch.exp(lp + 2.0)
    rest = -torch.minimum(q, q.clamp(max=float(np.float32(1) + np.float32(0.2))))
    t = 300 * U  # logp of some 10, its sum of 64 terms, the exponential: less than that, relative
    assert bool(((out.row_loss[7:].double() - rest).abs() <= t * rest.abs()).all()) and abs(float(out.loss) - float(rest.sum())) <= t * float(rest.abs().sum())
    assert int(out.n_clipped) == int((q > 1.2).sum())
    # with a KL term: its part alone where the advantage is 0, nothing where the weight is
    gm.policy_loss(x, labels, adv, out, old_logp=old, ref_logp=ref, row_weight=wgt, kl_coef=0.5, mean=False)
    torch.cuda.synchronize()
    lp = tc.Rows64(x, labels).logp
    assert bool((out.row_loss[3:6] == 0).all()) and bool((out.dlogits[3:6] == 0).all())
    for r in (0, 1, 2, 6):
        gap = -2.0 - lp[r]
        want = 0.5 * float(torch.expm1(gap) - gap)
        assert abs(float(out.row_loss[r]) - want) <= 300 * U * (abs(want) + float(gap.abs())), r
        p = torch.softmax(x[r].double(), 0)
        p[9] -= 1.0
        c = 0.5 * float(torch.expm1(gap))
        assert bool(((out.dlogits[r].double() - c * p).abs() <= 300 * U * (abs(c) + 1) * (p.abs() + U)).all()), r
    # an infinite factor that does count stays infinite
    gm.policy_loss(x, labels, -torch.ones(rows, device="cuda"), out, old_logp=old, mean=False)
    assert bool((out.row_loss[[0, 1, 2, 5, 6]] == inf).all()) and float(out.loss) == inf


# ------------------------------------------------------------------------------- calls that count and add up in launches of their own

# rows above what a call adds up by itself, for every width of the rows' kernels in both types; and on both sides of that border
LARGE = [(1000, 700, "f32"), (2048, 193, "bf16"), (2049, 193, "f32"), (4096, 260, "bf16"), (4099, 300, "f32"), (8192, 260, "f32"), (8200, 300, "f32"), (8200, 300, "bf16"),
         (20000, 1600, "f32"), (20000, 500, "bf16"), (32771, 4097, "f32"), (32771, 4097, "bf16"), (65543, 4097, "f32"), (65543, 4097, "bf16"), (131079, 4097, "bf16"),
         (1000, 192, "f32"), (1000, 193, "f32"), (32000, 976, "bf16"), (32000, 977, "bf16"), (32000, 3906, "f32"), (32000, 3907, "f32")]


def _rows_on_gpu(V, rows, dtype):
    """As tc.make_logits, drawn on the GPU: N(0, 2), labels lifted, a fifth left out."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(V + rows)
    x = torch.randn((rows, V), generator=g, device="cuda").mul_(2.0)
    labels = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    x.scatter_add_(1, labels.long()[:, None], torch.rand((rows, 1), generator=g, device="cuda") * 14.0)
    labels[torch.rand(rows, generator=g, device="cuda") < 0.2] = -1
    return x.to(tc.torch_type(dtype)), labels, lambda std: torch.randn(rows, generator=g, device="cuda") * std


@pytest.mark.parametrize("V,rows,dtype", LARGE)
def test_losses_of_many_rows_against_the_formulas(V, rows, dtype):
    """The finetuning and the policy loss, mean, scaled: terms, counts, loss and gradient, with every row's tolerance as in the tests of few rows."""
    torch = gc.require_gpu()
    gm = tc.head_model(V)
    x, labels, noise = _rows_on_gpu(V, rows, dtype)
    ref = tc.Rows64(x, labels)
    n = int(ref.keep.sum())
    assert 0 < n < rows
    scale = torch.tensor([0.5], device="cuda")
    out = tc.fresh_out(gm, rows, dtype)
    gm.sar_loss_grad(x, labels, out, mean=True, grad_scale=scale)
    torch.cuda.synchronize()
    ref.check_logp(out.row_logp)
    ref.check_logp(out.row_loss, -1.0)
    assert int(out.n_terms) == n
    total = float(ref.logp.sum())
    assert abs(float(out.loss) + total / n) <= _loss_tol(ref.logp, ref.logp_tol) / n + abs(total) / n * U
    c = torch.full_like(ref.logp, 0.5 / n)
    ref.check_gradient(out.dlogits, -c, c * 2 * U, dtype)
    del out
    adv, old, refp, weight = noise(1.0), ref.logp.float() + noise(0.4), ref.logp.float() + noise(0.5), noise(1.0).abs()
    out = tc.fresh_out(gm, rows, dtype)
    gm.policy_loss(x, labels, adv, out, old_logp=old, ref_logp=refp, clip_low=0.2, clip_high=0.3, kl_coef=0.3, row_weight=weight, mean=True, grad_scale=scale)
    torch.cuda.synchronize()
    ref.check_logp(out.row_logp)
    A, w, k = adv.double(), weight.double(), float(np.float32(0.3))
    q = torch.exp(ref.logp - old.double())
    lo, hi = float(np.float32(1) - np.float32(0.2)), float(np.float32(1) + np.float32(0.3))
    u, cl = q * A, q.clamp(lo, hi) * A
    t = ref.logp_tol + 4 * U
    gap = refp.double() - ref.logp
    # a ratio that is as near a border of the clamp as its own error goes either way: its row is left to the bound of both sides
    edge = ref.keep & (((q - lo).abs() <= q * t) | ((q - hi).abs() <= q * t))
    clipped = ref.keep & (u > cl)
    zero = torch.zeros_like(u)
    term = torch.where(ref.keep, w * (-torch.minimum(u, cl) + k * (torch.expm1(gap) - gap)), zero)
    term_tol = torch.where(ref.keep, w * (u.abs() + k * (torch.expm1(gap).abs() + 1) * (1 + t)) * t + term.abs() * U, zero)
    assert bool(((out.row_loss.double() - term).abs() <= term_tol).all())
    kl = torch.where(ref.keep, torch.expm1(gap) - gap, zero)
    assert bool(((out.row_kl.double() - kl).abs() <= torch.expm1(gap).abs() * t + kl.abs() * 2 * U + t * t).all())
    assert int(out.n_terms) == n and abs(int(out.n_clipped) - int(clipped.sum())) <= int(edge.sum()) and 0 < int(out.n_clipped) < n
    assert abs(float(out.loss) - float(term.sum()) / n) <= _loss_tol(term, term_tol) / n
    slope = -w * (torch.where(clipped, zero, u) + k * torch.expm1(gap))
    slope_tol = w * (u.abs() + k * torch.exp(gap)) * (t + 2 * U) + torch.where(edge, w * u.abs(), zero)
    ref.check_gradient(out.dlogits, slope * (0.5 / n), (slope_tol + slope.abs() * 3 * U) * (0.5 / n), dtype)
    assert gm.device_faults() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,fill", [(40, 0), (1000, 0), (1000, 130), (5003, 130), (32000, 0), (32000, 130), (131079, 0), (131079, 130)])
def test_preference_loss_of_masked_and_infinite_logits(V, fill, dtype):
    """Masks as in the finetuning loss: -inf and the type's lowest value beside the label, the label alone, a masked label in the chosen and in the
    rejected sequence, a NaN in one pair, anything in rows that do not count; in one launch behind the rows and in three (fill)."""
    torch = gc.require_gpu()
    gm = tc.head_model(V)
    t, inf = tc.torch_type(dtype), float("inf")
    start = [0, 3, 6, 8, 10, 12, 14, 16, 19, 19 + fill, 19 + 2 * fill]
    rows, y = start[-1], V // 2
    x, _ = tc.make_logits(np.random.default_rng(V), rows, V, dtype, lift=False)
    labels = torch.full((rows,), y, dtype=torch.int32, device="cuda")
    low = torch.finfo(t).min
    x[0, :y] = -inf                                       # pair 0: masks beside the label
    x[1, y + 1:] = -inf
    x[2, :] = -inf; x[2, y] = 1.5                         # the label alone
    x[3, :] = low; x[3, y] = 0.25; x[3, V - 1] = 0.25
    x[4, :] = low
    x[5, ::2] = -inf; x[5, y] = 0.0
    x[7, 1] = float("nan")                                # pair 1: a NaN
    x[13, y] = -inf                                       # pair 2: the rejected label masked
    x[14, y] = -inf                                       # pair 3: the chosen label masked
    labels[16] = -1; x[16, :] = -inf                      # rows that do not count
    labels[9] = -5; x[9, 0] = float("nan")
    labels[11] = -1; x[11, 0] = inf
    out = tc.fresh_out(gm, rows, dtype, pairs=5)
    gm.preference_loss(x, labels, torch.tensor(start, dtype=torch.int32, device="cuda"), out, beta=0.25, mean=False)
    torch.cuda.synchronize()
    fine = [r for r in range(rows) if r not in (6, 7, 8, 9)]
    ref = tc.Rows64(x[fine].nan_to_num(nan=0.0, posinf=0.0, neginf=-inf), labels[fine])
    assert bool(torch.isnan(out.dlogits[[6, 7, 8]]).all()) and np.isnan(float(out.pair_loss[1])) and np.isnan(float(out.loss)) and np.isnan(float(out.row_logp[7]))
    assert bool((out.dlogits[[9, 11, 16]] == 0).all()) and bool((out.row_logp[[9, 11, 16]] == 0).all())
    assert float(out.pair_loss[2]) == 0.0 and float(out.pair_loss[3]) == inf and float(out.seq_logp[5]) == -inf and float(out.seq_logp[6]) == -inf
    # slopes: those of pairs 2 and 3 are limits, 0 and -beta
    S = [ref.logp[[fine.index(r) for r in range(a, b)]].sum() if r0 != 1 else None for r0, a, b in zip([0, 0, 1, 1, 2, 2, 3, 3, 4, 4], start[:-1], start[1:])]
    tol = [ref.logp_tol[[fine.index(r) for r in range(a, b)]].sum() if r0 not in (1, 2, 3) else None for r0, a, b in
           zip([0, 0, 1, 1, 2, 2, 3, 3, 4, 4], start[:-1], start[1:])]
    c, c_tol = torch.zeros(len(fine), dtype=torch.float64, device="cuda"), torch.zeros(len(fine), dtype=torch.float64, device="cuda")
    for p in (0, 2, 3, 4):
        z_tol = 0.0
        slope = {2: 0.0, 3: -0.25}.get(p)
        if slope is None:
            z = 0.25 * (S[2 * p] - S[2 * p + 1])
            z_tol = 0.25 * float(tol[2 * p] + tol[2 * p + 1]) + 4 * U * float(abs(S[2 * p]) + abs(S[2 * p + 1]))
            slope = -0.25 * float(torch.sigmoid(-z))
            want = float(torch.nn.functional.softplus(-z, threshold=50))
            assert abs(float(out.pair_loss[p]) - want) <= z_tol + want * 2 * U, p
        for which, sign in ((0, 1.0), (1, -1.0)):
            for r in range(start[2 * p + which], start[2 * p + which + 1]):
                c[fine.index(r)], c_tol[fine.index(r)] = sign * slope, 0.25 * z_tol + abs(slope) * 4 * U
    ref.check_gradient(out.dlogits[fine], c, c_tol, dtype)
    assert gm.device_faults() == 0


@pytest.mark.parametrize("types", [["f32"], ["bf16", "f32"]])
@pytest.mark.parametrize("chunks", [1, 2, 17, 63, 64, 65, 66, 127, 129, 200, 319, 320, 321, 1000, 2048, 2049, 4500])
def test_norms_of_so_many_chunks(chunks, types):
    """On both sides of what takes the root in the squares' own launch and of the workgroups of a launch: norm and clipping against 64 bits, twice
    with one scratch, and in a graph that is replayed with other gradients; norm: one rounding of a 64-bit sum."""
    torch = gc.require_gpu()
    from paper_2402_11809_amd import binding
    gm = tc.head_model(40)
    g = torch.Generator(device="cuda").manual_seed(chunks)
    k = min(chunks, 7)
    sizes = [8192 * (chunks // k)] * (k - 1)
    sizes.append(8192 * (chunks - (chunks // k) * (k - 1)) - 5)
    grads = [torch.empty(n, dtype=tc.torch_type(types[i % len(types)]), device="cuda") for i, n in enumerate(sizes)]
    outs = [torch.empty(n, device="cuda") for n in sizes]
    gs = binding.GradSet(gm, grads, outs)

    def check():
        torch.cuda.synchronize()
        want = _norm64(grads)
        assert abs(float(gs.norm) - want) <= want * U * 1.001 and bool((gs.work[:2] == 0).all())
        for a, o in zip(grads, outs):
            exact = a.double() * (0.5 / want)
            assert bool(((o.double() - exact).abs() <= exact.abs() * 4 * U).all())

    def draw():
        for a in grads:
            a.copy_(torch.randn(a.shape, generator=g, device="cuda"))

    for _ in range(2):
        draw(), tc.spoil(gs.work[2:]), gm.grad_clip(gs, 0.5), check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gm.grad_clip(gs, 0.5)
    for _ in range(3):
        draw(), tc.spoil(gs.norm)
        graph.replay()
        check()
        gm.grad_clip(gs, 0.5)
        check()
