"""verify_drafts, commit_drafts, topk_distill and its gradient on the GPU in calls that the documentation allows and ordinary inputs do not make: against
64-bit restatements (draft_reference.py, distill_slope.py).  Bounds are those of test_gpu_drafts.py, where they are derived."""
import numpy as np
import pytest
import torch

import distill_slope as S
import draft_reference as R
import test_gpu_drafts as T
from test_gpu_drafts import BF, D, FF, HF, f32, f64, i32, u_of

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------- topk_distill and gradient
@pytest.mark.parametrize("dt", [FF, BF, HF])
@pytest.mark.parametrize("rows,vocab", [(4, 9), (5, 3001), (3, 40000), (320, 2000)])
@pytest.mark.parametrize("temp,high,low", [(1.0, 900.0, 100.0), (2.0 ** -6, 20.0, 8.0), (2.0 ** -6, 20.0, -8.0)])
@pytest.mark.parametrize("rest", [True, False])
def test_topk_distill_others_far_below_the_entries_have_no_gradient(dt, rows, vocab, temp, high, low, rest):
    """Others whose sum is below 2^-1000 of the row, although their logits are finite, positive and large against T; ordinary rows between them."""
    import paper_2410_03960_b200 as P
    z, _, _, weight = T.teacher(21, rows, vocab, 2, dt, temp)
    z = (z * 0.25 * temp).clone()                        # (the others lie within a few T of one another)
    ids = torch.tensor([[vocab // 2, 1]], dtype=torch.int32, device="cuda").repeat(rows, 1)
    lp = torch.log(torch.tensor([[0.25, 0.75]], device="cuda")).repeat(rows, 1)
    far = torch.arange(rows, device="cuda") % 2 == 0
    z[far] += low
    z[far, 1] = high
    z[far, vocab // 2] = high - temp
    got = T.check_distill(z, ids, lp, weight, temp, rest)
    alone = P.topk_distill_bwd(z, ids, lp, got["lse"], got["rest_lse"], weight, temperature=temp, rest=rest)
    others = torch.ones(vocab, dtype=torch.bool, device="cuda")
    others[[1, vocab // 2]] = False
    for grad in (got["grad_logits"], alone):
        assert (grad[far][:, others] == 0).all() and (grad[far][:, ~others] != 0).all() and (grad[~far][:, others] != 0).any(1).all()
    P.op_status()


@pytest.mark.parametrize("dt", [FF, BF])
@pytest.mark.parametrize("rows,vocab", [(64, 12), (300, 4099)])
def test_topk_distill_gradient_alone_stays_a_softmax_where_log_sums_are_coarse(dt, rows, vocab):
    """At T = 2^-30 fp32 log sums are 2^10 apart, so exponents of the others' softmax are off by hundreds either way; none of its terms is above 1, nor is any q."""
    import paper_2410_03960_b200 as P
    z = torch.full((rows, vocab), -1.0, device="cuda")
    top = torch.arange(1, rows + 1, device="cuda") * 0.37
    z[:, 3], z[:, 7], z[:, 9] = top, top, top                # an entry and two others, equally likely
    z, temp = z.to(dt), 2.0 ** -30
    ids, lp, weight = i32([[3, 5]] * rows), torch.log(f32([[0.25, 0.125]] * rows)), f32(np.linspace(-1, 1, rows))
    got = P.topk_distill(z, ids, lp, temperature=temp, grad_loss=weight)
    alone = P.topk_distill_bwd(z, ids, lp, got["lse"], got["rest_lse"], weight, temperature=temp)
    for grad in (got["grad_logits"], alone):
        assert (grad.double().abs() <= (weight.double().abs() / temp)[:, None] * (1 + u_of(dt) + 1e-6)).all()
    P.op_status()


def special(dt, rows, vocab, kind, seed=31):
    """Rows whose teacher's outcomes do not sum to one, every second row; ordinary ones between them."""
    z, ids, lp, weight = T.teacher(seed, rows, vocab, 4, dt, 1.0, sharp=1.5)
    z, lp, odd = z.clone(), lp.clone(), torch.arange(rows, device="cuda") % 2 == 0
    if kind == "others masked":
        keep = torch.zeros((rows, vocab), dtype=torch.bool, device="cuda").scatter_(1, ids.long(), True)
        z[odd[:, None] & ~keep] = -float("inf")
        lp[odd] = torch.log(f32([0.4, 0.3, 0.06, 0.04]))
    elif kind == "above one":
        lp[odd] = torch.log(f32([0.5, 0.4, 0.1, 0.02]))
    elif kind == "nothing":
        lp[odd] = -float("inf")
    elif kind == "whole vocabulary":                       # (vocab = 4: there are no others)
        lp[odd] = torch.log(f32([0.4, 0.3, 0.06, 0.04]))
    return z, ids, lp, weight


@pytest.mark.parametrize("dt", [FF, BF, HF])
@pytest.mark.parametrize("rows,vocab,kind", [(r, v, k) for r, v in ((6, 40), (5, 4097), (3, 40000), (320, 2001)) for k in ("others masked", "above one", "nothing")] + [(6, 4, "whole vocabulary")])
@pytest.mark.parametrize("temp,rest", [(1.0, True), (1.0, False), (0.7, True), (3.0, True)])
def test_topk_distill_gradient_where_the_teacher_does_not_sum_to_one(dt, rows, vocab, kind, temp, rest):
    """The slope of the returned loss: P q - p with P = sum p + p_r.  An error d of lse changes P q_k by P q_k d; elsewhere (P q_r - p_r) s, with s the others'
    softmax, by P q_r s d and, through s, by |P q_r - p_r| 2 d; the gradient alone has rounded log sums and exponents beside."""
    import paper_2410_03960_b200 as P
    z, ids, lp, weight = special(dt, rows, vocab, kind)
    kept, g, ids_h = f64(z), f64(weight), ids.cpu().numpy()
    loss, lse, rest_lse, y, qr, pr = S.distill(kept, ids_h, f64(lp), temp, rest, g)
    mass = S.masses(kept, ids_h, f64(lp), temp, rest)
    got = P.topk_distill(z, ids, lp, temperature=temp, rest=rest, grad_loss=weight)
    alone = P.topk_distill_bwd(z, ids, lp, got["lse"], got["rest_lse"], weight, temperature=temp, rest=rest)
    given = np.zeros(kept.shape, bool)
    np.put_along_axis(given, ids_h.astype(np.int64), True, 1)
    with np.errstate(invalid="ignore"):
        s = np.nan_to_num(np.exp(np.minimum(kept / temp - np.where(np.isfinite(rest_lse), rest_lse, np.inf)[:, None], 0.0)))
    q = np.exp(kept / temp - lse[:, None])
    size = np.abs(np.where(np.isfinite(kept), kept, 0.0)) / temp + np.abs(np.where(np.isfinite(rest_lse), rest_lse, 0.0))[:, None] + np.abs(lse)[:, None]
    inv = (np.abs(g) / temp)[:, None]
    for x, more in ((got["grad_logits"], 0.0), (alone, 1.0)):
        off = np.where(given, mass[:, None] * q, s * (mass * qr + 2 * np.abs(mass * qr - pr))[:, None]) * inv * (D * (1 + more) + more * 4 * size * 2.0 ** -24)
        assert (np.abs(f64(x) - y) <= off + u_of(dt) * (np.abs(y) + off) + (2.0 ** -25 if dt == HF else 1e-37)).all(), np.abs(f64(x) - y).max()
    assert (np.abs(f64(got["loss"]) - loss) <= (np.abs(mass * qr - pr) + D) * D + 2.0 ** -24 * np.abs(loss) + 1e-12).all()
    P.op_status()


@pytest.mark.parametrize("kind", ["others masked", "above one", "nothing"])
@pytest.mark.parametrize("rest", [True, False])
def test_topk_distill_gradient_against_differences_where_the_teacher_does_not_sum_to_one(kind, rest):
    """Central differences of the 64-bit loss, as in test_gpu_drafts.py; and both calls."""
    import paper_2410_03960_b200 as P
    z, ids, lp, weight = special(FF, 4, 40, kind, 32)
    got = P.topk_distill(z, ids, lp, temperature=1.3, rest=rest, grad_loss=weight)
    alone = P.topk_distill_bwd(z, ids, lp, got["lse"], got["rest_lse"], weight, temperature=1.3, rest=rest)
    x, h = f64(z), 1e-4
    loss = lambda a: R.distill(a, ids.cpu().numpy(), f64(lp), 1.3, rest)[0]  # noqa: E731
    for v in range(40):
        up, down = x.copy(), x.copy()
        up[:, v] += h
        down[:, v] -= h
        with np.errstate(invalid="ignore"):
            want = (loss(up) - loss(down)) / (2 * h) * f64(weight)
        for grad in (got["grad_logits"], alone):
            assert (np.abs(f64(grad)[:, v] - want) <= (h * h + 1e-11 + 2 * D) * np.abs(f64(weight))).all(), v


@pytest.mark.parametrize("dt", [FF, BF])
@pytest.mark.parametrize("vocab,rows", [(6, 6), (700, 6), (40000, 6), (3000, 320)])
@pytest.mark.parametrize("rest", [True, False])
def test_topk_distill_entries_that_are_missing_or_double(monkeypatch, dt, vocab, rows, rest):
    """The rows of the test of that name in test_gpu_drafts.py, with the loss's own slope."""
    monkeypatch.setattr(R, "distill", S.distill)
    T.test_topk_distill_entries_that_are_missing_or_double(dt, vocab, rows, rest)


@pytest.mark.parametrize("dt", [FF, BF, HF])
@pytest.mark.parametrize("vocab", [12, 3001, 50000])
def test_topk_distill_masked_logits(monkeypatch, dt, vocab):
    """Likewise."""
    monkeypatch.setattr(R, "distill", S.distill)
    T.test_topk_distill_masked_logits(dt, vocab)


# ---------------------------------------------------------------------------------------------------- verify_drafts
@pytest.mark.parametrize("dt", [FF, BF])
@pytest.mark.parametrize("n_seqs,vocab", [(1500, 1024), (1500, 2048), (40, 8192), (4, 70000)])
@pytest.mark.parametrize("repeats,holes", [(2, False), (4, False), (4, True)])
@pytest.mark.parametrize("probs", [False, True])
def test_verify_drafts_draws_at_a_border_between_tiles(dt, n_seqs, vocab, repeats, holes, probs):
    """Rows that repeat themselves, and random numbers at the borders between the repetitions, where sums that are rounded in another order lie on either side: somebody
    writes a token, and it is one whose prefix sums enclose the target.  (Weights are good to 1e-14 and at most vocab sums to 2^-53 each: 1e-11 covers both.)"""
    import paper_2410_03960_b200 as P
    g = torch.Generator(device="cuda").manual_seed(vocab + repeats)
    part = torch.randn((n_seqs, vocab // repeats), generator=g, device="cuda") * 2
    if holes:                                              # most tokens are masked: whole lanes have no weight
        part[torch.rand(part.shape, generator=g, device="cuda") < 0.95] = -float("inf")
        part[:, 0] = 1.0
    row = part.to(dt).repeat(1, repeats)
    news = 2 if probs else 1
    z = row.repeat_interleave(news, 0)
    places = torch.arange(n_seqs, device="cuda") % (repeats - 1) + 1
    u = torch.full((n_seqs, news), 0.99999, device="cuda")
    u[:, 0] = places / repeats
    q = None
    left = torch.softmax(row.double(), 1)
    if probs:                                              # the drafted token falls: what it was given goes off the row, the same in every repetition
        q = torch.zeros((news * n_seqs, vocab), device="cuda")
        q[1::2, torch.arange(repeats, device="cuda") * (vocab // repeats)] = 1.0 / repeats
        left = (left - q[1::2].double()).clamp(min=0.0)
    out = {k: torch.full((n_seqs, news) if k != "n_accepted" else (n_seqs,), -77, dtype=torch.int32, device="cuda") for k in ("n_accepted", "tokens", "path")}
    tokens = torch.zeros(news * n_seqs, dtype=torch.int32, device="cuda")
    P.verify_drafts(z, tokens, i32(news * np.arange(n_seqs + 1)), news, u.flatten(), draft_probs=q, out=out)
    assert (out["n_accepted"] == 0).all()
    token = out["tokens"][:, 0].long()
    assert ((token >= 0) & (token < vocab)).all()
    sums = left.cumsum(1)
    total, target = sums[:, -1], u[:, 0].double() * sums[:, -1]
    until, weight = sums.gather(1, token[:, None])[:, 0], left.gather(1, token[:, None])[:, 0]
    assert (weight > 0).all() and (until >= target - 1e-11 * total).all() and (until - weight <= target + 1e-11 * total).all()
    P.op_status()


@pytest.mark.parametrize("dt", [FF, BF])
@pytest.mark.parametrize("news,vocab", [([2] * 8, 4), ([5] * 40, 1000), ([6, 1, 8, 3], 40001), ([4] * 300, 5003)])
def test_verify_drafts_ids_that_are_none_with_the_drafters_probabilities(dt, news, vocab):
    """A shorter draft padded with -1, ids at or beyond the vocabulary, at several depths: nothing was drawn from such a row of draft_probs, whatever it holds, and nothing
    of it goes off the target."""
    import paper_2410_03960_b200 as P
    z, tokens, cu, _, q, u = T.drafts(vocab, news, vocab, dt, probs=True)
    junk = [0.0, float("nan"), float("inf"), 1.0, -1.0]
    for b, n in enumerate(news):
        if n < 2:
            continue
        j = 1 + b % (n - 1)
        tokens[cu[b] + j:cu[b] + n] = -1
        q[cu[b] + j:cu[b] + n] = junk[b % 5]
    for temps in (None, np.random.default_rng(1).choice([1.0, 0.0, 0.5], len(news))):
        T.check_verify(z, tokens, cu, None, q, u, temps)
    P.op_status()
    tokens[tokens == -1] = vocab
    T.check_verify(z, tokens, cu, None, q, u)
    with pytest.raises(P.SwiftKVError):
        P.op_status()
    z = torch.zeros((2, 4), dtype=dt, device="cuda")
    q = f32([[0, 0, 0, 0], [1, 0, 0, 0]])
    assert P.verify_drafts(z, i32([0, -1]), i32([0, 2]), 2, f32([0, 0]), draft_probs=q)["tokens"].tolist() == [[0, -1]]


def test_verify_drafts_refuses_temperatures_that_32_bits_round_to_0():
    import paper_2410_03960_b200 as P
    z, args = torch.randn((2, 50), device="cuda"), (i32([0, 1]), i32([0, 2]), 2, f32([0.5, 0.5]))
    for t in (1e-50, -1e-50, 5e-324, 1e-46, 1e39, -1e39):
        with pytest.raises(P.SwiftKVError) as e:
            P.verify_drafts(z, *args, temperature=t)
        assert e.value.code == -1
    for t in (0.0, -0.0, 0, 2.0 ** -64, 2.0 ** 100, 1):
        P.verify_drafts(z, *args, temperature=t)
    P.op_status()


@pytest.mark.parametrize("n_seqs,vocab", [(6, 300), (6, 40000), (200, 3000)])
def test_verify_drafts_weights_below_the_range_of_32_bits(n_seqs, vocab):
    """Drafted tokens whose weight is below 2^-126 against products of a small random number and a small probability: 64 bits decide."""
    z = torch.full((2 * n_seqs, vocab), -500.0, device="cuda")
    z[:, 3] = 0.0
    at = torch.arange(n_seqs, device="cuda") % 3
    z[0::2, 7] = f32([-95.0, -103.0, -90.0])[at]
    q = torch.full((2 * n_seqs, vocab), 2.0 ** -120, device="cuda")
    u = torch.full((2 * n_seqs,), 2.0 ** -24, device="cuda")
    counts, _, _ = T.check_verify(z, np.full(2 * n_seqs, 7), 2 * np.arange(n_seqs + 1), None, q, u)
    assert counts.tolist() == [[1, 0, 1][b % 3] for b in range(n_seqs)]
