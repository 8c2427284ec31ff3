"""verify_drafts, commit_drafts, topk_distill and its gradient on the GPU in calls that the documentation allows and ordinary inputs do not make: against
64-bit restatements (draft_reference.py).  Bounds are those of test_gpu_drafts.py, where they are derived."""
import numpy as np
import pytest
import torch

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
