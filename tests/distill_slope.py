"""The slope of topk_distill's loss where the teacher's outcomes do not sum to one, for the tests.

The loss is  sum p_k (log p_k - z_k + lse) + p_r (log p_r - rest_lse + lse)  of logits z = logits / T.  With the mass P = sum p_k + p_r its
derivative is  P q_k - p_k  at an entry and  (P q_r - p_r) exp(z - rest_lse)  elsewhere, divided by T.  P is 1 in ordinary rows; it is not where p_r is
cut off at 0 (sum p_k > 1), where p_r counts as 0 because there are no others, and where nothing has any probability (P = 0).
draft_reference.distill takes P = 1 always."""
import math

import numpy as np

import draft_reference as R

without_mass = R.distill


def outcomes(z, ids, logprobs, temp, rest):
    """Per row (P, tokens of the entries, their probabilities)."""
    found = []
    pr = without_mass(z, ids, logprobs, temp, rest)[5]
    for r in range(z.shape[0]):
        seen, p = [], []
        for k, i in enumerate(ids[r]):
            if 0 <= i < z.shape[1] and i not in seen:
                seen.append(int(i))
                p.append(math.exp(logprobs[r][k]))
        p = np.array(p)
        if not rest and p.sum() > 0:
            p = p / p.sum()
        found.append((float(rest and p.sum() + pr[r] or not rest and p.sum() > 0), seen, p))
    return found


def masses(*case):
    return np.array([m for m, _, _ in outcomes(*case)])


def distill(z, ids, logprobs, temp, rest, g=None):
    """draft_reference.distill with the loss's own slope in the gradient's place."""
    loss, lse, rest_lse, grad, qr, pr = without_mass(z, ids, logprobs, temp, rest, g)
    if g is not None:
        for r, (mass, seen, p) in enumerate(outcomes(z, ids, logprobs, temp, rest)):
            if not seen or mass == 1.0:
                continue
            y = z[r] / temp
            others = np.ones(z.shape[1], bool)
            others[seen] = False
            grad[r] = 0.0
            if rest_lse[r] >= lse[r] - 1000 * math.log(2):
                grad[r, others] = (mass * qr[r] - pr[r]) * np.exp(y[others] - rest_lse[r])
            grad[r, seen] = mass * np.exp(y[seen] - lse[r]) - p
            grad[r] *= g[r] / temp
    return loss, lse, rest_lse, grad, qr, pr
