"""Plain numpy oracle of the responses' token log-probabilities and of the clipped policy loss.

TEST INFRASTRUCTURE ONLY: imported by the tests, never by the product path.

Log-probabilities are taken member by member in the repeated layout: the rows that predict a member's tokens are the
prefix's last row (a copy for every member) and its own rows but the last. Gradients of the copies are summed.
The loss is the definition, token by token, with the average written as nested means.
"""
import math

import numpy as np


def token_logprobs_oracle(prefix_lens, group_sizes, suffix_lens, logits_last, logits_suf, tokens, temperature=1.0,
                          dlogp=None):
    """(logp, lse, entropy) per response row, and with ``dlogp`` also (dlogits_last, dlogits_suf); float64."""
    vocab = logits_suf.shape[1]
    n = int(sum(suffix_lens))
    logp, lse, ent = np.zeros(n), np.full(n, -np.inf), np.zeros(n)
    d_last, d_suf = np.zeros(logits_last.shape), np.zeros(logits_suf.shape)
    at = m = 0
    for g, (p, size) in enumerate(zip(prefix_lens, group_sizes)):
        for s in suffix_lens[m:m + int(size)]:
            for j in range(int(s)):
                r = at + j
                if j == 0 and p == 0:
                    continue  # nothing predicts the first token
                x = np.asarray(logits_last[g] if j == 0 else logits_suf[r - 1], np.float64) / temperature
                top = x.max()
                tok = int(tokens[r])
                inside = 0 <= tok < vocab
                if top == -np.inf:
                    logp[r] = -np.inf if inside else 0.0
                    continue
                e = np.exp(x - top)
                tot = e.sum()
                lse[r] = top + math.log(tot)
                prob = e / tot
                live = prob > 0
                ent[r] = -np.sum(prob[live] * (x[live] - lse[r]))
                if not inside:
                    continue
                logp[r] = (x[tok] - top) - math.log(tot)
                if dlogp is not None and dlogp[r] != 0:
                    grad = -prob
                    grad[tok] += 1.0
                    (d_last[g] if j == 0 else d_suf[r - 1])[:] += float(dlogp[r]) / temperature * grad
            at += int(s)
            m += 1
    return (logp, lse, ent) if dlogp is None else (logp, lse, ent, d_last, d_suf)


def policy_loss_oracle(group_sizes, suffix_lens, logp, advantages, logp_old=None, logp_ref=None, mask=None,
                       clip=(0.2, 0.2), beta=0.0, average="group"):
    """(stats [loss, policy term, KL term, share clipped], dloss/dlogp), float64."""
    n = int(sum(suffix_lens))
    mask = np.ones(n, bool) if mask is None else np.asarray(mask) != 0
    groups, total = sum(1 for g in group_sizes if g > 0), int(mask.sum())
    stats, grad = np.zeros(4), np.zeros(n)
    at = m = 0
    for size in group_sizes:
        for s in suffix_lens[m:m + int(size)]:
            rows = [r for r in range(at, at + int(s)) if mask[r]]
            for r in rows:
                w = 1.0 / total if average == "token" else 1.0 / groups / int(size) / len(rows)
                lp, adv = float(logp[r]), float(advantages[m])
                ratio = math.exp(lp - (lp if logp_old is None else float(logp_old[r])))
                bound = min(max(ratio, 1 - clip[0]), 1 + clip[1])
                cut = bound * adv < ratio * adv
                pol = -(bound if cut else ratio) * adv
                d = 0.0 if cut else -ratio * adv
                kl = 0.0
                if logp_ref is not None:
                    x = float(logp_ref[r]) - lp
                    kl = math.expm1(x) - x
                    d -= beta * math.expm1(x)
                stats += w * np.array([pol + beta * kl, pol, kl, float(cut)])
                grad[r] = w * d
            at += int(s)
            m += 1
    return stats, grad
