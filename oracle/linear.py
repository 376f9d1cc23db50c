"""Plain numpy oracle of linear attention with a decay for each kv head, in the repeated-prefix layout.

TEST INFRASTRUCTURE ONLY: imported by the tests, never by the product path.

The definition, for one sequence x = [P; R_i] of the Repeated-Prefix Forward and query head h of kv head g:
    o_t = scale * sum_{s <= t} exp(log_decay[g])^(t - s) (q_t . k_s) v_s  [+ exp(log_decay[g])^(t + 1) scale S_in^T q_t],
formed with the full masked matrix of every sequence, without states or chunks; gradients are those of that
sum, the prefix's summed over its copies, its upstream gradient counted once. Beside every value stands
its magnitude: the same sums with absolute values, which bound what roundings of their terms can move.
"""
import numpy as np


def decay_matrix(n, log_decay):
    """[n, n]: decay^(t - s) for s <= t, else 0 (decay 0 keeps the diagonal)."""
    gap = np.arange(n)[:, None] - np.arange(n)[None]
    with np.errstate(invalid="ignore", over="ignore"):
        m = np.where(gap == 0, 1.0, np.exp(np.where(gap > 0, log_decay * np.maximum(gap, 1), -np.inf)))
    return m


def linear_sequences(q, k, v, d_o, log_decay, scale, state_in):
    """One sequence: q, d_o [n, h_q, d], k, v [n, h_kv, d]. Returns dict of o, dq, dk, dv, state."""
    n, hq, d = q.shape
    hkv = k.shape[1]
    rep = hq // hkv
    out = {"o": np.zeros((n, hq, d)), "dq": np.zeros((n, hq, d)), "dk": np.zeros((n, hkv, d)),
           "dv": np.zeros((n, hkv, d)), "state": np.zeros((hkv, d, d))}
    for g in range(hkv):
        m = decay_matrix(n, log_decay[g])
        last = m[-1] if n else np.zeros(0)
        out["state"][g] = (k[:, g] * last[:, None]).T @ v[:, g]
        lam = np.exp(log_decay[g])
        if state_in is not None:
            out["state"][g] += lam ** n * state_in[g]
        for h in range(g * rep, (g + 1) * rep):
            w = (q[:, h] @ k[:, g].T) * m * scale
            out["o"][:, h] = w @ v[:, g]
            if state_in is not None:
                out["o"][:, h] += scale * (lam ** np.arange(1, n + 1))[:, None] * (q[:, h] @ state_in[g])
            if d_o is not None:
                dw = (d_o[:, h] @ v[:, g].T) * m * scale
                out["dq"][:, h] = dw @ k[:, g]
                out["dk"][:, g] += dw.T @ q[:, h]
                out["dv"][:, g] += w.T @ d_o[:, h]
    return out


def linear_oracle(prefix_lens, group_sizes, suffix_lens, t, scale, log_decay, state_in=None, grads=True,
                  magnitude=False):
    """Grouped results of the repeated computation. ``t``: arrays q_pre ... v_suf and, for gradients, do_pre, do_suf.
    Returns o_pre, o_suf, state_pre [groups, ...], state_suf [members, ...] and the six gradients. ``magnitude``:
    every input by its absolute value."""
    a = {n: (np.abs(x) if magnitude else np.asarray(x)).astype(np.float64) for n, x in t.items()}
    if state_in is not None:
        state_in = (np.abs(state_in) if magnitude else np.asarray(state_in)).astype(np.float64)
    res = {"o_pre": np.zeros(a["q_pre"].shape), "o_suf": np.zeros(a["q_suf"].shape)}
    hkv, d = a["k_pre"].shape[1:]
    res["state_pre"] = np.zeros((len(prefix_lens), hkv, d, d))
    res["state_suf"] = np.zeros((len(suffix_lens), hkv, d, d))
    if grads:
        for n, like in (("dq", "q"), ("dk", "k"), ("dv", "v")):
            res[n + "_pre"], res[n + "_suf"] = np.zeros(a[like + "_pre"].shape), np.zeros(a[like + "_suf"].shape)
    p0 = s0 = m = 0
    for g, (p, size) in enumerate(zip(prefix_lens, group_sizes)):
        p, pre = int(p), slice(p0, p0 + int(p))
        init = None if state_in is None else state_in[g]

        def run(suf, do_pre):
            cat = lambda n: np.concatenate([a[n + "_pre"][pre], a[n + "_suf"][suf]])  # noqa: E731
            d_o = np.concatenate([do_pre, a["do_suf"][suf]]) if grads else None
            return linear_sequences(cat("q"), cat("k"), cat("v"), d_o, log_decay, scale, init)

        none = slice(s0, s0)
        alone = run(none, a["do_pre"][pre] if grads else None)  # the prefix by itself, with its own upstream gradient
        res["o_pre"][pre], res["state_pre"][g] = alone["o"], alone["state"]
        if grads:
            for n in ("dq", "dk", "dv"):
                res[n + "_pre"][pre] = alone[n]
        for s in suffix_lens[m:m + int(size)]:
            suf = slice(s0, s0 + int(s))
            one = run(suf, np.zeros_like(a["q_pre"][pre]))
            res["o_suf"][suf], res["state_suf"][m] = one["o"][p:], one["state"]
            if grads:
                for n in ("dq", "dk", "dv"):
                    res[n + "_pre"][pre] += one[n][:p]
                    res[n + "_suf"][suf] = one[n][p:]
            s0 += int(s)
            m += 1
        p0 += p
    return res


def linear_steps(q, k, v, state, log_decay, scale):
    """One token of every sequence: (o, state'), float64."""
    q, k, v, state = (np.asarray(x, np.float64) for x in (q, k, v, state))
    rep = q.shape[1] // k.shape[1]
    with np.errstate(under="ignore"):
        new = np.exp(np.asarray(log_decay, np.float64))[None, :, None, None] * state + k[..., :, None] * v[..., None, :]
    o = np.stack([scale * np.einsum("ni,nij->nj", q[:, h], new[:, h // rep]) for h in range(q.shape[1])], 1)
    return o, new
