"""The operators as a GRPO step uses them: a small hybrid layer in the grouped layout, forward and backward, against the
same step in float64 on the repeated layout with torch autograd.

x -> q, k, v -> rotary embedding -> grouped attention, and beside it linear attention with a decay -> h = x + both
-> logits -> token log-probabilities -> clipped loss with KL, and back through every step by the library's backward
calls (the projections are plain torch products). The reference encodes every [prefix; response] by itself.

Bound: fp32 throughout; each of the six stages rounds a sum of at most 600 terms, 2^-24 each, so a result is within
6 * 600 * 2^-24 = 2.2e-4 of its norm.
"""
import numpy as np
import pytest

from oracle import grouped_positions

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

LENS = ((37, 0, 70), (3, 1, 2), (12, 1, 33, 5, 20, 0))
HQ, HKV, D, WIDTH, VOCAB, BETA, TEMP = 4, 2, 64, 96, 211, 0.05, 0.8


def _weights(gen):
    mk = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64) / s[0] ** 0.5  # noqa: E731
    return {"q": mk(WIDTH, HQ * D), "k": mk(WIDTH, HKV * D), "v": mk(WIDTH, HKV * D), "o": mk(HQ * D, WIDTH),
            "head": mk(WIDTH, VOCAB)}


def _rotate(x, pos):
    half = D // 2
    ang = pos[:, None].double() * 10000.0 ** (-2.0 * torch.arange(half).double() / D)
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _reference(x_pre, x_suf, w, ld, tokens, old, ref, adv):
    """float64, member by member on the repeated layout."""
    parts, logps = [], []
    p0 = s0 = m = 0
    for p, size in zip(LENS[0], LENS[1]):
        for s in LENS[2][m:m + size]:
            x = torch.cat([x_pre[p0:p0 + p], x_suf[s0:s0 + s]])
            n = p + s
            pos = torch.arange(n)
            q, k, v = (t.view(n, -1, D) for t in (x @ w["q"], x @ w["k"], x @ w["v"]))
            q, k = _rotate(q, pos), _rotate(k, pos)
            kk, vv = (t.repeat_interleave(HQ // HKV, 1) for t in (k, v))
            sc = torch.einsum("ihd,jhd->hij", q, kk) / D ** 0.5
            gap = (pos[:, None] - pos[None]).double()
            att = sc.masked_fill(gap < 0, float("-inf")).softmax(-1) if n else sc
            dec = torch.exp(ld.repeat_interleave(HQ // HKV)[:, None, None] * gap.clamp_min(0)) * (gap >= 0)
            y = torch.einsum("hij,jhd->ihd", att, vv) + torch.einsum("hij,jhd->ihd", sc * dec, vv)
            h = x + y.reshape(n, -1) @ w["o"]
            if s:
                lp = torch.log_softmax(h @ w["head"] / TEMP, -1)
                first = 0 if p else 1  # nothing predicts the first token where there is no prefix
                rows = torch.arange(p - 1 + first, n - 1)
                mine = lp[rows, tokens[s0 + first:s0 + s]]
                logps.append(torch.cat([mine.new_zeros(first), mine]))
            s0 += s
            m += 1
        p0 += p
    logp = torch.cat(logps)
    s0, loss = 0, 0.0
    member = torch.repeat_interleave(torch.arange(len(LENS[2])), torch.tensor(LENS[2]))
    weight = torch.cat([torch.full((s,), 1.0 / (3 * g * s), dtype=torch.float64) for s, g in zip(LENS[2], [3, 3, 3, 1, 2, 2]) if s])
    r, a = torch.exp(logp - old), adv[member]
    gone = ref - logp
    loss = (weight * (-torch.minimum(r * a, r.clamp(0.8, 1.2) * a) + BETA * (torch.exp(gone) - gone - 1))).sum()
    return loss, logp


def test_grpo_step_equals_the_repeated_layout():
    from paper_2506_05433_amd import binding as b
    print("[step] grouped layer forward and backward", flush=True)
    gen = torch.Generator().manual_seed(11)
    w = _weights(gen)
    tp, ts = sum(LENS[0]), sum(LENS[2])
    x = torch.randn(tp + ts, WIDTH, generator=gen, dtype=torch.float64)
    ld = -torch.tensor([0.02, 0.4], dtype=torch.float64)
    tokens = torch.randint(0, VOCAB, (ts,), generator=gen)
    adv = torch.randn(len(LENS[2]), generator=gen, dtype=torch.float64)
    leaves = {n: t.clone().requires_grad_() for n, t in w.items()}
    xr = x.clone().requires_grad_()
    with torch.no_grad():
        base = _reference(x[:tp], x[tp:], w, ld, tokens, torch.zeros(ts, dtype=torch.float64), torch.zeros(ts, dtype=torch.float64), adv)[1]
    old = (base + 0.2 * torch.randn(ts, generator=gen, dtype=torch.float64)).float().double()
    ref = (base + 0.2 * torch.randn(ts, generator=gen, dtype=torch.float64)).float().double()
    loss, logp = _reference(xr[:tp], xr[tp:], leaves, ld, tokens, old, ref, adv)
    loss.backward()

    # the grouped layout on the GPU, fp32
    f = lambda t: t.float().cuda()  # noqa: E731
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device="cuda")  # noqa: E731
    W, X, dld = {n: f(t) for n, t in w.items()}, f(x), f(ld)
    grp = (i32(np.concatenate([[0], np.cumsum(LENS[0])]).tolist()), i32(np.concatenate([[0], np.cumsum(LENS[2])]).tolist()), i32(LENS[1]))
    scale = D ** -0.5
    q, k, v = ((X @ W[n]).view(tp + ts, -1, D) for n in "qkv")
    rq_pre, rq_suf, rk_pre, rk_suf = b.rope(q[:tp], q[tp:], k[:tp], k[tp:], *grp)
    args = (rq_pre, rk_pre, v[:tp], rq_suf, rk_suf, v[tp:])
    a_pre, a_suf, lse_pre, lse_suf = b.fwd(*args, *grp, scale)
    l_pre, l_suf = b.linear_fwd(*args, dld, *grp, scale)
    y = torch.cat([a_pre + l_pre, a_suf + l_suf]).view(tp + ts, -1)
    h = X + y @ W["o"]
    last = torch.tensor([36, 0, 106], device="cuda")  # each group's last prefix row (the second has none)
    logits_last, logits_suf = h[last] @ W["head"], h[tp:] @ W["head"]
    tok = tokens.cuda()
    got_logp, lse = b.token_logprobs(logits_last, logits_suf, tok, *grp, tp, temperature=TEMP)
    stats, dlogp = b.policy_loss(got_logp, f(adv), *grp[1:], logp_old=f(old), logp_ref=f(ref), beta=BETA)
    d_last, d_suf = b.token_logprobs_bwd(logits_last, logits_suf, tok, lse, dlogp, *grp, tp, temperature=TEMP)
    grad = {"head": h[last].t() @ d_last + h[tp:].t() @ d_suf}
    dh = torch.zeros_like(h)
    dh[tp:] = d_suf @ W["head"].t()
    dh[last[[0, 2]]] += (d_last @ W["head"].t())[[0, 2]]
    assert bool((d_last[1] == 0).all())
    grad["o"] = y.t() @ dh
    dy = (dh @ W["o"].t()).view(tp + ts, HQ, D)
    dy_pre, dy_suf = dy[:tp].contiguous(), dy[tp:].contiguous()
    g1 = b.bwd(*args, a_pre, a_suf, lse_pre, lse_suf, dy_pre, dy_suf, *grp, scale)
    g2 = b.linear_bwd(*args, dy_pre, dy_suf, dld, *grp, scale)
    dq_pre, dk_pre, dv_pre, dq_suf, dk_suf, dv_suf = (p + r for p, r in zip(g1, g2))
    dq_pre, dq_suf, dk_pre, dk_suf = b.rope(dq_pre, dq_suf, dk_pre, dk_suf, *grp, inverse=True)
    dX = dh.clone()
    for n, parts in (("q", (dq_pre, dq_suf)), ("k", (dk_pre, dk_suf)), ("v", (dv_pre, dv_suf))):
        d = torch.cat(parts).view(tp + ts, -1)
        grad[n] = X.t() @ d
        dX += d @ W[n].t()

    def near(name, a, r):
        err = float((a.double().cpu() - r).norm() / r.norm())
        print(f"  {name}: {err:.2e}", flush=True)
        assert err <= 6 * 600 * 2.0 ** -24, (name, err)

    near("logp", got_logp, logp.detach())
    near("loss", stats[0], loss.detach())
    for n, t in leaves.items():
        near("d" + n, grad[n], t.grad)
    near("dx", dX, xr.grad)
