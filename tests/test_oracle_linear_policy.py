"""Pins of the oracles of linear attention, of the token log-probabilities and of the policy loss: the recurrence,
central differences and closed forms. CPU only."""
import numpy as np
import pytest

from oracle import linear_oracle, linear_steps, policy_loss_oracle, token_logprobs_oracle

LENS = ((3, 0, 2), (2, 1, 2), (2, 1, 3, 0, 2))  # prefixes, group sizes, responses


def _problem(seed=0, hq=2, hkv=1, d=3):
    rng = np.random.default_rng(seed)
    tp, ts = sum(LENS[0]), sum(LENS[2])
    t = {}
    for part, rows in (("pre", tp), ("suf", ts)):
        for n, h in (("q", hq), ("k", hkv), ("v", hkv), ("do", hq)):
            t[f"{n}_{part}"] = rng.standard_normal((rows, h, d))
    return t, -rng.uniform(0.05, 1.5, hkv)


@pytest.mark.parametrize("with_state", [False, True])
def test_linear_oracle_is_the_recurrence(with_state):
    t, ld = _problem(1, hq=4, hkv=2)
    rng = np.random.default_rng(2)
    s_in = rng.standard_normal((3, 2, 3, 3)) if with_state else None
    ref = linear_oracle(*LENS, t, 0.5, ld, state_in=s_in, grads=False)
    p0 = s0 = m = 0
    for g, (p, size) in enumerate(zip(LENS[0], LENS[1])):
        state = s_in[g].copy() if with_state else np.zeros((2, 3, 3))
        for i in range(p0, p0 + p):
            o, state = (x[0] for x in linear_steps(*(t[n + "_pre"][i][None] for n in "qkv"), state[None], ld, 0.5))
            np.testing.assert_allclose(ref["o_pre"][i], o, atol=1e-12)
        np.testing.assert_allclose(ref["state_pre"][g], state, atol=1e-12)
        for s in LENS[2][m:m + size]:
            mine = state.copy()
            for i in range(s0, s0 + s):
                o, mine = (x[0] for x in linear_steps(*(t[n + "_suf"][i][None] for n in "qkv"), mine[None], ld, 0.5))
                np.testing.assert_allclose(ref["o_suf"][i], o, atol=1e-12)
            np.testing.assert_allclose(ref["state_suf"][m], mine, atol=1e-12)
            s0 += s
            m += 1
        p0 += p


def test_linear_gradients_are_differences():
    t, ld = _problem(3)
    grad = linear_oracle(*LENS, t, 0.7, ld)

    def value():
        r = linear_oracle(*LENS, t, 0.7, ld, grads=False)
        return float((r["o_pre"] * t["do_pre"]).sum() + (r["o_suf"] * t["do_suf"]).sum())

    for n in "qkv":
        for part in ("pre", "suf"):
            x = t[f"{n}_{part}"]
            for i in np.ndindex(x.shape):
                old, e = x[i], 1e-5
                x[i] = old + e
                up = value()
                x[i] = old - e
                down = value()
                x[i] = old
                assert abs((up - down) / (2 * e) - grad[f"d{n}_{part}"][i]) < 1e-8, (n, part, i)


def test_no_memory_and_full_memory():
    """Decay 0: o = scale (q.k) v of the row itself; decay 1: the plain sum over all visible rows."""
    t, _ = _problem(4)
    none = linear_oracle(*LENS, t, 1.0, np.array([-np.inf]), grads=False)
    for part in ("pre", "suf"):
        w = (t["q_" + part] * t["k_" + part]).sum(-1, keepdims=True)
        np.testing.assert_allclose(none["o_" + part], w * t["v_" + part], atol=1e-12)
    full = linear_oracle(*LENS, t, 1.0, np.array([0.0]), grads=False)
    k, v = (np.concatenate([t[n + "_pre"][:3], t[n + "_suf"][:2]])[:, 0] for n in "kv")
    np.testing.assert_allclose(full["o_suf"][1, 0], (t["q_suf"][1, 0] @ k.T) @ v, atol=1e-12)


def _logits(seed, vocab=7):
    rng = np.random.default_rng(seed)
    tp, ts = len(LENS[0]), sum(LENS[2])
    return rng.standard_normal((tp, vocab)), rng.standard_normal((ts, vocab)), rng.integers(0, vocab, ts), rng.standard_normal(ts)


def test_logprobs_of_a_uniform_row_and_differences():
    last, suf, tok, d = _logits(5)
    logp, lse, ent = token_logprobs_oracle(*LENS, np.zeros_like(last), np.zeros_like(suf), tok)
    seen = lse > -np.inf  # all but the first token of the group without a prefix
    assert list(np.nonzero(~seen)[0]) == [3]
    np.testing.assert_allclose(logp[seen], -np.log(7))
    np.testing.assert_allclose(ent[seen], np.log(7))
    tok[2] = -1
    *_, gl, gs = token_logprobs_oracle(*LENS, last, suf, tok, 0.8, d)
    value = lambda: float((token_logprobs_oracle(*LENS, last, suf, tok, 0.8)[0] * d).sum())  # noqa: E731
    for x, gr in ((last, gl), (suf, gs)):
        for i in np.ndindex(x.shape):
            old, e = x[i], 1e-5
            x[i] = old + e
            up = value()
            x[i] = old - e
            down = value()
            x[i] = old
            assert abs((up - down) / (2 * e) - gr[i]) < 1e-8


@pytest.mark.parametrize("average", ["group", "token"])
@pytest.mark.parametrize("ref", [False, True])
def test_policy_gradient_is_differences(average, ref):
    rng = np.random.default_rng(6)
    ts = sum(LENS[2])
    lp, old = -rng.uniform(0.1, 3, ts), None
    old = lp + rng.choice([-0.4, -0.05, 0.06, 0.5], ts)
    lref = lp + rng.standard_normal(ts) if ref else None
    adv, mask = rng.standard_normal(len(LENS[2])), rng.random(ts) < 0.8
    args = dict(logp_old=old, logp_ref=lref, mask=mask, clip=(0.2, 0.28), beta=0.1 if ref else 0.0, average=average)
    stats, grad = policy_loss_oracle(LENS[1], LENS[2], lp, adv, **args)
    assert abs(stats[0] - stats[1] - args["beta"] * stats[2]) < 1e-12
    assert 0 <= stats[3] < 1
    for i in range(ts):
        e = 1e-6
        up, down = lp.copy(), lp.copy()
        up[i] += e
        down[i] -= e
        diff = (policy_loss_oracle(LENS[1], LENS[2], up, adv, **args)[0][0]
                - policy_loss_oracle(LENS[1], LENS[2], down, adv, **args)[0][0]) / (2 * e)
        assert abs(diff - grad[i]) < 1e-8
        if not mask[i]:
            assert grad[i] == 0


def test_on_policy_group_gradient_is_minus_the_advantage():
    _, grad = policy_loss_oracle((2,), (4, 2), np.zeros(6), np.array([1.0, -1.0]))
    np.testing.assert_allclose(grad, [-1 / 8] * 4 + [1 / 4] * 2)
