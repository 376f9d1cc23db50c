"""Token log-probabilities, their gradient and the policy loss on the GPU against their float64 oracles.

Bounds (derived). Log-probabilities are fp32: with z = x / T the two roundings of a log-probability and of m / T are at
most 2^-23 max |z|; the sum of V exponentials has, for each, the rounding of its argument (|z| 2^-23 at most) and of
the sums (V / 256 + 40 additions in a row, 2^-24 each), so lse and logp are within 2^-22 (max |z| + V / 256 + 40). The
entropy's sum adds that error times 1 + max |z|. A gradient w p, w the sum of dlogp / T over the row's targets, has the
error of p's argument (2 max |z| + lse's), four roundings and one for each target summed; a target's place adds one
rounding of w and p's error there; the result is rounded to its type (u |ref|).
The policy loss is computed in fp64 and rounded to fp32 once: 2^-24 relative, with 1e-12 of the sum of magnitudes.
"""
import numpy as np
import pytest

from oracle import policy_loss_oracle, token_logprobs_oracle
from tests._parity import to_host

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def _cu(x):
    return torch.tensor(np.concatenate([[0], np.cumsum(x)]), dtype=torch.int32, device="cuda")


def _grp(lens):
    return _cu(lens[0]), _cu(lens[2]), torch.tensor(list(lens[1]), dtype=torch.int32, device="cuda")


LENS = [  # prefixes, group sizes, responses
    ((1,), (1,), (1,)),
    ((3, 0, 2), (2, 2, 3), (2, 1, 3, 1, 5, 0, 2)),
    ((4, 9), (70, 0), tuple([1] * 69 + [3])),          # one row, seventy targets
    ((2,), (5,), (17, 40, 1, 0, 9)),
    ((0,), (3,), (4, 0, 1)),
]
# vocabularies around the 16-byte pieces, a workgroup's sweep and beyond it; row strides and offsets of odd elements
SHAPES = [(1, 0, 0), (2, 3, 1), (7, 0, 0), (8, 0, 0), (255, 2, 1), (1000, 24, 8), (2049, 0, 3), (8200, 5, 2), (50001, 0, 0)]


def _logits(rows, vocab, pad, off, dt, gen, std=2.0):
    """[rows, vocab] whose rows lie vocab + pad elements apart, the first `off` elements into the allocation."""
    flat = torch.randn(off + rows * (vocab + pad) + 16, generator=gen, device="cuda").mul_(std).to(dt)
    return torch.as_strided(flat, (rows, vocab), (vocab + pad, 1), off), flat


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_logprobs_and_gradient(shape, dt):
    from paper_2506_05433_amd import binding
    vocab, pad, off = SHAPES[shape]
    lens = LENS[shape % len(LENS)]
    tp, ts, ng = sum(lens[0]), sum(lens[2]), len(lens[0])
    print(f"[logprobs] {lens} vocab {vocab} pad {pad} offset {off} {dt}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(shape)
    last, _ = _logits(ng, vocab, pad, off, dt, gen)
    suf, _ = _logits(ts, vocab, pad, off, dt, gen)
    tok = torch.randint(0, vocab, (ts,), generator=gen, device="cuda", dtype=torch.int64 if shape % 2 else torch.int32)
    if ts > 4:
        tok[2] = -100       # padding
        tok[4] = vocab      # outside
    if shape == 2:
        tok[:40] = 1        # many members with the same first token
    dlogp = torch.randn(ts, generator=gen, device="cuda")
    if ts > 5:
        dlogp[5] = 0.0
    temp = 0.7 if shape % 3 else 1.0
    host = (to_host(last), to_host(suf), tok.cpu().numpy())
    lp, lse, ent, gl, gs = token_logprobs_oracle(*lens, *host, temp, dlogp.double().cpu().numpy())
    got = binding.token_logprobs(last, suf, tok, *_grp(lens), tp, temperature=temp, entropy=True)
    zmax = max(np.abs(x).max() if x.size else 0.0 for x in host[:2]) / temp
    tol = 2.0 ** -22 * (zmax + vocab / 256 + 40)
    for name, a, b, t in (("logp", got[0], lp, tol), ("lse", got[1], lse, tol), ("entropy", got[2], ent, tol * (1 + 2 * zmax))):
        a = a.double().cpu().numpy()
        assert np.array_equal(np.isfinite(a), np.isfinite(b)), name
        f = np.isfinite(b)
        assert np.abs(a[f] - b[f]).max(initial=0.0) <= t, (name, np.abs(a[f] - b[f]).max(), t)
    again = binding.token_logprobs(last, suf, tok, *_grp(lens), tp, temperature=temp)
    assert len(again) == 2 and torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])

    # the gradient: into tensors of another stride and alignment, whose padding stays; then in place
    d_last, fl = _logits(ng, vocab, 3, 1, dt, gen)
    d_suf, fs = _logits(ts, vocab, 3, 1, dt, gen)
    before = [f.clone() for f in (fl, fs)]
    binding.token_logprobs_bwd(last, suf, tok, got[1], dlogp, *_grp(lens), tp, temperature=temp, out=(d_last, d_suf))
    for name, a, b, rows in (("dlogits_last", d_last, gl, ng), ("dlogits_suf", d_suf, gs, ts)):
        x = to_host(a).astype(np.float64)
        # w: the sum of |dlogp| / T over the row's targets, hit: where they lie
        w, hit = np.zeros((rows, 1)), np.zeros(b.shape)
        r = m = 0
        for g, size in enumerate(lens[1]):
            for s in lens[2][m:m + size]:
                for j in range(s):
                    at = (g if name == "dlogits_last" else None) if j == 0 else (r + j - 1 if name == "dlogits_suf" else None)
                    if at is not None and 0 <= int(tok[r + j]) < vocab:
                        w[at] += abs(float(dlogp[r + j])) / temp
                        hit[at, int(tok[r + j])] = 1.0
                r += s
            m += size
        z = (host[0] if name == "dlogits_last" else host[1]).astype(np.float64) / temp
        p = np.exp(z - z.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        rel = 2.0 ** -23 * (2 * zmax + 8) + tol + len(lens[2]) * 2.0 ** -24
        lim = U[dt] * np.abs(b) * 1.01 + rel * w * p + (rel + 2.0 ** -22) * w * hit + 1e-37
        assert np.isfinite(x).all() and (np.abs(x - b) <= lim).all(), (name, (np.abs(x - b) / lim).max())
    for f, o, rows in ((fl, before[0], ng), (fs, before[1], ts)):
        inside = torch.zeros(f.numel(), dtype=torch.bool, device="cuda")
        torch.as_strided(inside, (rows, vocab), (vocab + 3, 1), 1).fill_(True)
        assert torch.equal(f[~inside], o[~inside])
    c_last, c_suf = last.clone(), suf.clone()
    g2 = binding.token_logprobs_bwd(c_last, c_suf, tok, got[1], dlogp, *_grp(lens), tp, temperature=temp, out=(c_last, c_suf))
    assert torch.equal(g2[0], d_last) and torch.equal(g2[1], d_suf)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [13, 3000])
def test_masked_and_special_rows(dt, vocab):
    """Rows masked with -inf (some tokens, all), with the type's lowest value, NaN and +inf rows: the others keep theirs."""
    from paper_2506_05433_amd import binding
    lens = ((2, 2), (1, 1), (8, 1))
    print(f"[logprobs] special rows, vocab {vocab} {dt}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(3)
    low = torch.finfo(dt).min
    last, suf = (torch.randn(n, vocab, generator=gen, device="cuda").to(dt) for n in (2, 9))
    suf[0, 1:] = -float("inf")          # one token left
    suf[1] = -float("inf")              # none left
    suf[2, :-2] = low                   # masked with the lowest value
    suf[3] = low                        # all masked so: uniform
    suf[4, 2] = float("nan")
    suf[5, 3] = float("inf")
    tok = torch.zeros(9, dtype=torch.int64, device="cuda")
    tok[3] = vocab - 1
    tok[2] = 5                          # predicted by the row with nothing left
    lp, lse, ent = (t.cpu().numpy() for t in binding.token_logprobs(last, suf, tok, *_grp(lens), 4, entropy=True))
    # one token left, x = m: its term is 2^d with d = c x - fl(c m), |d| <= 2^-24 c |m|, c = log2 e; so s = 2^d, and
    # ln s, the entropy ln s - ln 2 d and lse - m are each at most 2 ln 2 |d| <= 2^-23 |m|, and one rounding of lse more
    x0 = float(suf[0, 0])
    assert max(abs(lp[1]), abs(ent[1]), abs(float(lse[1]) - x0)) <= 2.0 ** -22 * abs(x0)
    assert lp[2] == -np.inf and lse[2] == -np.inf and ent[2] == 0.0
    two = suf[2, -2:].double().cpu().numpy()
    want = two[1] - np.log(np.exp(two).sum())
    assert abs(lp[3] - want) < 2.0 ** -20
    assert abs(lp[4] + np.log(vocab)) < 2.0 ** -19 and abs(ent[4] - np.log(vocab)) < 2.0 ** -18
    assert np.isnan(lp[5]) and np.isnan(lp[6])
    assert np.isfinite(lp[[0, 7, 8]]).all()
    d = torch.ones(9, device="cuda")
    _, gs = binding.token_logprobs_bwd(last, suf, tok, torch.from_numpy(lse).cuda(), d, *_grp(lens), 4)
    g = gs.double().cpu().numpy()
    assert (g[1] == 0).all()                                    # nothing left: no gradient
    assert (g[0, 1:] == 0).all() and abs(g[0, 0]) <= 2.0 ** -20   # a certain token: onehot - softmax = 0 up to rounding
    assert (g[2, :-2] == 0).all() and abs(g[2].sum()) < 2.0 ** -7
    u = U[dt] + 2.0 ** -18
    assert (np.abs(g[3, 1:] + 1 / vocab) <= u / vocab).all() and abs(g[3, 0] - (1 - 1 / vocab)) <= u
    assert np.isnan(g[4]).all() and np.isnan(g[5]).all()
    assert np.isfinite(g[[6, 7, 8]]).all() and (g[[7, 8]] == 0).all()   # the members' last rows


def test_zero_dlogp_rows_are_not_read():
    """A token without a gradient (masked out of the loss) gives zeros, also where its logits are not numbers."""
    from paper_2506_05433_amd import binding
    lens = ((2,), (2,), (3, 2))
    gen = torch.Generator(device="cuda").manual_seed(4)
    last, suf = (torch.randn(n, 100, generator=gen, device="cuda") for n in (1, 5))
    suf[0] = float("nan")
    tok = torch.tensor([1, 2, 3, 4, 5], device="cuda")
    lp, lse = binding.token_logprobs(last, suf, tok, *_grp(lens), 2)
    d = torch.tensor([0.0, 0.0, 1.0, 0.0, 1.0], device="cuda")
    gl, gs = binding.token_logprobs_bwd(last, suf, tok, lse, d, *_grp(lens), 2)
    assert bool((gl == 0).all()) and bool((gs[[0, 2, 4]] == 0).all())
    assert bool(torch.isfinite(gs).all()) and bool((gs[[1, 3]] != 0).any(1).all())


@pytest.mark.parametrize("average", ["group", "token"])
@pytest.mark.parametrize("lens,old,ref,mask", [
    (((1,), (1,), (1,)), True, True, False),
    (((3, 0, 2), (2, 2, 3), (2, 1, 3, 1, 5, 0, 2)), True, True, True),
    (((3, 0, 2), (2, 0, 3), (200, 1, 3, 500, 70)), False, False, False),
    (((1, 1), (90, 3), tuple(range(93))), True, False, True),
    (((5,), (4,), (9000, 1, 0, 15000)), True, True, True),
])
def test_policy_loss(lens, old, ref, mask, average):
    from paper_2506_05433_amd import binding
    ts, ns = sum(lens[2]), len(lens[2])
    print(f"[policy] {len(lens[0])} groups, {ns} members, {ts} tokens, {average}", flush=True)
    rng = np.random.default_rng(ts)
    f = lambda x: x.astype(np.float32)  # noqa: E731
    lp = f(-rng.uniform(0.0, 6.0, ts))
    lold = f(lp + 0.3 * rng.standard_normal(ts)) if old else None
    if old and ts > 3:  # ratios exactly at, one step inside and outside of the border
        edge = np.float32(np.log1p(0.28))
        lp[:4], lold[:4] = [edge, np.nextafter(edge, np.float32(9)), np.nextafter(edge, np.float32(-9)), 0.0], 0.0
    lref = f(lp + 0.5 * rng.standard_normal(ts)) if ref else None
    m = rng.random(ts) < 0.7 if mask else None
    if mask and ts > 9:
        m[:2] = False                       # a member without kept tokens, in the second case
        lp[1] = np.nan                      # what is dropped does not count
        lold[1] = np.inf
    adv = f(rng.standard_normal(ns))
    args = dict(clip=(0.2, 0.28), beta=0.07 if ref else 0.0, average=average)
    clean = lp.copy()
    clean[np.isnan(clean)] = 0.0
    cold = None if lold is None else np.where(np.isinf(lold), 0.0, lold)
    cref = None if lref is None else np.nan_to_num(lref)
    want, grad = policy_loss_oracle(lens[1], lens[2], clean, adv, cold, cref, m, **args)
    t = lambda x: None if x is None else torch.from_numpy(x).cuda()  # noqa: E731
    _, cs, gs = _grp(lens)
    stats, d = binding.policy_loss(t(lp), t(adv), cs, gs, logp_old=t(lold), logp_ref=t(lref), mask=t(m), grad_scale=0.5, **args)
    stats, d = stats.double().cpu().numpy(), d.double().cpu().numpy()
    mags = np.abs(want).sum() + 1.0
    assert (np.abs(stats - want) <= 2.0 ** -24 * np.abs(want) + 1e-12 * mags).all(), (stats, want)
    assert (np.abs(d - 0.5 * grad) <= 2.0 ** -24 * np.abs(0.5 * grad) + 1e-14).all()
    if m is not None:
        assert (d[~m] == 0).all()
    again = binding.policy_loss(t(lp), t(adv), cs, gs, logp_old=t(lold), logp_ref=t(lref), mask=t(m), grad_scale=0.5, **args)
    assert np.array_equal(again[0].double().cpu().numpy(), stats) and np.array_equal(again[1].double().cpu().numpy(), d)


def test_policy_loss_without_tokens_and_all_masked():
    from paper_2506_05433_amd import binding
    none = torch.empty(0, device="cuda")
    stats, d = binding.policy_loss(none, torch.ones(2, device="cuda"), _cu([0, 0]), torch.tensor([2], dtype=torch.int32, device="cuda"))
    assert bool((stats == 0).all()) and d.numel() == 0
    lp = torch.full((5,), float("nan"), device="cuda")
    for average in ("group", "token"):
        stats, d = binding.policy_loss(lp, torch.ones(2, device="cuda"), _cu([3, 2]), torch.tensor([2], dtype=torch.int32, device="cuda"),
                                       mask=torch.zeros(5, dtype=torch.uint8, device="cuda"), average=average)
        assert bool((stats == 0).all()) and bool((d == 0).all())


def test_extreme_ratios():
    """Ratios beyond the range of fp32: clipped where the clip holds them, infinite where it does not; an advantage of 0
    gives 0 whatever the ratio."""
    from paper_2506_05433_amd import binding
    lp = torch.tensor([0.0, 0.0, -1000.0, -1000.0, 0.0], device="cuda")
    old = torch.tensor([-1000.0, -1000.0, 0.0, 0.0, -1000.0], device="cuda")
    adv = torch.tensor([1.0, -1.0, 1.0, -1.0, 0.0], device="cuda")
    stats, d = binding.policy_loss(lp, adv, _cu([1] * 5), torch.tensor([5], dtype=torch.int32, device="cuda"), logp_old=old, average="token")
    d = d.cpu().numpy()
    assert d[0] == 0 and d[1] == np.inf and d[2] == 0 and d[3] == 0 and d[4] == 0
    assert stats[0].item() == np.inf


def test_inconsistent_grouping_does_no_work():
    from paper_2506_05433_amd import binding
    bad, gs = torch.tensor([0, 7, 5], dtype=torch.int32, device="cuda"), torch.tensor([2], dtype=torch.int32, device="cuda")
    more = torch.tensor([3], dtype=torch.int32, device="cuda")
    x = torch.zeros(5, 16, device="cuda")
    tok, f = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(5, device="cuda")
    for cs, sizes in ((bad, gs), (_cu([3, 2]), more)):
        out = (torch.full((5,), 3.0, device="cuda"), torch.full((5,), 3.0, device="cuda"))
        ws = torch.empty(binding.token_logprobs_workspace_bytes(1, 2, 5, 16), dtype=torch.uint8, device="cuda")
        binding.token_logprobs(x[:1], x, tok, _cu([4]), cs, sizes, 4, out=out, workspace=ws)
        with pytest.raises(binding.PgError):
            binding.plan_status(ws)
        assert all(bool((t == 3.0).all()) for t in out)
        out = (torch.full((1, 16), 3.0, device="cuda"), torch.full((5, 16), 3.0, device="cuda"))
        binding.token_logprobs_bwd(x[:1], x, tok, f, f, _cu([4]), cs, sizes, 4, out=out, workspace=ws)
        with pytest.raises(binding.PgError):
            binding.plan_status(ws)
        assert all(bool((t == 3.0).all()) for t in out)
        out = (torch.full((4,), 3.0, device="cuda"), torch.full((5,), 3.0, device="cuda"))
        ws = torch.empty(binding.policy_loss_workspace_bytes(1, 2, 5), dtype=torch.uint8, device="cuda")
        binding.policy_loss(f, f[:2], cs, sizes, out=out, workspace=ws)
        with pytest.raises(binding.PgError):
            binding.plan_status(ws)
        assert all(bool((t == 3.0).all()) for t in out)


def test_captured_with_eager_work_between():
    """Log-probabilities, loss and gradient captured together; three replays equal the eager calls bit for bit."""
    from paper_2506_05433_amd import binding
    lens = ((3, 0, 2), (2, 2, 3), (200, 1, 33, 1, 5, 0, 77))
    ts, vocab = sum(lens[2]), 1003
    print("[policy] capture", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(9)
    last, suf = (torch.randn(n, vocab, generator=gen, device="cuda").bfloat16() for n in (3, ts))
    tok = torch.randint(0, vocab, (ts,), generator=gen, device="cuda")
    old, mask = -torch.rand(ts, generator=gen, device="cuda") - 7.0, torch.rand(ts, generator=gen, device="cuda") < 0.9
    adv, grp = torch.randn(7, generator=gen, device="cuda"), _grp(lens)
    ws = torch.empty(binding.token_logprobs_workspace_bytes(3, 7, ts, vocab), dtype=torch.uint8, device="cuda")
    wp = torch.empty(binding.policy_loss_workspace_bytes(3, 7, ts), dtype=torch.uint8, device="cuda")
    lp = (torch.empty(ts, device="cuda"), torch.empty(ts, device="cuda"))
    loss = (torch.empty(4, device="cuda"), torch.empty(ts, device="cuda"))
    grad = (torch.empty_like(last), torch.empty_like(suf))

    def step():
        binding.token_logprobs(last, suf, tok, *grp, 5, out=lp, workspace=ws)
        binding.policy_loss(lp[0], adv, *grp[1:], logp_old=old, logp_ref=old, mask=mask, beta=0.05, out=loss, workspace=wp)
        binding.token_logprobs_bwd(last, suf, tok, lp[1], loss[1], *grp, 5, out=grad, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    outs = lp + loss + grad
    eager = [t.clone() for t in outs]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for rep in range(3):
        for t in outs:
            t.fill_(float("nan"))
        ws.fill_(255)
        wp.fill_(255)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(outs, eager)):
            assert torch.equal(a, b), f"replay {rep}, output {i}"


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("lens,vocab", [(((5, 3), (9, 40), tuple([30] * 9 + [25] * 40)), 301),
                                        (((2,), (700,), tuple([13] * 700)), 40)])
def test_many_short_rows(lens, vocab, dt):
    """Many rows of few elements, whole groups' first tokens among them: every row against float64, and the gradient."""
    from paper_2506_05433_amd import binding
    ts, ng = sum(lens[2]), len(lens[0])
    print(f"[logprobs] {ts} rows of {vocab} {dt}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    last, suf = (torch.randn(n, vocab, generator=gen, device="cuda").mul_(2).to(dt) for n in (ng, ts))
    tok = torch.randint(0, vocab, (ts,), generator=gen, device="cuda")
    d = torch.randn(ts, generator=gen, device="cuda")
    lp, lse, ent = binding.token_logprobs(last, suf, tok, *_grp(lens), sum(lens[0]), entropy=True)
    cu = np.concatenate([[0], np.cumsum(lens[2])])
    group = np.repeat(np.repeat(np.arange(ng), lens[1]), lens[2])
    first = np.isin(np.arange(ts), cu[:-1])
    src = torch.from_numpy(np.where(first, ng * 0 + group, ng + np.arange(ts) - 1)).cuda()
    x = torch.cat([last, suf]).double()[src]
    ref = torch.log_softmax(x, 1)
    zmax = float(x.abs().max())
    tol = 2.0 ** -22 * (zmax + vocab / 64 + 40)   # one wave a row: vocab / 64 additions in a row at most
    assert float((lp.double() - ref.gather(1, tok[:, None])[:, 0]).abs().max()) <= tol
    assert float((lse.double() - torch.logsumexp(x, 1)).abs().max()) <= tol
    assert float((ent.double() + (ref.exp() * ref).sum(1)).abs().max()) <= tol * (1 + 2 * zmax)
    gl, gs = binding.token_logprobs_bwd(last, suf, tok, lse, d, *_grp(lens), sum(lens[0]))
    g = -ref.exp() * d.double()[:, None]
    g[torch.arange(ts, device="cuda"), tok] += d.double()
    want = torch.zeros(ng + ts, vocab, dtype=torch.float64, device="cuda").index_add_(0, src, g)
    w = torch.zeros(ng + ts, dtype=torch.float64, device="cuda").index_add_(0, src, d.double().abs())
    lim = U[dt] * want.abs() * 1.01 + (2.0 ** -23 * (2 * zmax + 8) + tol + max(lens[1]) * 2.0 ** -23) * w[:, None]
    assert bool(((torch.cat([gl, gs]).double() - want).abs() <= lim).all())


def test_long_batches_without_a_mask_and_many_members():
    """The paths for more tokens than one workgroup takes, without a mask; and for more members than fit LDS."""
    from paper_2506_05433_amd import binding
    for lens, average in ((((1, 1), (3, 2), (5000, 0, 7001, 300, 40)), "group"), (((1, 1), (3, 2), (5000, 0, 7001, 300, 40)), "token"),
                          (((1,), (4200,), tuple(i % 3 for i in range(4200))), "group")):
        ts, ns = sum(lens[2]), len(lens[2])
        print(f"[policy] {ns} members, {ts} tokens, {average}", flush=True)
        rng = np.random.default_rng(ts)
        lp = -rng.uniform(0, 5, ts).astype(np.float32)
        old, adv = (lp + 0.3 * rng.standard_normal(ts)).astype(np.float32), rng.standard_normal(ns).astype(np.float32)
        want, grad = policy_loss_oracle(lens[1], lens[2], lp, adv, old, average=average)
        _, cs, gs = _grp(lens)
        t = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
        stats, d = binding.policy_loss(t(lp), t(adv), cs, gs, logp_old=t(old), average=average)
        assert (np.abs(stats.double().cpu().numpy() - want) <= 2.0 ** -24 * np.abs(want) + 1e-12 * (1 + np.abs(want).sum())).all()
        assert (np.abs(d.double().cpu().numpy() - grad) <= 2.0 ** -24 * np.abs(grad) + 1e-14).all()


def test_policy_loss_of_no_groups_is_zero():
    from paper_2506_05433_amd import binding
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    none = torch.empty(0, device="cuda")
    out = (torch.full((4,), 3.0, device="cuda"), none)
    binding.policy_loss(none, none, i32([0]), i32([]), out=out)
    assert bool((out[0] == 0).all())


def test_no_response_rows():
    """Members without a row: nothing to predict, logits are not read (they may be NULL); the gradient is zeros."""
    from paper_2506_05433_amd import binding
    cp, cs, gs = _grp(((3, 0), (2, 1), (0, 0, 0)))
    ws = torch.empty(binding.token_logprobs_workspace_bytes(2, 3, 0, 50), dtype=torch.uint8, device="cuda")
    p = lambda t: t.data_ptr()  # noqa: E731
    st = binding.lib().pg_token_logprobs(1, 8, 2, 3, 3, 0, p(cp), p(cs), p(gs), 50, 1.0, None, 50, None, 50, None, None, None,
                                         None, p(ws), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert st == 0, binding.lib().pg_last_error()
    torch.cuda.synchronize()
    none = torch.empty(0, device="cuda")
    last = torch.full((2, 50), float("nan"), device="cuda")
    out = binding.token_logprobs(last, none.view(0, 50), none.long(), cp, cs, gs, 3, entropy=True)
    assert [t.numel() for t in out] == [0, 0, 0]
    gl, _ = binding.token_logprobs_bwd(last, none.view(0, 50), none.long(), none, none, cp, cs, gs, 3)
    assert bool((gl == 0).all())


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [1, 13, 3000])
def test_rows_of_nothing_but_nan(dt, vocab):
    """A row of NaN, and one of NaN and -inf, is NaN throughout, not a row with nothing left; so is its gradient."""
    from paper_2506_05433_amd import binding
    last = torch.full((1, vocab), float("nan"), dtype=dt, device="cuda")
    suf = torch.zeros(4, vocab, dtype=dt, device="cuda")
    suf[0], suf[1], suf[1, vocab // 2] = float("nan"), -float("inf"), float("nan")
    tok, g = torch.zeros(4, dtype=torch.int64, device="cuda"), _grp(((2,), (1,), (4,)))
    lp, lse, ent = binding.token_logprobs(last, suf, tok, *g, 2, entropy=True)
    for t in (lp, lse, ent):
        assert t.isnan().tolist() == [True, True, True, False]
    gl, gs = binding.token_logprobs_bwd(last, suf, tok, lse, torch.ones(4, device="cuda"), *g, 2)
    assert bool(gl.isnan().all()) and gs.isnan().all(1).tolist() == [True, True, False, False]
    assert not bool(gs[2:].isnan().any())


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_rows_of_the_lowest_value_divided_by_a_temperature(dt):
    """The log-sum-exp of such a row is out of fp32's range; its log-probabilities and gradient are a uniform row's."""
    from paper_2506_05433_amd import binding
    vocab, temp = 13, 0.5
    suf = torch.zeros(2, vocab, dtype=dt, device="cuda")
    suf[0] = torch.finfo(dt).min
    tok, g = torch.tensor([0, 4], device="cuda"), _grp(((0,), (1,), (2,)))
    last = torch.zeros(1, vocab, dtype=dt, device="cuda")
    lp, lse = binding.token_logprobs(last, suf, tok, *g, 0, temperature=temp)
    # ln 13 < 4 by 13 terms of 1: its rounding and the function's, 2^-21 at most
    assert abs(lp[1].item() + np.log(vocab)) <= 2.0 ** -20 and lse[1].item() == torch.finfo(torch.float32).min
    _, gs = binding.token_logprobs_bwd(last, suf, tok, lse, torch.ones(2, device="cuda"), *g, 0, temperature=temp)
    want = np.full(vocab, -1.0 / vocab)
    want[4] += 1.0
    u = U[dt] + 2.0 ** -21  # the result's rounding; w, p and the target's sum, three of fp32
    assert (np.abs(gs[0].double().cpu().numpy() - want / temp) <= u * np.abs(want) / temp).all()
    assert bool((gs[1] == 0).all())


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [37, 9001])
def test_a_row_with_thousands_of_targets(dt, vocab):
    """One group of more members than a workgroup keeps at hand, some of them empty, many with the same first token."""
    from paper_2506_05433_amd import binding
    rng = np.random.default_rng(vocab)
    size = 2311
    lens = ((3,), (size,), tuple(int(x) for x in rng.integers(0, 3, size)))
    ts = sum(lens[2])
    print(f"[logprobs] {size} members, {ts} rows, vocab {vocab} {dt}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    last, _ = _logits(1, vocab, 0, 0, dt, gen)
    suf, _ = _logits(ts, vocab, 0, 0, dt, gen)
    tok = torch.randint(0, min(vocab, 1500), (ts,), generator=gen, device="cuda")
    tok[::7] = -1
    d = torch.randn(ts, generator=gen, device="cuda")
    d[::5] = 0.0
    g = _grp(lens)
    _, lse = binding.token_logprobs(last, suf, tok, *g, 3)
    gl, gs = binding.token_logprobs_bwd(last, suf, tok, lse, d, *g, 3)
    dn, tn, at = d.double().cpu().numpy(), tok.cpu().numpy(), np.concatenate([[0], np.cumsum(lens[2])])
    firsts = [r for r, s in zip(at, lens[2]) if s > 0 and tn[r] >= 0]
    x = to_host(last)[0].astype(np.float64)
    p = np.exp(x - x.max())
    p /= p.sum()
    add, mag = np.zeros(vocab), np.zeros(vocab)
    np.add.at(add, tn[firsts], dn[firsts])
    np.add.at(mag, tn[firsts], np.abs(dn[firsts]))
    want = add - dn[firsts].sum() * p
    # sums of at most n terms: n 2^-24 of the terms' magnitudes; p: its argument's error, as at the top; one fused product
    n, zmax = len(firsts), np.abs(x).max()
    ptol = 2.0 ** -23 * (2 * zmax + 8) + 2.0 ** -22 * (zmax + vocab / 256 + 40)
    lim = n * 2.0 ** -24 * (mag + mag.sum() * p) + (ptol + 2.0 ** -23) * mag.sum() * p + 1.01 * U[dt] * np.abs(want)
    lim += U[dt] * lim + 2.0 ** -23 * mag
    err = np.abs(to_host(gl)[0].astype(np.float64) - want)
    assert (err <= lim).all(), (err / lim).max()
    # the policy loss over that group: weights 1 / (members x tokens)
    adv = torch.randn(size, generator=gen, device="cuda")
    stats, dl = binding.policy_loss(d, adv, g[1], g[2])
    sizes = np.array(lens[2])
    w = np.repeat(1.0 / (size * np.maximum(sizes, 1)), sizes)
    a = np.repeat(adv.double().cpu().numpy(), sizes)
    assert (np.abs(dl.double().cpu().numpy() + w * a) <= 2.0 ** -24 * np.abs(w * a) + 1e-14).all()
    assert abs(stats[0].item() + (w * a).sum()) <= 2.0 ** -24 * abs((w * a).sum()) + 1e-12


def test_policy_loss_of_many_groups():
    """More groups than the planner takes at a time, some without members, and more tokens than one workgroup takes."""
    from paper_2506_05433_amd import binding
    rng = np.random.default_rng(8)
    groups = rng.integers(0, 4, 2500)
    sizes = rng.integers(0, 6, groups.sum())
    ts = int(sizes.sum())
    assert ts > 8192
    adv = torch.from_numpy(rng.standard_normal(len(sizes)).astype(np.float32)).cuda()
    stats, dl = binding.policy_loss(torch.zeros(ts, device="cuda"), adv, _cu(sizes), torch.tensor(groups, dtype=torch.int32, device="cuda"))
    w = np.repeat(1.0 / ((groups > 0).sum() * np.repeat(groups, groups) * np.maximum(sizes, 1)), sizes)
    a = np.repeat(adv.double().cpu().numpy(), sizes)
    assert (np.abs(dl.double().cpu().numpy() + w * a) <= 2.0 ** -24 * np.abs(w * a) + 1e-14).all()
    assert abs(stats[0].item() + (w * a).sum()) <= 2.0 ** -24 * abs((w * a).sum()) + 1e-12
