"""The calls around and beside the grouped attention that a GRPO step makes, over the range their users call them on.

* linear attention with a decay for each head over a shared prefix: layers of hybrid models (`linear_fwd`,
  `linear_bwd`, both in turn as a training step: `linear_step`; `prefill`: the forward that also hands the states to
  a decoder), and its recurrent form for single tokens (`decode`);
* log-probabilities of the response tokens from the logits, where the first token of every response is predicted by
  its group's last prefix row (`logprobs`, `logprobs_bwd`);
* the clipped policy loss with a KL term and its gradient (`policy`).

A case names how its lengths are drawn (`lengths` is the seed of that draw), so its work is known without its
tensors; the tensors come from the seed given to prepare(). Outputs and workspaces are allocated once, as a program
that runs many layers and steps keeps them.
"""
import math
import random

import torch

own = False

LIN = ("linear_fwd", "linear_bwd", "linear_step", "prefill")


def _attn(name, op, dtype, groups, size, p, s, heads, d, lengths=0):
    c = {"op": op, "dtype": dtype, "n_groups": groups, "group_size": size, "p_lo": p[0], "p_hi": p[1], "s_lo": s[0],
         "s_hi": s[1], "h_q": heads[0], "h_kv": heads[1], "d": d, "lengths": lengths}
    return {"name": name, **c} if name else c


def _rows(name, op, dtype, groups, size, s, vocab=0, lengths=0, **more):
    c = {"op": op, "dtype": dtype, "n_groups": groups, "group_size": size, "p_lo": 1, "p_hi": 64, "s_lo": s[0],
         "s_hi": s[1], "vocab": vocab, "lengths": lengths, **more}
    return {"name": name, **c} if name else c


def listed():
    return [
        # unit-test sized training step of one layer in fp32: launches and latency
        _attn("linear_step_tiny_fp32", "linear_step", "fp32", 1, 4, (64, 64), (16, 32), (2, 2), 64),
        # scoring one prompt with 8 answers: forward only
        _attn("linear_fwd_single_group", "linear_fwd", "bf16", 1, 8, (4096, 4096), (256, 1024), (32, 8), 128),
        # the backward of a long shared document with short answers
        _attn("linear_bwd_long_prefix", "linear_bwd", "bf16", 1, 16, (16384, 16384), (128, 512), (32, 8), 128),
        # the largest: training step of one layer on a large rollout group, most of its rows responses
        _attn("linear_step_large_group", "linear_step", "bf16", 1, 64, (8192, 8192), (128, 2048), (40, 8), 128),
        # prompts read for decoding: many ragged groups, 64-wide heads, the states handed on
        _attn("prefill_ragged_d64", "prefill", "bf16", 7, 6, (151, 3001), (1, 90), (16, 4), 64),
        # one token for each of 128 running sequences (8 prompts x 16 samples)
        _attn("decode_128", "decode", "bf16", 8, 16, (1, 1), (1, 1), (64, 8), 128),
        # one token for a handful of sequences: latency
        _attn("decode_5", "decode", "bf16", 1, 5, (1, 1), (1, 1), (32, 8), 128),
        # log-probabilities (and the entropy that trainers log) of 8 answers to one prompt
        _rows("logprobs_single_group", "logprobs", "bf16", 1, 8, (256, 1024), 131072, entropy=True),
        # their gradient on ragged groups, with an odd vocabulary whose rows start at any alignment
        _rows("logprobs_bwd_odd_vocab", "logprobs_bwd", "bf16", 7, 6, (17, 900), 50001),
        # fp32 logits, as trainers that upcast their last layer have them
        _rows("logprobs_bwd_fp32", "logprobs_bwd", "fp32", 2, 4, (40, 300), 32000),
        # the loss of one group: a few thousand tokens, latency
        _rows("policy_single_group", "policy", "fp32", 1, 8, (256, 1024), average="group", ref=True, mask=False),
        # the loss of a packed batch, with a reference policy and tokens masked out
        _rows("policy_packed", "policy", "fp32", 8, 16, (64, 4096), average="token", ref=True, mask=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A call of the ranges above: kind, type, head geometry or vocabulary, and lengths."""
    op = rng.choice(["linear_fwd", "linear_bwd", "linear_step", "prefill", "decode", "logprobs", "logprobs_bwd", "policy"])
    seed = rng.randrange(1 << 30)
    if op in LIN or op == "decode":
        h_kv, ratio, d = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128])
        dtype = "fp32" if rng.random() < 0.2 else "bf16"
        if op == "decode":
            return _attn(None, op, dtype, _log_int(rng, 1, 12), _log_int(rng, 1, 16), (1, 1), (1, 1), (ratio * h_kv, h_kv),
                         d, seed)
        p, s = _log_int(rng, 40, 16384), _log_int(rng, 2, 2048)
        groups, size = _log_int(rng, 1, 8), _log_int(rng, 1, 64)
        if dtype == "fp32":
            p, s, groups, size = min(p, 2000), min(s, 400), min(groups, 3), min(size, 12)
        p_lo = p if rng.random() < 0.5 else max(1, p // rng.randint(2, 16))
        c = _attn(None, op, dtype, groups, size, (p_lo, p), (max(0, s // 8), s), (ratio * h_kv, h_kv), d, seed)
        while work(c)["flops"] > 3e11 or work(c)["bytes"] > 4e9:  # below the largest listed step
            c["group_size"], c["p_hi"] = max(1, c["group_size"] // 2), max(c["p_lo"], c["p_hi"] // 2)
            c["n_groups"] = max(1, c["n_groups"] // 2)
        return c
    if op == "policy":
        s = _log_int(rng, 16, 4096)
        return _rows(None, op, "fp32", _log_int(rng, 1, 8), _log_int(rng, 2, 64), (s // 8, s), 0, seed,
                     average=rng.choice(["group", "token"]), ref=rng.random() < 0.7, mask=rng.random() < 0.5)
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    vocab = _log_int(rng, 1000, 140000)
    groups, size = _log_int(rng, 1, 6), _log_int(rng, 1, 16)
    most = 5e8 / (vocab * groups * size)  # elements: below the listed backward
    s = max(2, min(_log_int(rng, 4, 1500), int(most)))
    more = {"entropy": rng.random() < 0.5} if op == "logprobs" else {}
    return _rows(None, op, dtype, groups, size, (s // 6 if groups * size > 3 else max(1, s // 6), s), vocab, seed, **more)


def _lengths(case):
    r = random.Random(case["lengths"])
    lo, hi = math.log(case["p_lo"]), math.log(case["p_hi"])
    p = [min(case["p_hi"], max(case["p_lo"], int(round(math.exp(r.uniform(lo, hi)))))) for _ in range(case["n_groups"])]
    s = [r.randint(case["s_lo"], case["s_hi"]) for _ in range(case["n_groups"] * case["group_size"])]
    return p, s


def _cu(x):
    c = [0]
    for v in x:
        c.append(c[-1] + v)
    return c


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _dt(case)

    def normal(*shape, std=1.0):
        # filled in the type that is kept, a slice at a time where it is large
        out = torch.empty(shape, device="cuda", dtype=dt)
        flat = out.view(-1)
        for i in range(0, flat.numel(), 1 << 28):
            part = flat[i:i + (1 << 28)]
            part.copy_(torch.randn(part.shape, generator=g, device="cuda").mul_(std))
        return out

    def normal32(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    st = {"case": case}
    op = case["op"]
    if op in LIN or op == "decode":
        hq, hkv, d = case["h_q"], case["h_kv"], case["d"]
        st["scale"] = 1.0 / math.sqrt(d)
        # half-lives from a few tokens to thousands, as retention-style layers give their heads
        st["log_decay"] = -torch.exp(math.log(2e-4) + torch.rand(hkv, generator=g, device="cuda") * (math.log(0.3) - math.log(2e-4)))
    if op == "decode":
        n = case["n_groups"] * case["group_size"]
        st.update(q=normal(n, hq, d), k=normal(n, hkv, d), v=normal(n, hkv, d),
                  state=4.0 * normal32(n, hkv, d, d), o=torch.empty((n, hq, d), device="cuda", dtype=dt),
                  state_out=torch.empty((n, hkv, d, d), device="cuda"))
        return st
    p, s = _lengths(case)
    sizes = [case["group_size"]] * case["n_groups"]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    st.update(cu_prefix=i32(_cu(p)), cu_suffix=i32(_cu(s)), group_sizes=i32(sizes), tp=sum(p), ts=sum(s))
    tp, ts, ng, ns = sum(p), sum(s), len(p), len(s)
    if op in LIN:
        for part, rows in (("pre", tp), ("suf", ts)):
            st["q_" + part], st["k_" + part], st["v_" + part] = normal(rows, hq, d), normal(rows, hkv, d), normal(rows, hkv, d)
            if op in ("linear_bwd", "linear_step"):
                st["do_" + part] = normal(rows, hq, d)
        if own:
            from paper_2506_05433_amd import binding
            q, k = st["q_pre"], st["k_pre"]
            args = (ng, ns, tp, ts, hq, hkv, d)
            if op != "linear_bwd":
                st["out_f"] = (torch.empty_like(q), torch.empty_like(st["q_suf"]))
                st["ws_f"] = torch.empty(binding.linear_workspace_bytes("fwd", *args), dtype=torch.uint8, device="cuda")
            if op == "prefill":
                st["out_f"] += (torch.empty((ng, hkv, d, d), device="cuda"), torch.empty((ns, hkv, d, d), device="cuda"))
            if op in ("linear_bwd", "linear_step"):
                st["out_b"] = (torch.empty_like(q), torch.empty_like(k), torch.empty_like(k), torch.empty_like(st["q_suf"]),
                               torch.empty_like(st["k_suf"]), torch.empty_like(st["k_suf"]))
                st["ws_b"] = torch.empty(binding.linear_workspace_bytes("bwd", *args), dtype=torch.uint8, device="cuda")
        return st
    if op == "policy":
        lp = -1.5 * torch.rand(ts, generator=g, device="cuda") ** 3 * 4
        st.update(logp=lp, logp_old=lp + 0.15 * normal32(ts), logp_ref=lp + 0.3 * normal32(ts) if case["ref"] else None,
                  mask=(torch.rand(ts, generator=g, device="cuda") < 0.8) if case["mask"] else None,
                  advantages=normal32(ns), beta=0.04 if case["ref"] else 0.0, clip=(0.2, 0.28))
        if own:
            from paper_2506_05433_amd import binding
            st["out"] = (torch.empty(4, device="cuda"), torch.empty(ts, device="cuda"))
            st["ws"] = torch.empty(binding.policy_loss_workspace_bytes(ng, ns, ts), dtype=torch.uint8, device="cuda")
        return st
    vocab = case["vocab"]
    # logits of a trained model: a few tokens stand out, the targets among them more often than not
    st.update(logits_last=normal(ng, vocab, std=2.5), logits_suf=normal(ts, vocab, std=2.5), temperature=0.9,
              tokens=torch.randint(0, vocab, (ts,), generator=g, device="cuda", dtype=torch.int64))
    if op == "logprobs_bwd":
        st["dlogp"] = normal32(ts) / max(1, ts)
        own_lse = _plain_logprobs(st, False)[1]
        st["lse"] = own_lse
    if own:
        from paper_2506_05433_amd import binding
        st["ws"] = torch.empty(binding.token_logprobs_workspace_bytes(ng, ns, ts, vocab), dtype=torch.uint8, device="cuda")
        if op == "logprobs":
            st["out"] = (torch.empty(ts, device="cuda"), torch.empty(ts, device="cuda")) + ((torch.empty(ts, device="cuda"),) if case["entropy"] else ())
        else:
            st["out"] = (torch.empty_like(st["logits_last"]), torch.empty_like(st["logits_suf"]))
    return st


def run(st):
    return _own(st) if own else _plain(st)


def _own(st):
    from paper_2506_05433_amd import binding as b
    op = st["case"]["op"]
    if op == "decode":
        return b.linear_step(st["q"], st["k"], st["v"], st["state"], st["log_decay"], st["scale"], out=(st["o"], st["state_out"]))
    grp = (st["cu_prefix"], st["cu_suffix"], st["group_sizes"])
    if op in LIN:
        qkv = [st[n] for n in ("q_pre", "k_pre", "v_pre", "q_suf", "k_suf", "v_suf")]
        res = ()
        if op != "linear_bwd":
            res += tuple(b.linear_fwd(*qkv, st["log_decay"], *grp, st["scale"], states=op == "prefill", out=st["out_f"], workspace=st["ws_f"]))
        if op in ("linear_bwd", "linear_step"):
            res += tuple(b.linear_bwd(*qkv, st["do_pre"], st["do_suf"], st["log_decay"], *grp, st["scale"], out=st["out_b"], workspace=st["ws_b"]))
        return res
    if op == "logprobs":
        return b.token_logprobs(st["logits_last"], st["logits_suf"], st["tokens"], *grp, st["tp"], temperature=st["temperature"],
                                entropy=st["case"]["entropy"], out=st["out"], workspace=st["ws"])
    if op == "logprobs_bwd":
        return b.token_logprobs_bwd(st["logits_last"], st["logits_suf"], st["tokens"], st["lse"], st["dlogp"], *grp, st["tp"],
                                    temperature=st["temperature"], out=st["out"], workspace=st["ws"])
    return b.policy_loss(st["logp"], st["advantages"], st["cu_suffix"], st["group_sizes"], logp_old=st["logp_old"], logp_ref=st["logp_ref"],
                         mask=st["mask"], clip=st["clip"], beta=st["beta"], average=st["case"]["average"], out=st["out"], workspace=st["ws"])


def _plain(st):
    op = st["case"]["op"]
    if op == "decode":
        return _plain_decode(st)
    if op == "policy":
        return _plain_policy(st)
    if op == "logprobs":
        return _plain_logprobs(st, st["case"]["entropy"])
    if op == "logprobs_bwd":
        return _plain_logprobs_bwd(st)
    res = ()
    qs, ks, vs = [(st[n + "_pre"].float(), st[n + "_suf"].float()) for n in "qkv"]
    dt = st["q_pre"].dtype
    if op != "linear_bwd":
        o, states = _plain_linear(st, qs, ks, vs)
        res += tuple((x * st["scale"]).to(dt) for x in o) + (tuple(states) if op == "prefill" else ())
    if op in ("linear_bwd", "linear_step"):
        do = (st["do_pre"].float(), st["do_suf"].float())
        dq = _plain_linear(st, do, vs, ks)[0]
        dk = _plain_linear(st, vs, do, qs, reverse=True)[0]
        dv = _plain_linear(st, ks, qs, do, reverse=True)[0]
        res += tuple((x[i] * st["scale"]).to(dt) for i in (0, 1) for x in (dq, dk, dv))
    return res


CHUNK = 64


def _padded(x, at, valid, heads):
    """Rows `at` [n, T] of x [rows, h, d] as [n, chunks, CHUNK, heads, h / heads, d], zero where not valid."""
    y = torch.zeros(at.shape + x.shape[1:], device=x.device)
    y[valid] = x[at[valid]]
    return y.view(at.shape[0], -1, CHUNK, heads, x.shape[1] // heads, x.shape[2])


def _plain_walk(q, k, v, ld, cu, init, reverse):
    """o_t = sum_{s<=t} l^(t-s) (q_t.k_s) v_s + l^(t+1) q_t init of every segment of `cu`, rows taken in order or backwards,
    summed over the heads of k and v that share a decay; and the state after each segment's last row."""
    h, n, d = ld.numel(), cu.numel() - 1, q.shape[2]
    lens = (cu[1:] - cu[:-1]).long()
    span = -(-max(1, int(lens.max()) if n else 1) // CHUNK) * CHUNK
    i = torch.arange(span, device=q.device)
    valid = i[None] < lens[:, None]
    at = torch.where(valid, (cu[1:, None].long() - 1 - i) if reverse else (cu[:-1, None].long() + i), 0)
    qp, kp, vp = (_padded(x, at, valid, h) for x in (q, k, v))
    c = torch.arange(CHUNK, device=q.device)
    gap = (c[:, None] - c[None]).float()
    decay = torch.exp(ld[:, None, None] * gap.clamp_min(0)) * (gap >= 0)
    w = torch.einsum("nbihad,nbjhed->nbhaeij", qp, kp) * decay[None, None, :, None, None]
    o = torch.einsum("nbhaeij,nbjhed->nbihad", w, vp)
    # the state before each chunk: the segment's initial state and the earlier chunks' shares
    share = torch.einsum("nbjhed,nbjhef->nbhdf", kp * torch.exp(ld[:, None] * (CHUNK - 1 - c)[None]).t()[None, None, :, :, None, None], vp)
    b = torch.arange(span // CHUNK, device=q.device)
    back = (b[:, None] - 1 - b[None]).float()
    carry = torch.exp(ld[:, None, None] * CHUNK * back.clamp_min(0)) * (back >= 0)
    before = torch.matmul(carry, share.permute(0, 2, 1, 3, 4).reshape(n, h, b.numel(), d * d)).view(n, h, b.numel(), d, d)
    before = before + torch.exp(ld[:, None] * CHUNK * b[None])[None, :, :, None, None] * init[:, :, None]
    o = o + torch.einsum("nbihad,nhbdf->nbihaf", qp, before) * torch.exp(ld[None] * (c[:, None] + 1))[None, None, :, :, None, None]
    out = torch.zeros_like(q)
    out[at[valid]] = o.reshape(n, span, -1, d)[valid]
    left = (lens[:, None] - 1 - i[None]).clamp_min(0)
    last = kp.view(n, span, h, -1, d) * torch.exp(ld * left[:, :, None])[..., None, None]
    state = torch.einsum("nthed,nthef->nhdf", last, vp.view(n, span, h, -1, d)) + torch.exp(ld * lens[:, None])[..., None, None] * init
    return out, state


def _plain_linear(st, q, k, v, reverse=False):
    """The walk over the prefixes and the members, each from the state that the other leaves it."""
    ld, cp, cs = st["log_decay"], st["cu_prefix"], st["cu_suffix"]
    d, ng, ns = q[0].shape[2], cp.numel() - 1, cs.numel() - 1
    group = torch.repeat_interleave(torch.arange(ng, device=ld.device), st["group_sizes"].long())
    zero = lambda n: torch.zeros((n, ld.numel(), d, d), device=ld.device)  # noqa: E731
    if not reverse:
        o_pre, s_pre = _plain_walk(q[0], k[0], v[0], ld, cp, zero(ng), False)
        o_suf, s_suf = _plain_walk(q[1], k[1], v[1], ld, cs, s_pre[group], False)
    else:
        o_suf, s_suf = _plain_walk(q[1], k[1], v[1], ld, cs, zero(ns), True)
        o_pre, s_pre = _plain_walk(q[0], k[0], v[0], ld, cp, zero(ng).index_add(0, group, s_suf), True)
    return (o_pre, o_suf), (s_pre, s_suf)


def _plain_decode(st):
    q, k, v = st["q"].float(), st["k"].float(), st["v"].float()
    n, hkv, d = k.shape
    state = torch.exp(st["log_decay"])[None, :, None, None] * st["state"] + k[..., :, None] * v[..., None, :]
    o = torch.matmul(q.view(n, hkv, -1, d), state) * st["scale"]
    return o.view(q.shape).to(st["q"].dtype), state


def _targets(st):
    """For every response row: its member's group, whether it is its member's first, and whether it is its last."""
    cs, ts = st["cu_suffix"].long(), st["ts"]
    row = torch.arange(ts, device=cs.device)
    member = torch.searchsorted(cs, row, right=True) - 1
    group = torch.repeat_interleave(torch.arange(st["group_sizes"].numel(), device=cs.device), st["group_sizes"].long())[member]
    return group, row == cs[member], row == cs[member + 1] - 1


def _plain_lse(x):
    m = x.amax(1)
    return m + torch.log(torch.exp(x - m[:, None]).sum(1))


def _plain_logprobs(st, entropy):
    group, first, _ = _targets(st)
    before = (torch.arange(st["ts"], device=group.device) - 1).clamp_min(0)
    tok = st["tokens"].long()
    xl, xs = st["logits_last"].float() / st["temperature"], st["logits_suf"].float() / st["temperature"]
    ll, ls = _plain_lse(xl), _plain_lse(xs)
    lse = torch.where(first, ll[group], ls[before])
    res = (torch.where(first, xl[group, tok], xs[before, tok]) - lse, lse)
    if entropy:
        el, es = ((l - (torch.exp(x - l[:, None]) * x).sum(1)) for x, l in ((xl, ll), (xs, ls)))
        res += (torch.where(first, el[group], es[before]),)
    return res


def _plain_logprobs_bwd(st):
    group, first, last = _targets(st)
    dt, tok, d = st["logits_suf"].dtype, st["tokens"].long(), st["dlogp"]
    # response rows predict their successor
    row = torch.nonzero(~last).view(-1)
    lse = torch.zeros_like(st["lse"]).index_copy(0, row, st["lse"][row + 1])
    w = torch.zeros_like(d).index_copy(0, row, d[row + 1])
    gs = torch.exp(st["logits_suf"].float() / st["temperature"] - lse[:, None]) * -w[:, None]
    gs[row, tok[row + 1]] += d[row + 1]
    # the last prefix row of a group predicts the first token of each of its members
    row = torch.nonzero(first).view(-1)
    ng = st["logits_last"].shape[0]
    lse = torch.zeros(ng, device=d.device).index_copy(0, group[row], st["lse"][row])
    w = torch.zeros(ng, device=d.device).index_add(0, group[row], d[row])
    gl = torch.exp(st["logits_last"].float() / st["temperature"] - lse[:, None]) * -w[:, None]
    gl.index_put_((group[row], tok[row]), d[row], accumulate=True)
    return (gl / st["temperature"]).to(dt), (gs / st["temperature"]).to(dt)


def _plain_policy(st):
    # in 64 bits: the ratio next to the clip's border, and long sums of terms of both signs
    cs, ts = st["cu_suffix"].long(), st["ts"]
    ns, sizes = cs.numel() - 1, st["group_sizes"].double()
    member = torch.searchsorted(cs, torch.arange(ts, device=cs.device), right=True) - 1
    keep = torch.ones(ts, device=cs.device, dtype=torch.float64) if st["mask"] is None else st["mask"].double()
    if st["case"]["average"] == "group":
        count = torch.zeros(ns, device=cs.device, dtype=torch.float64).index_add(0, member, keep)
        per_member = 1.0 / (sizes.repeat_interleave(st["group_sizes"].long()) * (sizes > 0).sum())
        w = keep * (per_member / count.clamp_min(1.0))[member]
    else:
        w = keep / keep.sum().clamp_min(1.0)
    lp, a = st["logp"].double(), st["advantages"].double()[member]
    r = torch.exp(lp - st["logp_old"].double())
    lo, hi = 1.0 - st["clip"][0], 1.0 + st["clip"][1]
    cut = ((a > 0) & (r > hi)) | ((a < 0) & (r < lo))
    term = -torch.minimum(r * a, r.clamp(lo, hi) * a)
    grad = torch.where(cut, 0.0, -r * a)
    kl = torch.zeros_like(lp)
    if st["logp_ref"] is not None:
        x = st["logp_ref"].double() - lp
        kl = torch.exp(x) - x - 1.0
        grad = grad + st["beta"] * (1.0 - torch.exp(x))
    stats = torch.stack([(w * (term + st["beta"] * kl)).sum(), (w * term).sum(), (w * kl).sum(), (w * cut).sum()])
    return stats.float(), (w * grad).float()


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    op = case["op"]
    if op == "decode":
        n, hq, hkv, d = case["n_groups"] * case["group_size"], case["h_q"], case["h_kv"], case["d"]
        return {"bytes": n * (e * d * (2 * hq + 2 * hkv) + 8 * hkv * d * d), "flops": n * (3 * hkv + 2 * hq) * d * d}
    p, s = _lengths(case)
    rows = sum(s)
    if op in LIN:
        rows += sum(p)
        hq, hkv, d = case["h_q"], case["h_kv"], case["d"]
        # the recurrence's products: forward S += k v^T and q S; backward S, R and three products with them
        fwd, bwd = (2 * hkv + 2 * hq) * d * d, (2 * hkv + 2 * hq) * d * d + (2 * hq + 4 * hkv) * d * d
        nb, nf = 0, 0
        if op != "linear_bwd":
            nb, nf = nb + rows * e * d * (2 * hq + 2 * hkv), nf + rows * fwd
        if op == "prefill":
            nb += 4 * hkv * d * d * (len(p) + len(s))
        if op in ("linear_bwd", "linear_step"):
            nb, nf = nb + rows * e * d * (3 * hq + 4 * hkv), nf + rows * bwd
        return {"bytes": nb, "flops": nf}
    if op == "policy":
        # log-probabilities new, old and (where there is one) of the reference policy, the gradient, the mask
        return {"bytes": rows * (12 + 4 * case["ref"] + case["mask"]) + 4 * len(s), "flops": 20 * rows}
    used = rows - sum(1 for x in s if x) + len(p)  # a member's last row predicts nothing
    if op == "logprobs":
        return {"bytes": used * case["vocab"] * e + rows * (8 + 8 + (4 if case["entropy"] else 0)), "flops": 4 * used * case["vocab"]}
    return {"bytes": used * case["vocab"] * e + (rows + len(p)) * case["vocab"] * e + rows * 16, "flops": 4 * used * case["vocab"]}


def exact(case, seed):
    """The operators' definitions in 64 bits, row against row, without states or chunks."""
    st = prepare(case, seed)
    op = case["op"]
    f8 = torch.float64
    if op == "decode":
        q, k, v = (st[n].to(f8) for n in "qkv")
        rep = case["h_q"] // case["h_kv"]
        lam = st["log_decay"].to(f8).exp()
        new = torch.einsum("h,nhij->nhij", lam, st["state"].to(f8)) + torch.einsum("nhi,nhj->nhij", k, v)
        return torch.einsum("nhi,nhij->nhj", q, new.repeat_interleave(rep, 1)) * st["scale"], new
    p, s = _lengths(case)
    size = case["group_size"]
    if op in LIN:
        hq, hkv, d = case["h_q"], case["h_kv"], case["d"]
        rep = hq // hkv
        cp, cs = _cu(p), _cu(s)
        pairs = sum(x * x / 2 for x in p) + sum(x * (p[m // size] + x / 2) for m, x in enumerate(s))
        if pairs * hq * d > 8e12:
            return None
        back = op in ("linear_bwd", "linear_step")
        names = ("q", "k", "v") + (("do",) if back else ())
        full = {n: (st[n + "_pre"].transpose(0, 1), st[n + "_suf"].transpose(0, 1)) for n in names}
        new = lambda h: (torch.zeros((h, cp[-1], d), dtype=f8, device="cuda"), torch.zeros((h, cs[-1], d), dtype=f8, device="cuda"))  # noqa: E731
        o, dq, dk, dv = new(hq), new(hq), new(hkv), new(hkv)
        s_pre = torch.zeros((len(p), hkv, d, d), dtype=f8, device="cuda")
        s_suf = torch.zeros((len(s), hkv, d, d), dtype=f8, device="cuda")
        for h in range(hkv):
            ld, heads = float(st["log_decay"][h]), slice(h * rep, (h + 1) * rep)
            for g in range(len(p)):
                pre = slice(cp[g], cp[g + 1])
                kp, vp = full["k"][0][h, pre].to(f8), full["v"][0][h, pre].to(f8)
                # the queries in blocks: pieces of the prefix, then each member
                blocks = [(0, a, min(a + 2048, p[g]), None) for a in range(0, p[g], 2048)]
                blocks += [(1, 0, s[m], m) for m in range(g * size, (g + 1) * size) if s[m]]
                for part, a, b, m in blocks:
                    rows = slice(cp[g] + a, cp[g] + b) if part == 0 else slice(cs[m], cs[m + 1])
                    if part == 0:
                        kk, vv, at = kp[:b], vp[:b], torch.arange(a, b, device="cuda")
                    else:
                        kk = torch.cat([kp, full["k"][1][h, rows].to(f8)])
                        vv = torch.cat([vp, full["v"][1][h, rows].to(f8)])
                        at = p[g] + torch.arange(b, device="cuda")
                    gap = at[:, None] - torch.arange(kk.shape[0], device="cuda")[None]
                    dec = torch.where(gap >= 0, torch.exp(ld * gap.clamp_min(0).to(f8)), 0.0) * st["scale"]
                    q = full["q"][part][heads, rows].to(f8)
                    w = torch.matmul(q, kk.t().contiguous()) * dec
                    if op != "linear_bwd":
                        o[part][heads, rows] = torch.matmul(w, vv)
                    if back:
                        do = full["do"][part][heads, rows].to(f8)
                        dw = torch.matmul(do, vv.t().contiguous()) * dec
                        dq[part][heads, rows] = torch.matmul(dw, kk)
                        gk = sum(torch.matmul(dw[r].t(), q[r]) for r in range(rep))
                        gv = sum(torch.matmul(w[r].t(), do[r]) for r in range(rep))
                        n = b if part == 0 else p[g]
                        dk[0][h, cp[g]:cp[g] + n] += gk[:n]
                        dv[0][h, cp[g]:cp[g] + n] += gv[:n]
                        if part:
                            dk[1][h, rows] += gk[n:]
                            dv[1][h, rows] += gv[n:]
                if op == "prefill":
                    age = torch.exp(ld * torch.arange(p[g] - 1, -1, -1, device="cuda").to(f8))
                    s_pre[g, h] = torch.matmul((kp * age[:, None]).t(), vp)
                    for m in range(g * size, (g + 1) * size):
                        own_rows = slice(cs[m], cs[m + 1])
                        kk = torch.cat([kp, full["k"][1][h, own_rows].to(f8)])
                        vv = torch.cat([vp, full["v"][1][h, own_rows].to(f8)])
                        age = torch.exp(ld * torch.arange(kk.shape[0] - 1, -1, -1, device="cuda").to(f8))
                        s_suf[m, h] = torch.matmul((kk * age[:, None]).t(), vv)
        turn = lambda x: tuple(y.transpose(0, 1).contiguous() for y in x)  # noqa: E731
        res = ()
        if op != "linear_bwd":
            res += turn(o) + ((s_pre, s_suf) if op == "prefill" else ())
        if back:
            (a0, a1), (b0, b1), (c0, c1) = turn(dq), turn(dk), turn(dv)
            res += (a0, b0, c0, a1, b1, c1)
        return res
    if op == "policy":
        lp, old = st["logp"].to(f8).cpu(), st["logp_old"].to(f8).cpu()
        ref = None if st["logp_ref"] is None else st["logp_ref"].to(f8).cpu()
        mask = torch.ones(len(lp), dtype=torch.bool) if st["mask"] is None else st["mask"].cpu()
        adv, at, total = st["advantages"].to(f8).cpu(), 0, int(mask.sum())
        grad, sums = torch.zeros_like(lp), [0.0, 0.0, 0.0]
        for m, n in enumerate(s):
            rows = slice(at, at + n)
            at += n
            on = mask[rows]
            if not int(on.sum()):
                continue
            w = 1.0 / (case["n_groups"] * size * int(on.sum())) if case["average"] == "group" else 1.0 / total
            a = float(adv[m])
            r = torch.exp(lp[rows] - old[rows])
            lo, hi = 1.0 - st["clip"][0], 1.0 + st["clip"][1]
            free = r <= hi if a > 0 else (r >= lo) | (a == 0)
            val = torch.where(free, -r * a, -(hi if a > 0 else lo) * a)
            gr = torch.where(free, -r * a, 0.0)
            kl = torch.zeros_like(r)
            if ref is not None:
                x = ref[rows] - lp[rows]
                kl = torch.expm1(x) - x
                gr = gr - st["beta"] * torch.expm1(x)
            grad[rows] = torch.where(on, w * gr, 0.0)
            for i, y in enumerate((val, kl, (~free).to(f8))):
                sums[i] += float((y * on).sum()) * w
        return torch.tensor([sums[0] + st["beta"] * sums[1], *sums], dtype=f8), grad
    tok, t = st["tokens"].cpu(), st["temperature"]
    logp, lse, ent = (torch.zeros(sum(s), dtype=f8, device="cuda") for _ in range(3))
    d_last = torch.zeros(st["logits_last"].shape, dtype=f8, device="cuda") if op == "logprobs_bwd" else None
    d_suf = torch.zeros(st["logits_suf"].shape, dtype=f8, device="cuda") if op == "logprobs_bwd" else None
    at = 0
    for m, n in enumerate(s):
        if not n:
            continue
        x = torch.cat([st["logits_last"][m // size][None], st["logits_suf"][at:at + n - 1]]).to(f8) / t
        lp = torch.log_softmax(x, 1)
        mine = tok[at:at + n].cuda()
        if op == "logprobs":
            logp[at:at + n] = lp.gather(1, mine[:, None])[:, 0]
            lse[at:at + n] = torch.logsumexp(x, 1)
            ent[at:at + n] = -(lp.exp() * lp).sum(1)
        else:
            gr = -lp.exp()
            gr[torch.arange(n, device="cuda"), mine] += 1.0
            gr *= st["dlogp"][at:at + n, None].to(f8) / t
            d_last[m // size] += gr[0]
            d_suf[at:at + n - 1] = gr[1:]
        at += n
    if op == "logprobs":
        return (logp, lse) + ((ent,) if case["entropy"] else ())
    return d_last, d_suf
