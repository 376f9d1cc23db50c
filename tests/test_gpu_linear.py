"""Linear attention over shared prefixes on the GPU against its float64 oracle, element by element.

Bounds (derived, u = half a step of the type: bf16 2^-8, fp32 2^-24): let A be the sum of the absolute values of all
products behind an element (the oracle on absolute inputs). A bf16 call rounds the decayed scores or the state once
(u A in all, each product passes through one of the two), the decayed rows of a state in two parts (2^-16 A, as
(2^-8)^2), and the result (u |ref|). fp32 work adds, for every product, at most N roundings of 2^-23 relative: N = rows
seen in a chain of sums (a chunk's rows, the chunks, the heads) and the power of the decay, 2^x with x rounded
(|x| 2^-24 ln 2 of a value 2^x, below one more rounding each chunk). N = rows / 32 + 2 * 128 + 32 covers every shape
here; where heads or members are summed, their number is added.
"""
import numpy as np
import pytest

from oracle import linear_oracle, linear_steps
from paper_2506_05433_amd.inputs import make_problem
from tests._parity import GRADS, host_view, to_host

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def _bound(ref, mag, dtype, chain, out_u=None):
    u = U[dtype]
    ops = (u + 2.0 ** -16) if dtype == "bf16" else 0.0
    return (u if out_u is None else out_u) * np.abs(ref) * 1.01 + (ops + chain * 2.0 ** -23) * mag + 1e-30


def _close(name, got, ref, mag, dtype, chain, out_u=None):
    got = to_host(got).astype(np.float64)
    assert got.shape == ref.shape and np.isfinite(got).all(), name
    over = np.abs(got - ref) / _bound(ref, mag, dtype, chain, out_u)
    worst = float(over.max()) if over.size else 0.0
    print(f"  {name}: {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0, f"{name}: {worst} of its bound"


def _decays(h_kv, seed):
    rng = np.random.default_rng(seed)
    ld = -np.exp(rng.uniform(np.log(1e-4), np.log(0.7), h_kv)).astype(np.float32)
    ld[0] = {0: 0.0, 1: -3.0, 2: -np.inf}.get(seed % 4, ld[0])  # no decay, a strong one, none of the past
    return ld


CASES = [  # prefixes, group sizes, responses, h_q, h_kv, d, dtype
    (((1,), (1,), (1,)), 1, 1, 64, "fp32"),
    (((0,), (1,), (1,)), 2, 1, 128, "bf16"),
    (((33,), (3,), (0, 31, 65)), 2, 2, 64, "bf16"),
    (((64, 0, 129), (2, 2, 0), (64, 1, 0, 128)), 4, 2, 128, "bf16"),
    (((31, 200), (1, 3), (5, 63, 32, 33)), 5, 1, 128, "fp32"),
    (((0, 0), (2, 1), (96, 0, 17)), 3, 3, 64, "fp32"),
    (((700,), (4,), (300, 2, 0, 129)), 8, 2, 128, "bf16"),
    (((300, 1, 90), (1, 4, 2), (150, 20, 0, 7, 64, 257, 31)), 8, 8, 64, "bf16"),
    (((513,), (0,), ()), 4, 4, 128, "bf16"),          # a prefix alone
    (((150, 40), (2, 0), (260, 300)), 16, 1, 64, "bf16"),
]


def _problem(case):
    lens, hq, hkv, d, dtype = CASES[case]
    prob = make_problem("tiny" if dtype == "fp32" else "single_group", seed=40 + case, lengths=lens, h_q=hq, h_kv=hkv,
                        head_dim=d)
    assert prob.dtype == dtype
    return prob, _decays(hkv, case)


def _chain(prob, heads=1):
    return (prob.total_prefix + prob.total_suffix) / 32 + 288 + heads * prob.h_q / prob.h_kv + len(prob.suffix_lens)


def _oracles(prob, ld, **more):
    t = {k: np.asarray(v, np.float64) for k, v in host_view(prob).items()}
    args = (prob.prefix_lens, prob.group_sizes, prob.suffix_lens, t, prob.scale, ld.astype(np.float64))
    return linear_oracle(*args, **more), linear_oracle(*args, magnitude=True, **more)


def _args(dev):
    return [dev[n] for n in ("q_pre", "k_pre", "v_pre", "q_suf", "k_suf", "v_suf")]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_forward_backward_and_states(case):
    from paper_2506_05433_amd import binding
    prob, ld = _problem(case)
    print(f"[linear] case {case} {CASES[case]} log_decay {ld}", flush=True)
    dev = binding.to_device(prob, "cuda")
    grp = (dev["cu_prefix"], dev["cu_suffix"], dev["group_sizes"])
    dld = torch.from_numpy(ld).cuda()
    ref, mag = _oracles(prob, ld)
    o = binding.linear_fwd(*_args(dev), dld, *grp, prob.scale)
    for n, x in zip(("o_pre", "o_suf"), o):
        _close(n, x, ref[n], mag[n], prob.dtype, _chain(prob))
    g = binding.linear_bwd(*_args(dev), dev["do_pre"], dev["do_suf"], dld, *grp, prob.scale)
    for n, x in zip(GRADS, g):
        _close(n, x, ref[n], mag[n], prob.dtype, _chain(prob, 32))
    # with states: the same outputs up to the finer split of the state updates; states in fp32 (three bf16 parts)
    o2 = binding.linear_fwd(*_args(dev), dld, *grp, prob.scale, states=True)
    for n, x in zip(("o_pre", "o_suf"), o2):
        _close(n, x, ref[n], mag[n], prob.dtype, _chain(prob))
    for n, x in zip(("state_pre", "state_suf"), o2[2:]):
        _close(n, x, ref[n], mag[n], "fp32", _chain(prob) + 2, out_u=0.0)
    torch.cuda.synchronize()


@pytest.mark.parametrize("case", [3, 4, 7])
def test_initial_states_and_reading_in_pieces(case):
    """state_in against the oracle; and a prompt read in two pieces ends in the states of one reading."""
    from paper_2506_05433_amd import binding
    prob, ld = _problem(case)
    print(f"[linear] state_in, case {case}", flush=True)
    dev = binding.to_device(prob, "cuda")
    grp = (dev["cu_prefix"], dev["cu_suffix"], dev["group_sizes"])
    dld = torch.from_numpy(ld).cuda()
    rng = np.random.default_rng(case)
    s_in = rng.standard_normal((len(prob.prefix_lens), prob.h_kv, prob.head_dim, prob.head_dim)).astype(np.float32)
    ref, mag = _oracles(prob, ld, state_in=s_in, grads=False)
    out = binding.linear_fwd(*_args(dev), dld, *grp, prob.scale, state_in=torch.from_numpy(s_in).cuda(), states=True)
    for n, x in zip(("o_pre", "o_suf", "state_pre", "state_suf"), out):
        state = n.startswith("state")
        _close(n, x, ref[n], mag[n], "fp32" if state else prob.dtype, _chain(prob) + 2, out_u=0.0 if state else None)
    # the prefix alone, then the responses as sequences that start from its states
    ng, ns = len(prob.prefix_lens), len(prob.suffix_lens)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    empty = lambda t: t[:0].contiguous()  # noqa: E731
    first = binding.linear_fwd(*_args(dev)[:3], *[empty(t) for t in _args(dev)[3:]], dld, grp[0], i32([0] * (ng + 1)),
                               i32([1] * ng), prob.scale, state_in=torch.from_numpy(s_in).cuda(), states=True)
    torch.testing.assert_close(first[3], first[2], rtol=0, atol=0)  # empty responses: the prefix's states
    group = torch.repeat_interleave(torch.arange(ng), torch.from_numpy(prob.group_sizes)).cuda()
    second = binding.linear_fwd(*_args(dev)[3:], *[empty(t) for t in _args(dev)[:3]], dld, dev["cu_suffix"], i32([0]),
                                i32([0] * ns), prob.scale, state_in=first[2][group].contiguous(), states=True)
    _close("o_suf in pieces", second[0], ref["o_suf"], mag["o_suf"], prob.dtype, _chain(prob) + 2)
    _close("states in pieces", second[2], ref["state_suf"], mag["state_suf"], "fp32", _chain(prob) + 4, out_u=0.0)


def test_gradients_are_differences_of_the_forward():
    """fp32: the directional derivative of sum(o * do) along each input against central differences of the kernel's own
    forward. The loss is linear in each input on its own, so the difference has no truncation error: what is left are
    the forward's roundings, at most (chain + 64) 2^-23 of the sum of magnitudes on either side."""
    from paper_2506_05433_amd import binding
    prob, ld = _problem(4)
    dev = binding.to_device(prob, "cuda")
    grp = (dev["cu_prefix"], dev["cu_suffix"], dev["group_sizes"])
    dld = torch.from_numpy(ld).cuda()
    g = binding.linear_bwd(*_args(dev), dev["do_pre"], dev["do_suf"], dld, *grp, prob.scale)
    _, mag = _oracles(prob, ld, grads=False)
    size = sum(float((mag["o_" + p] * np.abs(prob.as_float("do_" + p))).sum()) for p in ("pre", "suf"))

    def value(args):
        o = binding.linear_fwd(*args, dld, *grp, prob.scale)
        return sum(float((x.double() * dev["do_" + p].double()).sum()) for x, p in zip(o, ("pre", "suf")))

    rng = torch.Generator(device="cuda").manual_seed(1)
    for i, part in enumerate(("pre", "suf")):
        for j in range(3):
            x = _args(dev)[3 * i + j]
            step = x * torch.randint(0, 2, x.shape, generator=rng, device="cuda").mul_(2).sub_(1)  # |x|, random sign
            up, down = _args(dev), _args(dev)
            up[3 * i + j], down[3 * i + j] = x + step, x - step
            diff = (value(up) - value(down)) / 2
            want = float((g[3 * i + j].double() * step.double()).sum())
            assert abs(diff - want) <= (_chain(prob, 32) + 64) * 2.0 ** -23 * 6 * size, (part, j, diff, want)


@pytest.mark.parametrize("n,hq,hkv,d,dtype", [(1, 1, 1, 64, "bf16"), (3, 4, 2, 128, "bf16"), (7, 17, 1, 64, "fp32"),
                                              (5, 40, 8, 128, "fp32"), (130, 8, 4, 128, "bf16"), (300, 6, 2, 64, "bf16")])
def test_single_tokens(n, hq, hkv, d, dtype):
    """Against the recurrence; in place gives the same bits; nothing beyond the n sequences is touched."""
    from paper_2506_05433_amd import binding
    print(f"[linear step] n={n} hq={hq} hkv={hkv} d={d} {dtype}", flush=True)
    rng = torch.Generator(device="cuda").manual_seed(n)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    mk = lambda *s: torch.randn(*s, generator=rng, device="cuda").to(dt)  # noqa: E731
    q, k, v = mk(n, hq, d), mk(n, hkv, d), mk(n, hkv, d)
    whole = torch.randn(n + 1, hkv, d, d, generator=rng, device="cuda")
    state, ld = whole[:n], _decays(hkv, n)
    dld = torch.from_numpy(ld).cuda()
    host = [to_host(t) for t in (q, k, v, state)]
    ref_o, ref_s = linear_steps(*host, ld, 0.25)
    mag_o, mag_s = linear_steps(*[np.abs(t) for t in host], ld, 0.25)
    new = torch.full_like(whole, 7.0)
    o, s = binding.linear_step(q, k, v, state, dld, 0.25, out=(torch.empty_like(q), new[:n]))
    # d products and the state's own two roundings behind an output, one decay and two roundings behind a state
    _close("o", o, ref_o, mag_o, "fp32", d + 8, out_u=U[dtype])
    _close("state", s, ref_s, mag_s, "fp32", 8)
    assert bool((new[n] == 7.0).all())
    o2, s2 = binding.linear_step(q, k, v, state, dld, 0.25)
    assert s2.data_ptr() == state.data_ptr()
    assert torch.equal(o2, o) and torch.equal(s2, s)


def test_steps_continue_a_forward():
    """Reading a prompt and then single tokens gives the rows that the forward over everything gives."""
    from paper_2506_05433_amd import binding
    lens = ((90, 37), (2, 3), (6, 6, 6, 6, 6))
    prob = make_problem("tiny", seed=77, lengths=lens, h_q=4, h_kv=2, head_dim=64)
    ld = _decays(2, 3)
    dev = binding.to_device(prob, "cuda")
    dld = torch.from_numpy(ld).cuda()
    ref, mag = _oracles(prob, ld, grads=False)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    *_, state = binding.linear_fwd(*_args(dev)[:3], *[t[:0] for t in _args(dev)[3:]], dld, dev["cu_prefix"], i32([0] * 6),
                                   dev["group_sizes"], prob.scale, states=True)
    q, k, v = (dev[n + "_suf"].view(5, 6, -1, 64) for n in "qkv")
    for j in range(6):
        o, state = binding.linear_step(q[:, j].contiguous(), k[:, j].contiguous(), v[:, j].contiguous(), state, dld, prob.scale)
        rows = np.arange(5) * 6 + j
        _close(f"token {j}", o, ref["o_suf"][rows], mag["o_suf"][rows], "fp32", _chain(prob) + 8 * (j + 1))


def test_deterministic_and_captured():
    """Two eager calls and three replays of a captured forward, backward and step give the same bits."""
    from paper_2506_05433_amd import binding
    prob, ld = _problem(7)
    print("[linear] capture", flush=True)
    dev = binding.to_device(prob, "cuda")
    grp = (dev["cu_prefix"], dev["cu_suffix"], dev["group_sizes"])
    dld = torch.from_numpy(ld).cuda()
    sizes = (len(prob.prefix_lens), len(prob.suffix_lens), prob.total_prefix, prob.total_suffix, prob.h_q, prob.h_kv, prob.head_dim)
    ws = [torch.empty(binding.linear_workspace_bytes(k, *sizes), device="cuda", dtype=torch.uint8) for k in ("fwd", "bwd")]
    of = tuple(torch.empty_like(x) for x in binding.linear_fwd(*_args(dev), dld, *grp, prob.scale, states=True))
    ob = tuple(torch.empty_like(t) for t in _args(dev))
    q, k, v = (dev[n + "_pre"][:len(prob.suffix_lens)].contiguous() for n in "qkv")
    os_ = (torch.empty_like(q), torch.empty_like(of[3]))

    def step():
        binding.linear_fwd(*_args(dev), dld, *grp, prob.scale, states=True, out=of, workspace=ws[0])
        binding.linear_bwd(*_args(dev), dev["do_pre"], dev["do_suf"], dld, *grp, prob.scale, out=ob, workspace=ws[1])
        binding.linear_step(q, k, v, of[3], dld, prob.scale, out=os_)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    eager = [t.clone() for t in of + ob + os_]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for rep in range(3):
        for t in of + ob + os_:
            t.fill_(float("nan"))
        for w in ws:
            w.fill_(255)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(of + ob + os_, eager)):
            assert torch.equal(a, b), f"replay {rep}, output {i}"


def test_inconsistent_grouping_does_no_work():
    from paper_2506_05433_amd import binding
    prob, ld = _problem(2)
    dev = binding.to_device(prob, "cuda")
    dld = torch.from_numpy(ld).cuda()
    bad = torch.tensor([0, 50, 20, 96], dtype=torch.int32, device="cuda")
    sizes = (1, 3, prob.total_prefix, prob.total_suffix, prob.h_q, prob.h_kv, prob.head_dim)
    for kind in ("fwd", "bwd"):
        ws = torch.empty(binding.linear_workspace_bytes(kind, *sizes), device="cuda", dtype=torch.uint8)
        if kind == "fwd":
            out = tuple(torch.full_like(dev[n], 3.0) for n in ("q_pre", "q_suf"))
            binding.linear_fwd(*_args(dev), dld, dev["cu_prefix"], bad, dev["group_sizes"], prob.scale, out=out, workspace=ws)
        else:
            out = tuple(torch.full_like(t, 3.0) for t in _args(dev))
            binding.linear_bwd(*_args(dev), dev["do_pre"], dev["do_suf"], dld, dev["cu_prefix"], bad, dev["group_sizes"],
                               prob.scale, out=out, workspace=ws)
        with pytest.raises(binding.PgError) as e:
            binding.plan_status(ws)
        assert e.value.status == 1
        assert all(bool((t == 3.0).all()) for t in out)


SHORT = [  # few rows: no states between workgroups (P, members, h_q, h_kv, d, dtype)
    (((64,), (4,), (24, 17, 0, 32)), 2, 2, 64, "fp32"),
    (((60, 0, 68), (2, 1, 3), (10, 33, 7, 0, 5, 40)), 4, 4, 64, "bf16"),
    (((100,), (2,), (20, 40)), 2, 1, 128, "bf16"),
    (((33,), (5,), (1, 31, 32, 33, 2)), 4, 2, 128, "fp32"),
    (((1, 3), (1, 1), (1, 200)), 1, 1, 128, "bf16"),
]


@pytest.mark.parametrize("case", range(len(SHORT)))
def test_few_rows(case):
    """The path without states between workgroups, against the oracle, and its initial states."""
    from paper_2506_05433_amd import binding
    lens, hq, hkv, d, dtype = SHORT[case]
    prob = make_problem("tiny" if dtype == "fp32" else "single_group", seed=70 + case, lengths=lens, h_q=hq, h_kv=hkv, head_dim=d)
    ld = _decays(hkv, case + 3)
    print(f"[linear] few rows {SHORT[case]}", flush=True)
    dev = binding.to_device(prob, "cuda")
    grp = (dev["cu_prefix"], dev["cu_suffix"], dev["group_sizes"])
    dld = torch.from_numpy(ld).cuda()
    ref, mag = _oracles(prob, ld)
    for n, x in zip(("o_pre", "o_suf"), binding.linear_fwd(*_args(dev), dld, *grp, prob.scale)):
        _close(n, x, ref[n], mag[n], prob.dtype, _chain(prob))
    for n, x in zip(GRADS, binding.linear_bwd(*_args(dev), dev["do_pre"], dev["do_suf"], dld, *grp, prob.scale)):
        _close(n, x, ref[n], mag[n], prob.dtype, _chain(prob, 32))
    s_in = np.random.default_rng(case).standard_normal((len(lens[0]), hkv, d, d)).astype(np.float32)
    ref, mag = _oracles(prob, ld, state_in=s_in, grads=False)
    for n, x in zip(("o_pre", "o_suf"), binding.linear_fwd(*_args(dev), dld, *grp, prob.scale, state_in=torch.from_numpy(s_in).cuda())):
        _close(n, x, ref[n], mag[n], prob.dtype, _chain(prob) + 2)


def _repeat_oracle_free(prob, ld, dev, grp, scale):
    """The same problem with every member a group of its own prefix copy, by the library: forward and backward."""
    from paper_2506_05433_amd import binding
    pre, suf, at = [], [], 0
    for p, size in zip(prob.prefix_lens, prob.group_sizes):
        pre += [np.arange(at, at + p)] * int(size)
        at += p
    idx = torch.from_numpy(np.concatenate(pre)).cuda()
    lens = np.repeat(prob.prefix_lens, prob.group_sizes)
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    g2 = (i32(np.concatenate([[0], np.cumsum(lens)])), dev["cu_suffix"], i32(np.ones(len(lens))))
    rep = lambda n: dev[n][idx].contiguous()  # noqa: E731
    args = [rep("q_pre"), rep("k_pre"), rep("v_pre"), dev["q_suf"], dev["k_suf"], dev["v_suf"]]
    o = binding.linear_fwd(*args, ld, *g2, scale)
    share = torch.from_numpy(1.0 / np.repeat(np.repeat(prob.group_sizes, prob.group_sizes), lens)).cuda()
    g = binding.linear_bwd(*args, (rep("do_pre").double() * share[:, None, None]).to(dev["do_pre"].dtype), dev["do_suf"], ld, *g2, scale)
    summed = [torch.zeros(t.shape, dtype=torch.float64, device="cuda").index_add_(0, idx, x.double())
              for t, x in zip((dev["q_pre"], dev["k_pre"], dev["v_pre"]), g[:3])]
    return o, summed, g[3:]


@pytest.mark.parametrize("lens,hq,hkv,d", [
    (((900, 300), (40, 30), tuple(20 + 7 * i for i in range(70))), 16, 8, 64),     # whole members, ordered by length
    (((257, 31, 0), (64, 4, 2), tuple([5, 260, 64, 0, 1, 33, 190] * 10)), 8, 8, 128),
])
def test_whole_members_equal_the_repeated_layout(lens, hq, hkv, d):
    """Enough members that each is one item (longest first, states handed on by the gradient kernel): fp32, against the
    library on the layout in which every member has its own copy of the prefix. Bound: both sides are within chain *
    2^-23 of the magnitudes of the sums, which are at most 60 times the result's norm for these random rows."""
    from paper_2506_05433_amd import binding
    prob = make_problem("tiny", seed=91, lengths=lens, h_q=hq, h_kv=hkv, head_dim=d)
    ld = torch.from_numpy(_decays(hkv, 3)).cuda()
    print(f"[linear] whole members, {len(lens[2])} of them", flush=True)
    dev = binding.to_device(prob, "cuda")
    grp = (dev["cu_prefix"], dev["cu_suffix"], dev["group_sizes"])
    o = binding.linear_fwd(*_args(dev), ld, *grp, prob.scale)
    g = binding.linear_bwd(*_args(dev), dev["do_pre"], dev["do_suf"], ld, *grp, prob.scale)
    ro, pre, suf = _repeat_oracle_free(prob, ld, dev, grp, prob.scale)
    tol = 2 * 60 * 300 * 2.0 ** -23
    for name, a, b in [("o_suf", o[1], ro[1])] + list(zip(GRADS, g, list(pre) + list(suf))):
        err = float((a.double() - b.double()).norm() / b.double().norm())
        print(f"  {name}: {err:.2e}", flush=True)
        assert err <= tol, (name, err)


def test_both_planners_agree(monkeypatch):
    """The items of the planner for large grouping arrays, forced, give the same bits."""
    from paper_2506_05433_amd import binding
    prob = make_problem("single_group", seed=92, lengths=((300, 90), (40, 31), tuple(10 + 3 * i for i in range(71))), h_q=16,
                        h_kv=8, head_dim=64)
    ld = torch.from_numpy(_decays(8, 3)).cuda()
    dev = binding.to_device(prob, "cuda")
    grp = (dev["cu_prefix"], dev["cu_suffix"], dev["group_sizes"])

    def both():
        o = binding.linear_fwd(*_args(dev), ld, *grp, prob.scale, states=True)
        return o + binding.linear_bwd(*_args(dev), dev["do_pre"], dev["do_suf"], ld, *grp, prob.scale)

    one = both()
    monkeypatch.setenv("PG_PLAN_MULTI", "1")
    for a, b in zip(one, both()):
        assert torch.equal(a, b)


def test_a_stray_value_stays_in_its_member():
    """NaN in one member's rows reaches neither the prefix's and the other members' outputs nor, without it in the upstream
    gradient, their own rows' gradients of q."""
    from paper_2506_05433_amd import binding
    prob = make_problem("single_group", seed=93, lengths=((70, 10), (3, 1), (40, 33, 70, 9)), h_q=4, h_kv=2, head_dim=128)
    ld = torch.from_numpy(_decays(2, 3)).cuda()
    dev = binding.to_device(prob, "cuda")
    grp = (dev["cu_prefix"], dev["cu_suffix"], dev["group_sizes"])
    clean = binding.linear_fwd(*_args(dev), ld, *grp, prob.scale)
    dev["v_suf"][45] = float("nan")  # the second member
    o = binding.linear_fwd(*_args(dev), ld, *grp, prob.scale)
    keep = torch.cat([torch.arange(0, 40), torch.arange(73, prob.total_suffix)]).cuda()
    assert torch.equal(o[0], clean[0]) and torch.equal(o[1][keep], clean[1][keep])
    assert bool(torch.isnan(o[1][45:73]).any(-1).all())
