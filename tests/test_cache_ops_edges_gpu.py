"""Edges of the operators on bounded and shared caches: scratch anywhere in memory, infinite values, loose bounds, odd
probabilities.  Statements in 64 bits and tolerances are those of test_cache_ops_gpu."""
import numpy as np
import pytest
import torch

import cache_reference as R
from paper_2407_14057_b200 import binding as B
from paper_2407_14057_b200 import build
from test_cache_ops_gpu import (BF16, CALLS, F32, HEADS, IDS, check_step, cu, f64, gen, half_step, mass_case, prefix_case,
                                prefix_expected, randn, run_prefix, step_case, step_expected, verify_case, weight_error)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    B.lib()


# ------------------------------------------------------------------------------------------- scratch
@pytest.fixture
def late_scratch(monkeypatch):
    """Makes every call's scratch a slice of just the size asked for, 4 bytes behind a 16-byte boundary, between guards."""
    made = []

    def scratch(n, dtype):
        n = max(int(n), 1)
        buf = torch.full((n + 65,), -7, dtype=dtype, device="cuda")
        assert buf.data_ptr() % 16 == 0
        buf[1:1 + n] = float("nan") if dtype.is_floating_point else 0
        made.append((buf, n))
        return buf[1:1 + n]

    monkeypatch.setattr(B, "_scratch", scratch)
    yield made
    assert made
    for buf, n in made:
        assert buf[0].item() == -7 and torch.all(buf[1 + n:] == -7)


@pytest.mark.parametrize("name", [n for n in CALLS if n != "verify"])
def test_scratch_may_start_anywhere(name, late_scratch, monkeypatch):
    inputs, call = CALLS[name]
    got = [t.clone() for t in call(inputs(80))]
    monkeypatch.undo()
    want = call(inputs(80))
    B.lazy_device_status()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# (sequences, heads, budget): a part's logits have no room in shared memory, because many CTAs share an SM (over 8 KiB, the
# first ones) or at all (over 40 KiB); odd groups, two blocks of columns, parts cut by a cluster
STEP_LOGITS = [(40, (32, 8, 128, BF16), 700), (40, (24, 8, 64, BF16), 650), (300, (16, 1, 32, BF16), 330), (75, (20, 4, 96, BF16), 560),
               (15, (8, 1, 64, BF16), 10500), (20, (32, 8, 64, BF16), 1500)]


@pytest.mark.parametrize("n_seqs,heads,budget", STEP_LOGITS, ids=[f"{s}x{h[0]}on{h[1]}x{h[2]}-{b}" for s, h, b in STEP_LOGITS])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_step_keeps_logits_in_the_scratch(n_seqs, heads, budget, in_place, late_scratch):
    H, Hkv, dh, dtype = heads
    lens = [budget if s % 3 else (0, 1, budget - 1, budget // 2)[s // 3 % 4] for s in range(n_seqs)]
    c, new = step_case(81 + n_seqs, lens, budget, H, Hkv, dh, dtype)
    check_step(c, new, H, budget, budget // 8, in_place=in_place)


# ------------------------------------------------------------------------------------------- infinite values
def with_infinities(v, g):
    """Columns 1 and 2: every second row +inf, every second -inf; 3: one row +inf; 5: infinities of both signs."""
    n, some = v.shape[0], torch.rand((2, v.shape[0]), generator=g) < 0.5
    v[some[0], 1], v[some[1], 2] = float("inf"), -float("inf")
    if n > 2:
        v[n // 3, 3] = float("inf")
        v[0, 5], v[n // 2, 5] = float("inf"), -float("inf")


def same_with_infinities(got, want, tol):
    odd = ~np.isfinite(want)
    assert odd.any() and not odd.all()
    assert np.array_equal(got[odd], want[odd], equal_nan=True)
    assert np.all(np.abs(got[~odd] - want[~odd]) <= tol[~odd])


@pytest.mark.parametrize("heads", HEADS, ids=IDS)
@pytest.mark.parametrize("n_pre,rows,own", [(0, [1], [20]), (0, [3, 5], [200, 300]), (70, [2, 1], [3, 90]), (300, [1] * 40, [4] * 40),
                                            (130, [2, 2], [2, 2]), (0, [1] * 30, [300] * 30)])
def test_attention_prefix_infinite_values(heads, n_pre, rows, own):
    """An infinite value gives every row that sees it the infinity that the formula has, wherever its key lies."""
    H, Hkv, dh, dtype = heads
    d = prefix_case(82, n_pre, rows, own, H, Hkv, dh, dtype)
    for name, lines in (("v_pre", n_pre), ("v", d["v"].shape[0])):
        for g in range(Hkv):
            if lines:
                with_infinities(d[name][:, g * dh:(g + 1) * dh], gen(83 + g))
    with np.errstate(invalid="ignore"):
        want, tol = prefix_expected(d, rows, own, H, Hkv, dh)
    got = f64(run_prefix(d, rows, own, H, Hkv, dh)).reshape(want.shape)
    B.lazy_device_status()
    same_with_infinities(got, want, tol)


@pytest.mark.parametrize("heads", HEADS + [(16, 1, 64, BF16)], ids=IDS + ["16on1x64"])
@pytest.mark.parametrize("lens,budget", [([1, 2], 2), ([40, 39], 40), ([700], 700)])
def test_evict_step_infinite_values(heads, lens, budget):
    H, Hkv, dh, dtype = heads
    c, new = step_case(84, lens, budget, H, Hkv, dh, dtype)
    for s, n in enumerate(lens):
        for g in range(Hkv):
            with_infinities(c["vc"][s, :n, g], gen(85 + g))
    new["v_new"].view(len(lens), Hkv, dh)[:, :, 7] = float("inf")
    with np.errstate(invalid="ignore"):
        _, _, o, amount, _, _, e = step_expected(c, new, H, budget, 1 if budget > 1 else 0)
    dev = {k: v.cuda() for k, v in {**c, **new}.items()}
    got, _, _ = B.lazy_k_evict_step(**dev, n_heads=H, budget=budget, n_recent=1)
    B.lazy_device_status()
    with np.errstate(invalid="ignore"):
        same_with_infinities(f64(got).reshape(o.shape), o, e * amount + half_step(dtype) * np.abs(o) * (1 + e) + 1e-30)


# ------------------------------------------------------------------------------------------- verification
@pytest.mark.parametrize("V", [299, 300, 4096])
def test_verify_negative_and_nan_entries_count_as_zero(V):
    """In both distributions, in the acceptance and in what is drawn from: no id is given weight by a negative one."""
    g = gen(86)
    drafts = [1] * 64
    d = verify_case(87, drafts, V, near=2.0)
    p, q = d["p"], d["q"]
    odd = torch.tensor([-1.0, -0.25, float("nan"), -float("inf"), -1e-6])
    q[:] = torch.where(torch.rand(q.shape, generator=g) < 0.3, odd[torch.randint(0, 5, q.shape, generator=g)], q)
    p[:] = torch.where(torch.rand(p.shape, generator=g) < 0.5, odd[torch.randint(0, 5, p.shape, generator=g)], p)
    p[0::2][torch.rand(q.shape, generator=g) < 0.3] = 0.0
    acc, tokens = B.lazy_k_verify(p.cuda(), d["draft"].cuda(), cu(drafts), 1, d["u_accept"].cuda(), d["u_sample"].cuda(), q=q.cuda())
    B.lazy_device_status()
    acc, tokens = acc.cpu().tolist(), tokens.cpu().tolist()
    zeroed = lambda t: np.where(t.numpy() > 0, t.numpy(), 0.0)  # noqa: E731
    for s in range(64):
        want, token = R.verify(zeroed(p[2 * s:2 * s + 2]), zeroed(q[s:s + 1]), d["draft"][s:s + 1].numpy(),
                               d["u_accept"][s:s + 1].numpy(), d["u_sample"][s].item())
        assert acc[s] == want and tokens[s][want] == token, s
    assert 0 < sum(acc) < 64


@pytest.mark.parametrize("V,first,second", [(3, 0, 1), (4, 0, 1), (4096, 5, 3001), (4095, 1000, 1001)])
def test_verify_subtracts_in_64_bits(V, first, second):
    """Weights 1 and 1 - 2^-30: half of their total lies just below the first one; in 32 bits both would be 1."""
    p, q = torch.zeros((2, V)), torch.zeros((1, V))
    p[0, first] = p[0, second] = 1.0
    q[0, second] = 2.0 ** -30
    q[0, V - 1] = 1.0                       # the draft, which the target never takes
    half = torch.tensor([0.5]).cuda()
    acc, tokens = B.lazy_k_verify(p.cuda(), torch.tensor([V - 1], dtype=torch.int32).cuda(), cu([1]), 1, half, half, q=q.cuda())
    assert acc.item() == 0 and tokens[0].tolist() == [first, -1]
    assert R.verify(p.numpy(), q.numpy(), [V - 1], [0.5], 0.5) == (0, first)


@pytest.mark.parametrize("V", [3, 300, 4096, 32000])
@pytest.mark.parametrize("with_q", [True, False])
def test_verify_infinite_entries_count_as_the_largest_number(V, with_q):
    """Behind the last draft, after a rejection, and where the draft model's own entry is infinite."""
    g = gen(94)
    big = torch.finfo(F32).max
    drafts, at = [0, 1, 1], torch.randint(0, V - 1, (3,), generator=g)
    p, q = torch.rand((5, V), generator=g), torch.rand((2, V), generator=g)
    p[0, at[0]] = p[1, at[1]] = float("inf")
    p[1::2, V - 1] = 0.0                     # both drafts are rejected
    q[:, V - 1] = 1.0
    q[1, at[2]] = float("inf")
    half = torch.tensor([0.5] * 3).cuda()
    acc, tokens = B.lazy_k_verify(p.cuda(), torch.tensor([V - 1] * 2, dtype=torch.int32).cuda(), cu(drafts), 1, half[:2], half,
                                  q=q.cuda() if with_q else None)
    B.lazy_device_status()
    assert acc.tolist() == [0, 0, 0] and tokens[:, 1].tolist() == [-1, -1, -1]
    assert tokens[:2, 0].tolist() == at[:2].tolist()
    want = R.verify(p[3:].clamp(max=big).numpy(), q[1:].clamp(max=big).numpy() if with_q else None, [V - 1], [0.5], 0.5)
    assert tokens[2, 0].item() == want[1] and (not with_q or want[1] != at[2])


# ------------------------------------------------------------------------------------------- loose bounds
@pytest.mark.parametrize("heads", HEADS, ids=IDS)
@pytest.mark.parametrize("lens,window", [([257, 31], 0), ([257, 31], 20), ([5], 1)])
def test_attention_mass_takes_any_bound(heads, lens, window):
    """max_len is a bound, not a length: the largest number is one, and no call after it finds an error left behind."""
    H, Hkv, dh, dtype = heads
    q, k, dq, dk = mass_case(88, lens, H, Hkv, dh, dtype, fused=True)
    n = sum(lens)
    want = R.attention_mass(f64(q).reshape(n, H, dh), f64(k).reshape(n, Hkv, dh), lens, H, Hkv, dh, window)
    e = weight_error(f64(q).reshape(n, H, dh), f64(k).reshape(n, Hkv, dh), dh)
    for bound in (2 ** 31 - 1, 2 ** 31 - 100, 10 ** 7):
        got = B.lazy_k_attention_mass(dq, dk, cu(lens), bound, H, Hkv, dh, window)
        assert np.all(np.abs(f64(got) - want) <= e * want + 1e-30), bound
    c, new = step_case(89, [3], 5, 4, 2, 64, F32)
    check_step(c, new, 4, 5, 1)


# ------------------------------------------------------------------------------------------- one scratch, call after call
@pytest.mark.parametrize("name", [n for n in CALLS if n.startswith(("prefix", "mass"))])
def test_a_captured_call_uses_nothing_that_its_scratch_held(name, monkeypatch):
    """A call in a graph whose scratch is spoilt before every replay, on inputs that change between them."""
    inputs, call = CALLS[name]
    made = []
    make = B._scratch
    monkeypatch.setattr(B, "_scratch", lambda n, dtype: made.append(make(n, dtype)) or made[-1])
    x = inputs(90)
    want = {seed: [t.clone() for t in call(inputs(seed))] for seed in (91, 92)}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = call(x)
    for i in range(40):
        seed = 91 + i % 2
        for key, t in inputs(seed).items():
            x[key].copy_(t)
        made[-1].fill_(float("nan"))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, want[seed])), i
    B.lazy_device_status()


@pytest.mark.parametrize("heads", [HEADS[1], HEADS[7]], ids=[IDS[1], IDS[7]])
def test_one_scratch_for_a_batch_that_shrinks(heads):
    """Scratch sized once for the largest batch serves every smaller one, down to a single request."""
    H, Hkv, dh, dtype = heads
    d = prefix_case(95, 1500, [1] * 70, [9] * 70, H, Hkv, dh, dtype)
    dev = {k: v.cuda() for k, v in d.items()}
    scratch = B.lazy_k_attention_prefix_scratch(70, 70, 1, 1500, 9, H, Hkv, dh)
    for n in (70, 65, 64, 33, 32, 31, 16, 5, 1):
        args = (dev["q"][:n], cu([1] * n), 1, dev["k_pre"], dev["v_pre"], dev["k"], dev["v"], dev["kv_idx"][:9 * n], cu([9] * n), 9,
                H, Hkv, dh)
        got = B.lazy_k_attention_prefix(*args, scratch=scratch)
        assert torch.equal(got, B.lazy_k_attention_prefix(*args)), n
    lens = [5000, 4000, 30]
    _, _, q, k = mass_case(96, lens, H, Hkv, dh, dtype, fused=False)
    scratch = B.lazy_k_attention_mass_scratch(3, sum(lens), max(lens), H, Hkv)
    for part, window in ((lens, 0), (lens, 40), (lens[:1], 1), (lens[:2], 33), ([2000], 0)):
        n = sum(part)
        got = B.lazy_k_attention_mass(q[:n], k[:n], cu(part), max(part), H, Hkv, dh, window, scratch=scratch)
        assert torch.equal(got, B.lazy_k_attention_mass(q[:n], k[:n], cu(part), max(part), H, Hkv, dh, window))
    B.lazy_device_status()


# ------------------------------------------------------------------------------------------- wide groups, rows of nobody
WIDE = [(24, 1, 64, BF16), (100, 1, 64, BF16), (160, 1, 32, BF16), (34, 2, 128, BF16), (20, 1, 64, F32), (130, 1, 32, F32)]


@pytest.mark.parametrize("heads", WIDE, ids=[f"{h}on{k}x{d}{'' if t == BF16 else 'f32'}" for h, k, d, t in WIDE])
def test_wide_groups(heads):
    """More query heads to a key/value head than a block of columns, or than a tile of lanes, holds."""
    H, Hkv, dh, dtype = heads
    for lens, window in (([70, 1, 130], 0), ([200], 3)):
        n = sum(lens)
        q, k, dq, dk = mass_case(97, lens, H, Hkv, dh, dtype, fused=True)
        got = B.lazy_k_attention_mass(dq, dk, cu(lens), max(lens), H, Hkv, dh, window)
        qn, kn = f64(q).reshape(n, H, dh), f64(k).reshape(n, Hkv, dh)
        want = R.attention_mass(qn, kn, lens, H, Hkv, dh, window)
        assert np.all(np.abs(f64(got) - want) <= weight_error(qn, kn, dh) * want + 1e-30)
    c, new = step_case(98, [90, 3, 0], 90, H, Hkv, dh, dtype)
    check_step(c, new, H, 90, 10)
    for n_pre, rows, own in ((130, [1, 3], [40, 3]), (0, [2, 1], [70, 1])):
        d = prefix_case(99, n_pre, rows, own, H, Hkv, dh, dtype)
        want, tol = prefix_expected(d, rows, own, H, Hkv, dh)
        got = run_prefix(d, rows, own, H, Hkv, dh)
        assert np.all(np.abs(f64(got).reshape(want.shape) - want) <= tol)
    B.lazy_device_status()


@pytest.mark.parametrize("heads", [HEADS[1], HEADS[6], HEADS[7]], ids=[IDS[1], IDS[6], IDS[7]])
def test_rows_of_no_sequence(heads):
    """Rows before the first sequence's and behind the last one's: no weight, no part in an eviction; behind a prefix they are
    reported and see it alone."""
    H, Hkv, dh, dtype = heads
    lens, n = [40, 70], 120
    q, k, dq, dk = mass_case(100, [n], H, Hkv, dh, dtype, fused=False)
    dq[:3], dk[:3], dq[113:], dk[113:] = (float("nan"),) * 4
    table = torch.tensor([3, 43, 113], dtype=torch.int32).cuda()
    out = torch.full((Hkv, n), -7.0, device="cuda")
    B.lazy_k_attention_mass(dq, dk, table, 70, H, Hkv, dh, out=out)
    assert torch.all(out[:, :3] == -7) and torch.all(out[:, 113:] == -7)
    qn, kn = f64(q).reshape(n, H, dh)[3:113], f64(k).reshape(n, Hkv, dh)[3:113]
    want = R.attention_mass(qn, kn, lens, H, Hkv, dh, 0)
    assert np.all(np.abs(f64(out)[:, 3:113] - want) <= weight_error(qn, kn, dh) * want)
    cache = dict(kc=torch.zeros((2, 30, Hkv, dh), dtype=dtype, device="cuda"), vc=torch.zeros((2, 30, Hkv, dh), dtype=dtype, device="cuda"),
                 cmass=torch.zeros((2, Hkv, 30), device="cuda"), cpos=torch.zeros((2, Hkv, 30), dtype=torch.int32, device="cuda"),
                 clen=torch.zeros((2, Hkv), dtype=torch.int32, device="cuda"))
    out[:, :3] = out[:, 113:] = float("inf")
    B.lazy_k_evict(dk, dk, torch.arange(n, dtype=torch.int32).cuda(), out, table, 70, 30, 4, **cache)
    B.lazy_device_status()
    for s, a, ln in ((0, 3, 40), (1, 43, 70)):
        for h in range(Hkv):
            assert (cache["cpos"][s, h].cpu() - a).tolist() == R.kept_rows(out[h, a:a + ln].cpu().numpy(), ln, 30, 4)
    rows, own, n_pre = [2, 3], [40, 90], 75
    d = prefix_case(101, n_pre, [1] + rows + [2], [0] + own + [0], H, Hkv, dh, dtype)
    want, tol = prefix_expected(d, [1] + rows + [1, 1], [0] + own + [0, 0], H, Hkv, dh)
    dev = {name: t.cuda() for name, t in d.items()}
    got = B.lazy_k_attention_prefix(dev["q"], torch.tensor([1, 3, 6], dtype=torch.int32).cuda(), 3, dev["k_pre"], dev["v_pre"], dev["k"],
                                    dev["v"], dev["kv_idx"], cu(own), 90, H, Hkv, dh)
    with pytest.raises(B.LazyError, match="BADARG"):
        B.lazy_device_status()
    assert np.all(np.abs(f64(got).reshape(want.shape) - want) <= tol)


# ------------------------------------------------------------------------------------------- in place or not, each for itself
@pytest.mark.parametrize("heads", [HEADS[1], HEADS[7]], ids=[IDS[1], IDS[7]])
@pytest.mark.parametrize("apart", [(), ("mass",), ("pos",), ("len",), ("mass", "pos"), ("mass", "len"), ("pos", "len")])
def test_evict_step_some_state_in_place(heads, apart):
    """Masses, positions and lengths go to arrays of their own or stay, independently of one another."""
    H, Hkv, dh, dtype = heads
    lens, budget = [90, 41, 0], 90
    c, new = step_case(102, lens, budget, H, Hkv, dh, dtype)
    both = [{k: v.cuda() for k, v in {**c, **new}.items()} for _ in range(2)]
    want = B.lazy_k_evict_step(**both[0], n_heads=H, budget=budget, n_recent=5)
    outs = {f"{x}_out": both[1]["c" + x].clone() for x in apart}
    got = B.lazy_k_evict_step(**both[1], **outs, n_heads=H, budget=budget, n_recent=5)
    B.lazy_device_status()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    as_bytes = lambda t: t.contiguous().view(torch.uint8)  # noqa: E731
    for x in ("mass", "pos", "len"):
        after = outs[f"{x}_out"] if x in apart else both[1]["c" + x]
        assert torch.equal(as_bytes(after), as_bytes(both[0]["c" + x])), x
        if x in apart:
            assert torch.equal(as_bytes(both[1]["c" + x].cpu()), as_bytes(c["c" + x])), x
