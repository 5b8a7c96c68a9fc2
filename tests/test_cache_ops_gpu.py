"""Operators on bounded and shared caches against their statements in 64 bits, through the public binding.

Tolerances.  A logit is a dot product of dh products accumulated in 32 bits: its error is at most (dh + 4) 2^-24 S in
natural-log units with S = max sum_c |q_c k_c| / sqrt(dh), doubled for a tensor core's truncating adder; a weight takes
that error twice (numerator and normaliser), plus 2^-19 for the exponentials and the sums of up to 2^10 positive
terms.  So relative to itself a weight, or a sum of weights, is off by at most E = 4 (dh + 4) 2^-23 S / 2 + 2^-19, an
output by E sum_j w_j |v_j| plus half a step of its own type.
"""
import numpy as np
import pytest
import torch

import cache_reference as R
from helpers import to_np
from paper_2407_14057_b200 import binding as B
from paper_2407_14057_b200 import build

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
# (n_heads, n_kv_heads, head_dim, dtype): tensor-core widths, grouped and not, groups that do not divide a tile, other
# widths, fp32
HEADS = [(4, 4, 128, BF16), (8, 2, 128, BF16), (8, 1, 64, BF16), (6, 2, 64, BF16), (5, 1, 128, BF16), (2, 2, 96, BF16),
         (4, 2, 256, BF16), (4, 4, 64, F32), (6, 2, 32, F32), (8, 2, 32, BF16), (12, 2, 96, BF16), (4, 1, 160, F32)]
IDS = [f"{h}on{k}x{d}{'' if t == BF16 else 'f32'}" for h, k, d, t in HEADS]


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    B.lib()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dtype):
    return torch.randn(shape, generator=g).to(dtype)


def cu(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32).cuda()


def f64(t):
    return to_np(t).astype(np.float64)


def weight_error(q, k, dh):
    """E of the module's comment; q [.., dh], k [.., dh]: S is bounded through the largest norms."""
    s = np.sqrt((q ** 2).sum(-1).max() * (k ** 2).sum(-1).max()) * dh ** -0.5
    return 2 * (dh + 4) * 2.0 ** -23 * s + 2.0 ** -19


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------------------------------- weights of prompts
def mass_case(seed, lens, H, Hkv, dh, dtype, fused):
    g, n = gen(seed), sum(lens)
    q = randn(g, n, H * dh, dtype=dtype)
    k = randn(g, n, Hkv * dh, dtype=dtype)
    if fused:   # parts of one row, with something between and behind them
        row = torch.full((n, (H + Hkv) * dh + 64), float("nan"), dtype=dtype)
        row[:, 32:32 + H * dh] = q
        row[:, 32 + H * dh:32 + (H + Hkv) * dh] = k
        row = row.cuda()
        return q, k, row[:, 32:32 + H * dh], row[:, 32 + H * dh:32 + (H + Hkv) * dh]
    return q, k, q.cuda(), k.cuda()


@pytest.mark.parametrize("heads", HEADS, ids=IDS)
@pytest.mark.parametrize("lens,window", [([1], 0), ([2, 1, 3], 0), ([63, 64, 65], 0), ([130], 1), ([129, 1, 300], 7),
                                         ([257, 31], 64), ([200, 0, 5], 1000), ([385], 150)])
def test_attention_mass(heads, lens, window):
    H, Hkv, dh, dtype = heads
    q, k, dq, dk = mass_case(7 * len(lens) + lens[0] + window, lens, H, Hkv, dh, dtype, fused=window != 1)
    n = sum(lens)
    out = torch.full((Hkv, n + 1), -7.0, device="cuda")   # a poisoned column behind the last head's rows
    flat = out.view(-1)[:Hkv * n].view(Hkv, n)
    B.lazy_k_attention_mass(dq, dk, cu(lens), max(lens), H, Hkv, dh, window, out=flat)
    B.lazy_device_status()
    assert torch.all(out.view(-1)[Hkv * n:] == -7.0)
    qn, kn = f64(q).reshape(n, H, dh), f64(k).reshape(n, Hkv, dh)
    want = R.attention_mass(qn, kn, lens, H, Hkv, dh, window)
    err = np.abs(f64(flat) - want)
    assert np.all(err <= weight_error(qn, kn, dh) * want + 1e-30), (err / np.maximum(want, 1e-30)).max()
    again = B.lazy_k_attention_mass(dq, dk, cu(lens), max(lens), H, Hkv, dh, window)
    assert torch.equal(again, flat)


def test_attention_mass_of_one_row_is_the_score_times_heads():
    H, dh, lens = 4, 128, [300, 65]
    _, _, q, k = mass_case(3, lens, H, H, dh, BF16, fused=False)
    c = cu(lens)
    mass = B.lazy_k_attention_mass(q, k, c, 300, H, H, dh, 1)
    score = B.lazy_k_score(q, H * dh, k, H * dh, c, sum(lens), H, dh)
    assert torch.max(torch.abs(mass.mean(0) - score)).item() < 1e-5


def test_attention_mass_neighbours_do_not_leak():
    """NaN and infinities in another sequence change nothing in this one; large logits stay finite."""
    H, Hkv, dh, lens = 4, 2, 128, [70, 90, 130]
    _, _, q, k = mass_case(4, lens, H, Hkv, dh, BF16, fused=False)
    q[70:160] *= 30.0   # logits of several hundred
    want = B.lazy_k_attention_mass(q, k, cu(lens), 130, H, Hkv, dh)
    assert torch.isfinite(want).all()
    assert abs(want[:, 70:160].sum().item() / (90 * H) - 1.0) < 1e-5
    q[:70], k[:70] = float("nan"), float("inf")
    k[160:] = float("nan")
    got = B.lazy_k_attention_mass(q, k, cu(lens), 130, H, Hkv, dh)
    assert torch.equal(got[:, 70:160], want[:, 70:160])
    B.lazy_device_status()


def test_attention_mass_reports_a_bad_length_table():
    H, dh = 4, 128
    _, _, q, k = mass_case(5, [100], H, H, dh, BF16, fused=False)
    for table in ([0, 101], [0, 50, 40, 100], [-1, 100]):
        c = torch.tensor(table, dtype=torch.int32, device="cuda")
        B.lazy_k_attention_mass(q, k, c, 100, H, H, dh)
        with pytest.raises(B.LazyError):
            B.lazy_device_status()
    B.lazy_k_attention_mass(q, k, cu([100]), 99, H, H, dh)   # longer than declared
    with pytest.raises(B.LazyError):
        B.lazy_device_status()


def test_attention_mass_long_prompt_sums_to_its_rows():
    """Every row's weights add up to one, so a head group's masses add up to rows x heads; the first rows by the formula."""
    H, Hkv, dh, n = 8, 2, 128, 5000
    q, k, dq, dk = mass_case(6, [n], H, Hkv, dh, BF16, fused=False)
    got = f64(B.lazy_k_attention_mass(dq, dk, cu([n]), n, H, Hkv, dh))
    assert np.all(np.abs(got.sum(1) / (n * H / Hkv) - 1.0) < 1e-5)
    got = f64(B.lazy_k_attention_mass(dq, dk, cu([n]), n, H, Hkv, dh, 20))
    qn, kn = f64(q).reshape(n, H, dh), f64(k).reshape(n, Hkv, dh)
    want = R.attention_mass(qn, kn, [n], H, Hkv, dh, 20)
    assert np.all(np.abs(got - want) <= weight_error(qn, kn, dh) * want)


@pytest.mark.parametrize("heads", [(8, 8, 64), (32, 8, 128), (24, 8, 64)], ids=["8on8x64", "32on8x128", "24on8x64"])
@pytest.mark.parametrize("lens,window", [([5000], 33), ([300, 4500, 1], 100), ([4700], 1)])
def test_attention_mass_window_over_long_prompts(heads, lens, window):
    """Few rows over many keys: the form that cuts the keys into ranges."""
    H, Hkv, dh = heads
    q, k, dq, dk = mass_case(8, lens, H, Hkv, dh, BF16, fused=True)
    got = f64(B.lazy_k_attention_mass(dq, dk, cu(lens), max(lens), H, Hkv, dh, window))
    B.lazy_device_status()
    qn, kn = f64(q).reshape(-1, H, dh), f64(k).reshape(-1, Hkv, dh)
    want = R.attention_mass(qn, kn, lens, H, Hkv, dh, window)
    assert np.all(np.abs(got - want) <= weight_error(qn, kn, dh) * want)


@pytest.mark.parametrize("heads", [(8, 8, 64), (32, 8, 128), (10, 2, 128), (24, 24, 64)],
                         ids=["8on8x64", "32on8x128", "10on2x128", "24on24x64"])
@pytest.mark.parametrize("lens,window", [([4900], 0), ([2500, 1, 2700], 0), ([129, 4097, 640], 3000)])
def test_attention_mass_many_tiles(heads, lens, window):
    """Full prompts with more tiles than the machine takes at once, odd numbers of them among them."""
    H, Hkv, dh = heads
    q, k, dq, dk = mass_case(9, lens, H, Hkv, dh, BF16, fused=True)
    got = B.lazy_k_attention_mass(dq, dk, cu(lens), max(lens), H, Hkv, dh, window).double()
    B.lazy_device_status()
    want, a = torch.zeros_like(got), 0
    for n in lens:
        first = max(n - window, 0) if window else 0
        hide = torch.ones((n - first, n), dtype=torch.bool, device="cuda").triu(first + 1)
        for h in range(H):
            g = h // (H // Hkv)
            x = dq[a + first:a + n, h * dh:(h + 1) * dh].double() @ dk[a:a + n, g * dh:(g + 1) * dh].double().t() * dh ** -0.5
            want[g, a:a + n] += torch.softmax(x.masked_fill(hide, -float("inf")), -1).sum(0)
        a += n
    e = weight_error(f64(q).reshape(-1, H, dh), f64(k).reshape(-1, Hkv, dh), dh)
    assert torch.all((got - want).abs() <= (e + 2.0 ** -18) * want)   # and up to 2^14 positive terms, in chains of 2^8


# ------------------------------------------------------------------------------------------- compaction
def new_cache(n_seqs, cap, Hkv, dh, dtype):
    return dict(kc=torch.full((n_seqs, cap, Hkv, dh), 99.0, dtype=dtype, device="cuda"),
                vc=torch.full((n_seqs, cap, Hkv, dh), 98.0, dtype=dtype, device="cuda"),
                cmass=torch.full((n_seqs, Hkv, cap), -5.0, device="cuda"),
                cpos=torch.full((n_seqs, Hkv, cap), -6, dtype=torch.int32, device="cuda"),
                clen=torch.full((n_seqs, Hkv), -7, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("heads", [HEADS[1], HEADS[5], HEADS[8]], ids=[IDS[1], IDS[5], IDS[8]])
@pytest.mark.parametrize("lens,budget,recent", [([1], 1, 0), ([5, 0, 40], 8, 3), ([64, 8, 9], 8, 8), ([3000, 1500], 700, 0),
                                                ([2049], 2048, 100), ([70], 1, 1), ([1025, 33], 300, 299),
                                                ([200, 199, 201, 300, 192], 60, 8)])
@pytest.mark.parametrize("weights", ["distinct", "ties", "odd"])
def test_evict(heads, lens, budget, recent, weights):
    _, Hkv, dh, dtype = heads
    g, n, S = gen(sum(lens) + budget), sum(lens), len(lens)
    k, v = randn(g, n, Hkv * dh, dtype=dtype), randn(g, n, Hkv * dh, dtype=dtype)
    mass = torch.exp(2 * torch.randn((Hkv, n), generator=g))
    if weights == "ties":
        mass = torch.randint(0, 4, (Hkv, n), generator=g).float()
    elif weights == "odd":
        odd = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, -1.0, 1e-45, 3.0])
        mass = torch.where(torch.rand((Hkv, n), generator=g) < 0.5, odd[torch.randint(0, 8, (Hkv, n), generator=g)], mass)
    pos = torch.randint(0, 1 << 30, (n,), generator=g, dtype=torch.int32)
    row = torch.cat([k, v], 1).cuda()
    cap = budget + 2
    c = new_cache(S, cap, Hkv, dh, dtype)
    B.lazy_k_evict(row[:, :Hkv * dh], row[:, Hkv * dh:], pos.cuda(), mass.cuda(), cu(lens), max(lens), budget, recent, **c)
    B.lazy_device_status()
    a = 0
    got = {name: t.cpu() for name, t in c.items()}
    for s, ln in enumerate(lens):
        for h in range(Hkv):
            rows = R.kept_rows(mass[h, a:a + ln].numpy(), ln, budget, recent)
            m, at = len(rows), torch.tensor(rows, dtype=torch.int64) + a
            assert got["clen"][s, h].item() == m
            assert torch.equal(got["cpos"][s, h, :m], pos[at]) and torch.all(got["cpos"][s, h, m:] == -6)
            assert torch.equal(got["kc"][s, :m, h], k[at, h * dh:(h + 1) * dh])
            assert torch.equal(got["vc"][s, :m, h], v[at, h * dh:(h + 1) * dh])
            assert torch.all(got["kc"][s, m:, h] == 99) and torch.all(got["vc"][s, m:, h] == 98)
            assert np.array_equal(got["cmass"][s, h, :m].numpy(), mass[h, at].numpy(), equal_nan=True)
            assert torch.all(got["cmass"][s, h, m:] == -5)
        a += ln


def test_evict_long_sequence():
    """Longer than the keys that fit in shared memory, a few distinct weights, everything else equal."""
    n, Hkv, dh, budget = 60001, 1, 32, 500
    mass = torch.zeros((Hkv, n))
    heavy = torch.randperm(n, generator=gen(8))[:200]
    mass[0, heavy] = torch.rand(200, generator=gen(9)) + 0.5
    k = torch.arange(n, dtype=F32)[:, None].repeat(1, dh).cuda()
    c = new_cache(1, budget, Hkv, dh, F32)
    B.lazy_k_evict(k, k, torch.arange(n, dtype=torch.int32).cuda(), mass.cuda(), cu([n]), n, budget, 50, **c)
    B.lazy_device_status()
    want = R.kept_rows(mass[0].numpy(), n, budget, 50)
    assert c["cpos"][0, 0].cpu().tolist() == want
    assert c["kc"][0, :, 0, 0].cpu().tolist() == [float(w) for w in want]


def test_evict_reports_a_bad_length_table():
    c = new_cache(2, 4, 1, 32, F32)
    k = torch.zeros((10, 32), device="cuda")
    B.lazy_k_evict(k, k, torch.zeros(10, dtype=torch.int32).cuda(), torch.zeros((1, 10)).cuda(),
                   torch.tensor([0, 5, 11], dtype=torch.int32, device="cuda"), 10, 4, 0, **c)
    with pytest.raises(B.LazyError):
        B.lazy_device_status()
    assert c["clen"].cpu().tolist() == [[4], [-7]]   # the sequence that fits is served, the other left alone


# ------------------------------------------------------------------------------------------- one token
def step_case(seed, lens, budget, H, Hkv, dh, dtype, weights="distinct", cap=None):
    g, S = gen(seed), len(lens)
    cap = cap or budget + 1
    c = dict(kc=randn(g, S, cap, Hkv, dh, dtype=dtype), vc=randn(g, S, cap, Hkv, dh, dtype=dtype),
             cmass=torch.exp(2 * torch.randn((S, Hkv, cap), generator=g)),
             cpos=torch.stack([torch.stack([torch.randperm(cap, generator=g) for _ in range(Hkv)]) for _ in range(S)]).int(),
             clen=torch.tensor(lens, dtype=torch.int32)[:, None].repeat(1, Hkv))
    if weights == "ties":
        c["cmass"] = torch.randint(0, 3, (S, Hkv, cap), generator=g).float()
    for s, n in enumerate(lens):   # what lies behind the held slots must not matter
        c["kc"][s, n:], c["vc"][s, n:] = float("nan"), float("inf")
        c["cmass"][s, :, n:] = float("nan")
    new = dict(q=randn(g, S, H * dh, dtype=dtype), k_new=randn(g, S, Hkv * dh, dtype=dtype),
               v_new=randn(g, S, Hkv * dh, dtype=dtype), pos_new=torch.full((S,), cap + 3, dtype=torch.int32))
    return c, new


def step_expected(c, new, H, budget, recent):
    S, cap, Hkv, dh = c["kc"].shape
    kc, vc, cmass, cpos, clen = (c[k].clone() for k in ("kc", "vc", "cmass", "cpos", "clen"))
    o, amount = np.zeros((S, H, dh)), np.zeros((S, H, dh))
    slots, gones = np.zeros((S, Hkv), int), np.zeros((S, Hkv), int)
    m64 = cmass.numpy().astype(np.float64)
    e = 0.0
    for s in range(S):
        for g in range(Hkv):
            slot, gone, n = R.step_slot(cmass[s, g].numpy(), cpos[s, g].numpy(), int(clen[s, g]), budget,
                                        int(new["pos_new"][s]), recent)
            slots[s, g], gones[s, g] = slot, gone
            kc[s, slot, g] = new["k_new"][s, g * dh:(g + 1) * dh]
            vc[s, slot, g] = new["v_new"][s, g * dh:(g + 1) * dh]
            m64[s, g, slot], cpos[s, g, slot], clen[s, g] = 0.0, new["pos_new"][s], n
            K, V = f64(kc[s, :n, g]), f64(vc[s, :n, g])
            for h in range(g * (H // Hkv), (g + 1) * (H // Hkv)):
                qh = f64(new["q"][s, h * dh:(h + 1) * dh])
                w = R.softmax_row(qh, K, dh ** -0.5)
                o[s, h], amount[s, h] = w @ V, w @ np.abs(V)
                m64[s, g, :n] += w
                e = max(e, weight_error(qh[None], K, dh))
    return dict(kc=kc, vc=vc, cpos=cpos, clen=clen), m64, o, amount, slots, gones, e


def same_weights(got, want, e):
    """Grown weights: the gain (at most one per head, below it E of itself) and the sum's rounding; NaN and infinities alike."""
    fine = np.isfinite(want)
    if not np.array_equal(got[~fine], want[~fine], equal_nan=True):
        return False
    # a negative weight can cancel against its gain, which is at most |weight| + |sum| then
    size = np.where(want[fine] < 0, 2.0, np.abs(want[fine]))
    return bool(np.all(np.abs(got[fine] - want[fine]) <= (e + 2.0 ** -23) * size + 1e-30))


def check_step(c, new, H, budget, recent, in_place=False):
    dev = {k: v.cuda() for k, v in c.items()}
    dnew = {k: v.cuda() for k, v in new.items()}
    want, mass, o, amount, slots, gones, e = step_expected(c, new, H, budget, recent)
    outs = {} if in_place else dict(mass_out=dev["cmass"].clone(), pos_out=dev["cpos"].clone(), len_out=dev["clen"].clone())
    got_o, slot, gone = B.lazy_k_evict_step(**dnew, **dev, n_heads=H, budget=budget, n_recent=recent, **outs)
    B.lazy_device_status()
    assert np.array_equal(slot.cpu().numpy(), slots) and np.array_equal(gone.cpu().numpy(), gones)
    as_bytes = lambda t: t.contiguous().view(torch.uint8)  # noqa: E731
    for name in ("kc", "vc"):
        assert torch.equal(as_bytes(dev[name].cpu()), as_bytes(want[name])), name
    got_mass = (dev["cmass"] if in_place else outs["mass_out"]).cpu().numpy().astype(np.float64)
    assert torch.equal((dev["cpos"] if in_place else outs["pos_out"]).cpu(), want["cpos"])
    assert torch.equal((dev["clen"] if in_place else outs["len_out"]).cpu(), want["clen"])
    if not in_place:
        for name in ("cmass", "cpos", "clen"):
            assert torch.equal(as_bytes(dev[name].cpu()), as_bytes(c[name])), name   # the old state stays
    assert same_weights(got_mass, mass, e)
    go = f64(got_o).reshape(o.shape)
    tol = e * amount + half_step(c["kc"].dtype) * np.abs(o) * (1 + e) + 1e-30
    assert np.all(np.abs(go - o) <= tol), (np.abs(go - o) / tol).max()
    return dev, outs


@pytest.mark.parametrize("heads", HEADS, ids=IDS)
@pytest.mark.parametrize("lens,budget,recent", [([2], 2, 0), ([1, 0], 2, 1), ([64, 63, 65], 65, 10), ([300], 300, 299),
                                                ([129, 130, 0, 128], 130, 0), ([700], 700, 64)])
def test_evict_step(heads, lens, budget, recent):
    H, Hkv, dh, dtype = heads
    c, new = step_case(11 + budget, lens, budget, H, Hkv, dh, dtype)
    check_step(c, new, H, budget, recent)


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[1], HEADS[7]], ids=[IDS[0], IDS[1], IDS[7]])
def test_evict_step_ties_and_in_place(heads):
    H, Hkv, dh, dtype = heads
    c, new = step_case(12, [200, 180, 40], 200, H, Hkv, dh, dtype, weights="ties")
    check_step(c, new, H, 200, 30)
    check_step(c, new, H, 200, 30, in_place=True)


def test_evict_step_odd_weights_and_protected_slots():
    H, Hkv, dh, dtype = HEADS[1]
    c, new = step_case(13, [90, 90, 90], 90, H, Hkv, dh, dtype)
    c["cmass"][0, :, :90] = torch.tensor([float("inf"), 2.0, -0.0, 0.0, -1.0])[torch.arange(90) % 5]
    new["pos_new"][1] = -1                     # every position is newer: slot 0 is taken
    c["cmass"][2, 0, :90] = float("inf")
    check_step(c, new, H, 90, 5)
    c["cmass"][2, 1, 17] = float("nan")        # lighter than everything
    d = {k: v.cuda() for k, v in {**c, **new}.items()}
    d["pos_new"][:] = 1 << 20
    _, slot, _ = B.lazy_k_evict_step(**d, n_heads=H, budget=90, n_recent=5)
    B.lazy_device_status()
    assert slot[2, 1].item() == 17


@pytest.mark.parametrize("heads", [HEADS[1], HEADS[7]], ids=[IDS[1], IDS[7]])
def test_evict_step_reports_bad_lengths(heads):
    H, Hkv, dh, dtype = heads
    c, new = step_case(14, [20, 20, 20], 20, H, Hkv, dh, dtype)
    dev = {k: v.cuda() for k, v in c.items()}
    dev["clen"][0, 0], dev["clen"][2, Hkv - 1] = 21, -1
    before = {k: v.clone() for k, v in dev.items()}
    o, slot, gone = B.lazy_k_evict_step(**{k: v.cuda() for k, v in new.items()}, **dev, n_heads=H, budget=20, n_recent=2)
    with pytest.raises(B.LazyError) as err:
        B.lazy_device_status()
    assert err.value.status == -3
    G = H // Hkv
    for s, g in ((0, 0), (2, Hkv - 1)):
        assert slot[s, g].item() == gone[s, g].item() == -1
        assert torch.all(o.view(3, H, dh)[s, g * G:(g + 1) * G] == 0)
        assert torch.equal(dev["kc"][s, :20, g], before["kc"][s, :20, g])
        assert torch.equal(dev["cmass"][s, g, :20], before["cmass"][s, g, :20])
        assert dev["clen"][s, g] == before["clen"][s, g]
    assert torch.all(slot[1] >= 0) and torch.all(o.view(3, H, dh)[1].abs().amax(-1) > 0)


def test_evict_step_long_cache():
    H, Hkv, dh, dtype = HEADS[1]
    c, new = step_case(15, [9000], 9000, H, Hkv, dh, dtype)
    check_step(c, new, H, 9000, 1000)


@pytest.mark.parametrize("heads", [HEADS[2], HEADS[9], HEADS[10], (16, 1, 128, BF16)], ids=[IDS[2], IDS[9], IDS[10], "16on1x128"])
@pytest.mark.parametrize("lens", [[2100, 0], [2600, 2599, 17], [2049]])
def test_evict_step_long_caches_of_few_heads(heads, lens):
    """Many CTAs to a head, most of them without a slot where the cache is nearly empty."""
    H, Hkv, dh, dtype = heads
    c, new = step_case(28 + len(lens), lens, max(lens), H, Hkv, dh, dtype)
    check_step(c, new, H, max(lens), 100)


def test_evict_steps_in_a_row_and_replayed():
    """Forty steps in place from an almost empty cache, the same forty from one captured graph: the same state."""
    H, Hkv, dh, dtype, budget, S = 8, 2, 128, BF16, 24, 3
    start, _ = step_case(16, [0, 20, 24], budget, H, Hkv, dh, dtype)
    steps = [step_case(100 + i, [0, 0, 0], budget, H, Hkv, dh, dtype)[1] for i in range(40)]
    for i, st in enumerate(steps):
        st["pos_new"][:] = 1000 + i
    a, b = ({k: v.cuda() for k, v in start.items()} for _ in range(2))
    os = []
    for st in steps:
        o, _, _ = B.lazy_k_evict_step(**{k: v.cuda() for k, v in st.items()}, **a, n_heads=H, budget=budget, n_recent=4)
        os.append(o.clone())
    assert a["clen"].cpu().unique().tolist() == [budget]
    assert all(torch.all((a["cpos"] == 1000 + i).any(-1)) for i in range(36, 40))   # the newest are all there
    inp = {k: v.cuda() for k, v in steps[0].items()}
    scratch = B.lazy_k_evict_step_scratch(S, H, Hkv, dh, budget)
    out = tuple(t.clone() for t in B.lazy_k_evict_step(**inp, **{k: v.clone() for k, v in b.items()}, n_heads=H,
                                                        budget=budget, n_recent=4))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.lazy_k_evict_step(**inp, **b, n_heads=H, budget=budget, n_recent=4, scratch=scratch, out=out)
    for i, st in enumerate(steps):
        for k, v in st.items():
            inp[k].copy_(v)
        graph.replay()
        assert torch.equal(out[0], os[i]), i
    B.lazy_device_status()
    for name in ("cpos", "clen", "cmass"):
        valid = torch.arange(budget + 1, device="cuda") < b["clen"][..., None] if name != "clen" else None
        assert torch.equal(a[name] if valid is None else a[name][valid], b[name] if valid is None else b[name][valid])


# ------------------------------------------------------------------------------------------- shared prefix
def prefix_case(seed, n_pre, rows, own, H, Hkv, dh, dtype, pad=3):
    g, N, C = gen(seed), sum(rows), sum(own)
    d = dict(q=randn(g, N, H * dh, dtype=dtype), k_pre=randn(g, n_pre, Hkv * dh, dtype=dtype),
             v_pre=randn(g, n_pre, Hkv * dh, dtype=dtype), k=randn(g, C + pad, Hkv * dh, dtype=dtype),
             v=randn(g, C + pad, Hkv * dh, dtype=dtype),
             kv_idx=torch.randperm(C + pad, generator=g)[:C].to(torch.int32))
    unused = torch.ones(C + pad, dtype=torch.bool)
    unused[d["kv_idx"].long()] = False
    d["k"][unused], d["v"][unused] = float("nan"), float("inf")   # rows that no list names
    return d


def prefix_expected(d, rows, own, H, Hkv, dh, skip=()):
    n_pre = d["k_pre"].shape[0]
    o, tol = np.zeros((sum(rows), H, dh)), np.zeros((sum(rows), H, dh))
    kp, vp, k, v, q = (f64(d[x]) for x in ("k_pre", "v_pre", "k", "v", "q"))
    r = a = 0
    for T, C in zip(rows, own):
        for vis in R.prefix_visible(T, C):
            idx = [i for i in d["kv_idx"][a:a + vis].tolist() if i not in skip]
            for h in range(H):
                col = slice(h // (H // Hkv) * dh, (h // (H // Hkv) + 1) * dh)
                K, V = np.concatenate([kp[:, col], k[idx, col]]), np.concatenate([vp[:, col], v[idx, col]])
                if len(K):
                    qh = q[r, h * dh:(h + 1) * dh]
                    w = R.softmax_row(qh, K, dh ** -0.5)
                    o[r, h] = w @ V
                    e = weight_error(qh[None], K, dh)
                    tol[r, h] = e * (w @ np.abs(V)) + half_step(d["q"].dtype) * np.abs(o[r, h]) * (1 + e)
            r += 1
        a += C
    assert n_pre == kp.shape[0]
    return o, tol + 1e-30


def run_prefix(d, rows, own, H, Hkv, dh, **kw):
    dev = {k: v.cuda() for k, v in d.items()}
    return B.lazy_k_attention_prefix(dev["q"], cu(rows), max(rows), dev["k_pre"], dev["v_pre"], dev["k"], dev["v"],
                                     dev["kv_idx"], cu(own), max(own), H, Hkv, dh, **kw)


PREFIX_SHAPES = [(0, [1], [1]), (0, [1, 2], [0, 1]), (1, [1], [0]), (63, [1, 1, 1], [5, 64, 65]), (64, [5, 3], [5, 200]),
                 (65, [2], [1]), (300, [1] * 40, [1 + 3 * i for i in range(40)]), (129, [8, 1, 4], [129, 0, 128]),
                 (1000, [33], [40]), (200, [1, 0, 2], [3, 7, 2]), (0, [1, 1], [300, 20]), (0, [3, 5], [200, 4]),
                 (0, [4, 0, 8], [600, 9, 599])]


@pytest.mark.parametrize("heads", HEADS, ids=IDS)
@pytest.mark.parametrize("n_pre,rows,own", PREFIX_SHAPES)
def test_attention_prefix(heads, n_pre, rows, own):
    H, Hkv, dh, dtype = heads
    d = prefix_case(n_pre + sum(own), n_pre, rows, own, H, Hkv, dh, dtype)
    want, tol = prefix_expected(d, rows, own, H, Hkv, dh)
    got = run_prefix(d, rows, own, H, Hkv, dh)
    B.lazy_device_status()
    err = np.abs(f64(got).reshape(want.shape) - want)
    assert np.all(err <= tol), (err / tol).max()


def test_attention_prefix_pitches_and_poison():
    """Rows inside wider buffers; what surrounds prefix and queries is NaN."""
    H, Hkv, dh, rows, own, n_pre = 8, 2, 128, [3, 1], [10, 70], 150
    d = prefix_case(21, n_pre, rows, own, H, Hkv, dh, BF16)
    want, tol = prefix_expected(d, rows, own, H, Hkv, dh)
    w = Hkv * dh
    pre = torch.full((n_pre + 60, 2 * w + 8), float("nan"), dtype=BF16, device="cuda")
    kv = torch.full((d["k"].shape[0], 2 * w + 16), float("nan"), dtype=BF16, device="cuda")
    q = torch.full((4, H * dh + 24), float("nan"), dtype=BF16, device="cuda")
    pre[:n_pre, :w], pre[:n_pre, w:2 * w] = d["k_pre"].cuda(), d["v_pre"].cuda()
    kv[:, 8:8 + w], kv[:, 8 + w:8 + 2 * w] = d["k"].cuda(), d["v"].cuda()
    q[:, 16:16 + H * dh] = d["q"].cuda()
    out = torch.full((6, H * dh), 5.0, dtype=BF16, device="cuda")
    B.lazy_k_attention_prefix(q[:, 16:16 + H * dh], cu(rows), 3, pre[:n_pre, :w], pre[:n_pre, w:2 * w], kv[:, 8:8 + w],
                              kv[:, 8 + w:8 + 2 * w], d["kv_idx"].cuda(), cu(own), 70, H, Hkv, dh, out=out[:4])
    B.lazy_device_status()
    assert np.all(np.abs(f64(out[:4]).reshape(want.shape) - want) <= tol) and torch.all(out[4:] == 5)


def test_attention_prefix_large_logits_and_infinities():
    H, Hkv, dh, rows, own, n_pre = 8, 2, 128, [2, 2], [40, 300], 500
    d = prefix_case(22, n_pre, rows, own, H, Hkv, dh, BF16)
    d["q"] *= 20.0
    d["k_pre"][77] *= 30.0
    want, tol = prefix_expected(d, rows, own, H, Hkv, dh)
    got = run_prefix(d, rows, own, H, Hkv, dh)
    assert np.all(np.abs(f64(got).reshape(want.shape) - want) <= tol)
    # a key that a later row sees and an earlier one does not: NaN reaches the later row alone
    d = prefix_case(23, n_pre, rows, own, H, Hkv, dh, BF16)
    d["k"][int(d["kv_idx"][39])] = float("nan")
    d["v"][int(d["kv_idx"][39])] = float("nan")
    want, tol = prefix_expected({**d, "q": d["q"]}, rows, own, H, Hkv, dh)
    got = f64(run_prefix(d, rows, own, H, Hkv, dh)).reshape(want.shape)
    keep = [0, 2, 3]
    assert np.all(np.abs(got[keep] - want[keep]) <= tol[keep]) and np.all(np.isnan(got[1]))


@pytest.mark.parametrize("dh", [32, 64, 96, 128, 160])
@pytest.mark.parametrize("column", [0, 31, -1])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("n_pre", [0, 70])
def test_attention_prefix_hidden_values_at_every_width(dh, column, value, n_pre):
    """One odd number in one column of keys that only later rows see: the rows before are as without it."""
    H, Hkv, rows, own = 4, 2, [3, 5], [37, 18]
    d = prefix_case(24, n_pre, rows, own, H, Hkv, dh, BF16)
    want, tol = prefix_expected(d, rows, own, H, Hkv, dh)
    clean = run_prefix(d, rows, own, H, Hkv, dh)
    for j in (36, 37 + 15, 37 + 16):  # the first request's last key, the second's last but two and last but one
        d["v"][int(d["kv_idx"][j])].view(Hkv, dh)[:, column] = value
    got = f64(run_prefix(d, rows, own, H, Hkv, dh)).reshape(want.shape)
    clean = f64(clean).reshape(want.shape)
    assert np.all(np.abs(clean - want) <= tol)
    sees = [2, 5, 6, 7]
    hidden = [r for r in range(8) if r not in sees]
    assert np.array_equal(got[hidden], clean[hidden])
    odd = np.zeros(dh, bool)
    odd[column] = True
    assert np.all(~np.isfinite(got[sees][..., odd])) and np.all(np.isfinite(got[sees][..., ~odd]))


@pytest.mark.parametrize("dh", [32, 96, 160])
def test_other_widths_do_not_reach_beyond_their_heads(dh):
    """Rows and heads beside the ones in use hold NaN; nothing of it arrives, in products that fill a width up."""
    H, Hkv, n, rows, own, n_pre = 4, 2, 150, [2, 1], [20, 33], 90
    _, _, q, k = mass_case(25, [n], H, Hkv, dh, BF16, fused=False)
    want = B.lazy_k_attention_mass(q, k, cu([n]), n, H, Hkv, dh)
    wide_q = torch.full((n + 3, H * dh + 64), float("nan"), dtype=BF16, device="cuda")
    wide_k = torch.full((n + 3, Hkv * dh + 64), float("nan"), dtype=BF16, device="cuda")
    wide_q[:n, :H * dh], wide_k[:n, :Hkv * dh] = q, k
    got = B.lazy_k_attention_mass(wide_q[:n, :H * dh], wide_k[:n, :Hkv * dh], cu([n]), n, H, Hkv, dh)
    assert torch.equal(got, want)
    d = prefix_case(26, n_pre, rows, own, H, Hkv, dh, BF16)
    clean = run_prefix(d, rows, own, H, Hkv, dh)
    for name in ("k_pre", "v_pre"):
        x = torch.full((n_pre + 70, Hkv * dh + 64), float("nan"), dtype=BF16)
        x[:n_pre, :Hkv * dh] = d[name]
        d[name] = x
    dev = {key: v.cuda() for key, v in d.items()}
    got = B.lazy_k_attention_prefix(dev["q"], cu(rows), 2, dev["k_pre"][:n_pre, :Hkv * dh], dev["v_pre"][:n_pre, :Hkv * dh],
                                    dev["k"], dev["v"], dev["kv_idx"], cu(own), 33, H, Hkv, dh)
    assert torch.equal(got, clean)
    B.lazy_device_status()


@pytest.mark.parametrize("heads", [HEADS[1], HEADS[6], HEADS[10]], ids=[IDS[1], IDS[6], IDS[10]])
def test_attention_prefix_rows_of_nobody(heads):
    """Without a prefix, rows before the first request's and behind the last one's are reported and zero."""
    H, Hkv, dh, dtype = heads
    rows, own = [2, 3], [40, 90]
    d = prefix_case(29, 0, [1] + rows + [2], [1] + own + [2], H, Hkv, dh, dtype)
    dev = {k: v.cuda() for k, v in d.items()}
    cu_q = torch.tensor([1, 3, 6], dtype=torch.int32).cuda()
    cu_kv = torch.tensor([1, 41, 131], dtype=torch.int32).cuda()
    out = torch.full((8, H * dh), 7.0, dtype=dtype, device="cuda")
    got = B.lazy_k_attention_prefix(dev["q"], cu_q, 3, dev["k_pre"], dev["v_pre"], dev["k"], dev["v"], dev["kv_idx"], cu_kv,
                                    90, H, Hkv, dh, out=out)
    with pytest.raises(B.LazyError, match="BADARG"):
        B.lazy_device_status()
    want, tol = prefix_expected(d, [1] + rows + [2], [1] + own + [2], H, Hkv, dh)
    assert np.all(np.abs(f64(got).reshape(want.shape)[1:6] - want[1:6]) <= tol[1:6])
    assert not torch.any(got[0]) and not torch.any(got[6:])


@pytest.mark.parametrize("heads", [HEADS[1], HEADS[7]], ids=[IDS[1], IDS[7]])
def test_attention_prefix_takes_any_bounds(heads):
    """max_q and max_kv are bounds, not lengths: the largest number is one."""
    H, Hkv, dh, dtype = heads
    n_pre, rows, own = 65, [2, 1, 3], [5, 0, 70]
    d = prefix_case(27, n_pre, rows, own, H, Hkv, dh, dtype)
    want, tol = prefix_expected(d, rows, own, H, Hkv, dh)
    dev = {k: v.cuda() for k, v in d.items()}
    for max_q, max_kv in ((2 ** 31 - 1, 70), (3, 20000), (2 ** 31 - 1, 20000)):
        got = B.lazy_k_attention_prefix(dev["q"], cu(rows), max_q, dev["k_pre"], dev["v_pre"], dev["k"], dev["v"],
                                        dev["kv_idx"], cu(own), max_kv, H, Hkv, dh)
        assert np.all(np.abs(f64(got).reshape(want.shape) - want) <= tol)
    B.lazy_device_status()


@pytest.mark.parametrize("heads", [HEADS[1], HEADS[5]], ids=[IDS[1], IDS[5]])
def test_attention_prefix_reports_bad_rows_and_tables(heads):
    H, Hkv, dh, dtype = heads
    rows, own = [1, 2], [20, 30]
    d = prefix_case(24, 100, rows, own, H, Hkv, dh, dtype)
    d["kv_idx"][5], d["kv_idx"][33] = d["k"].shape[0], -1
    got = run_prefix(d, rows, own, H, Hkv, dh)
    with pytest.raises(B.LazyError):
        B.lazy_device_status()
    want, tol = prefix_expected(d, rows, own, H, Hkv, dh, skip=(d["k"].shape[0], -1))
    assert np.all(np.abs(f64(got).reshape(want.shape) - want) <= tol)
    d = prefix_case(25, 100, rows, own, H, Hkv, dh, dtype)
    dev = {k: v.cuda() for k, v in d.items()}
    for c_q, c_kv, max_q, max_kv in (([0, 1, 3], [0, 20, 51], 2, 31), ([0, 1, 3], [0, 20, 50], 2, 29),
                                     ([0, 1, 3], [0, 20, 50], 1, 30), ([0, 1, 2], [0, 20, 50], 2, 30)):
        B.lazy_k_attention_prefix(dev["q"], torch.tensor(c_q, dtype=torch.int32, device="cuda"), max_q, dev["k_pre"],
                                  dev["v_pre"], dev["k"], dev["v"], dev["kv_idx"],
                                  torch.tensor(c_kv, dtype=torch.int32, device="cuda"), max_kv, H, Hkv, dh)
        with pytest.raises(B.LazyError):
            B.lazy_device_status()


# ------------------------------------------------------------------------------------------- verification
def verify_case(seed, drafts, V, outright=False, near=0.7):
    g, total, n = gen(seed), sum(drafts), len(drafts)
    logits = 3 * torch.randn((total + n, V), generator=g)
    at = torch.cat([torch.arange(d) + sum(drafts[:i]) + i for i, d in enumerate(drafts)]) if total else torch.zeros(0).long()
    q = torch.softmax(logits[at] + near * torch.randn((total, V), generator=g), -1)
    draft = torch.multinomial(q, 1, generator=g).view(-1).int() if total else torch.zeros(0, dtype=torch.int32)
    return dict(p=torch.softmax(logits, -1), q=None if outright else q, draft=draft,
                u_accept=torch.rand(total, generator=g), u_sample=torch.rand(n, generator=g))


def check_verify(d, drafts, pitch=0):
    n, T = len(drafts), max(drafts)

    def put(t):
        if t is None or not pitch:
            return None if t is None else t.cuda()
        wide = torch.full((t.shape[0], t.shape[1] + pitch), float("nan"))
        wide[:, 1:1 + t.shape[1]] = t
        return wide.cuda()[:, 1:1 + t.shape[1]]
    acc, tokens = B.lazy_k_verify(put(d["p"]), d["draft"].cuda(), cu(drafts), T, d["u_accept"].cuda(), d["u_sample"].cuda(),
                                  q=put(d["q"]))
    acc, tokens = acc.cpu().tolist(), tokens.cpu().tolist()
    a = 0
    for s, t in enumerate(drafts):
        x = d["draft"][a:a + t].numpy()
        qs = None if d["q"] is None else d["q"][a:a + t].numpy()
        want, token = R.verify(d["p"][a + s:a + s + t + 1].numpy(), qs, x, d["u_accept"][a:a + t].numpy(),
                               d["u_sample"][s].item())
        assert acc[s] == want
        assert tokens[s] == x[:want].tolist() + [token] + [-1] * (T - want)
        a += t
    return acc


@pytest.mark.parametrize("V", [1, 5, 127, 1000, 2048, 32000, 128256])
@pytest.mark.parametrize("outright", [False, True])
def test_verify(V, outright):
    drafts = [4, 0, 1, 7, 3] if V < 100000 else [2, 0]
    check_verify(verify_case(31 + V, drafts, V, outright), drafts)
    B.lazy_device_status()


def test_verify_many_and_pitches():
    drafts = [(3 * i) % 6 for i in range(300)]
    acc = check_verify(verify_case(32, drafts, 777), drafts, pitch=5)
    assert len(set(zip(acc, drafts))) == 1 + 4   # none drafted; of three, none to all accepted
    check_verify(verify_case(33, [40, 33, 32, 31], 50, near=0.05), [40, 33, 32, 31])   # longer than one warp looks at
    check_verify(verify_case(34, [0, 0], 4096), [0, 0])
    B.lazy_device_status()


def test_verify_edges():
    """Equal distributions (nothing left after a rejection), one possible id, u = 0, zero probabilities, NaN."""
    V = 300
    d = verify_case(35, [2, 2, 1, 1], V)
    d["p"][0], d["q"][0] = d["q"][0], d["q"][0].clone()
    d["u_accept"][0] = 1.0                                     # rejected although p = q: the target's own row
    d["p"][3] = 0.0
    d["p"][3, 250] = 1.0                                        # one id holds everything
    d["u_sample"][:] = torch.tensor([0.3, 0.0, 0.999999, 0.5])
    d["p"][6, :100] = float("nan")
    d["u_accept"][4] = 1.0
    check_verify(d, [2, 2, 1, 1])
    d["p"][8] = 0.0                                             # the last sequence's rows: nothing to draw from
    d["p"][9] = 0.0
    acc, tokens = B.lazy_k_verify(d["p"].cuda(), d["draft"].cuda(), cu([2, 2, 1, 1]), 2, d["u_accept"].cuda(),
                                  d["u_sample"].cuda(), q=d["q"].cuda())
    with pytest.raises(B.LazyError):
        B.lazy_device_status()
    assert acc[3].item() == 0 and tokens[3].tolist() == [-1, -1, -1]


def test_verify_reports_bad_ids_and_tables():
    d = verify_case(36, [2, 1], 50)
    d["draft"][0] = 50
    acc, _ = B.lazy_k_verify(d["p"].cuda(), d["draft"].cuda(), cu([2, 1]), 2, d["u_accept"].cuda(), d["u_sample"].cuda(),
                             q=d["q"].cuda())
    with pytest.raises(B.LazyError):
        B.lazy_device_status()
    assert acc[0].item() == 0
    d = verify_case(36, [2, 1], 50)
    B.lazy_k_verify(d["p"].cuda(), d["draft"].cuda(), torch.tensor([0, 3, 2], dtype=torch.int32, device="cuda"), 2,
                    d["u_accept"].cuda(), d["u_sample"].cuda(), q=d["q"].cuda())
    with pytest.raises(B.LazyError):
        B.lazy_device_status()


def test_verify_leaves_the_target_distribution():
    """Accepted or replaced, the first token is distributed as the target's first row: counts over a grid of numbers."""
    V, n = 6, 20000
    g = gen(37)
    p = torch.tensor([0.3, 0.05, 0.25, 0.0, 0.3, 0.1])
    q = torch.tensor([0.1, 0.4, 0.1, 0.2, 0.1, 0.1])
    draft = torch.multinomial(q, n, replacement=True, generator=g).int()
    rows = torch.stack([p, p]).repeat(n, 1)
    _, tokens = B.lazy_k_verify(rows.cuda(), draft.cuda(), torch.arange(n + 1, dtype=torch.int32).cuda(), 1,
                                torch.rand(n, generator=g).cuda(), torch.rand(n, generator=g).cuda(), q=q.repeat(n, 1).cuda())
    share = torch.bincount(tokens[:, 0].cpu().long(), minlength=V) / n
    assert torch.all((share - p).abs() <= 5 * torch.sqrt(p * (1 - p) / n) + 1e-9)   # five standard deviations


# ------------------------------------------------------------------------------------------- refusals of the binding
def test_binding_refuses_what_does_not_fit():
    q = torch.zeros((4, 256), dtype=BF16, device="cuda")
    k = torch.zeros((4, 128), dtype=BF16, device="cuda")
    c = cu([4])
    with pytest.raises(ValueError):
        B.lazy_k_attention_mass(q, k.float(), c, 4, 4, 2, 64)
    with pytest.raises(ValueError):
        B.lazy_k_attention_mass(q.cpu(), k, c, 4, 4, 2, 64)
    with pytest.raises(ValueError):
        B.lazy_k_attention_mass(q, k[:3], c, 4, 4, 2, 64)
    with pytest.raises(ValueError):
        B.lazy_k_attention_mass(q, k, c.long(), 4, 4, 2, 64)
    with pytest.raises(ValueError):
        B.lazy_k_attention_mass(q, k, c, 4, 4, 2, 64, out=torch.zeros(7, device="cuda"))
    with pytest.raises(ValueError):
        B.lazy_k_verify(torch.zeros((3, 8), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), cu([1]), 1,
                        torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"))
    with pytest.raises(B.LazyError):
        B.lazy_k_attention_mass(q, k, c, 4, 4, 2, 64, scratch=torch.zeros(1, device="cuda"))


# ------------------------------------------------------------------------------------------- graphs and streams
def _mass_call(H, Hkv, dh, dtype, lens, window):
    def inputs(seed):
        _, _, q, k = mass_case(seed, lens, H, Hkv, dh, dtype, fused=False)
        return dict(q=q, k=k, cu=cu(lens))

    def call(x):
        return (B.lazy_k_attention_mass(x["q"], x["k"], x["cu"], max(lens), H, Hkv, dh, window),)
    return inputs, call


def _evict_call(Hkv, dh, dtype, lens, budget, recent):
    def inputs(seed):
        g, n = gen(seed), sum(lens)
        return dict(k=randn(g, n, Hkv * dh, dtype=dtype).cuda(), v=randn(g, n, Hkv * dh, dtype=dtype).cuda(),
                    pos=torch.arange(n, dtype=torch.int32).cuda(), mass=torch.rand((Hkv, n), generator=g).cuda(), cu=cu(lens),
                    **new_cache(len(lens), budget + 2, Hkv, dh, dtype))

    def call(x):
        c = {name: x[name] for name in ("kc", "vc", "cmass", "cpos", "clen")}
        B.lazy_k_evict(x["k"], x["v"], x["pos"], x["mass"], x["cu"], max(lens), budget, recent, **c)
        return tuple(c.values())
    return inputs, call


def _step_call(H, Hkv, dh, dtype, lens, budget):
    def inputs(seed):
        c, new = step_case(seed, lens, budget, H, Hkv, dh, dtype)
        return {name: t.cuda() for name, t in {**c, **new}.items()}

    def call(x):
        out = B.lazy_k_evict_step(**x, n_heads=H, budget=budget, n_recent=1)
        return (*out, x["cpos"], x["clen"], *(x["kc"][s, :n] for s, n in enumerate(lens)),
                *(x["cmass"][s, :, :min(n + 1, budget)] for s, n in enumerate(lens)))
    return inputs, call


def _prefix_call(H, Hkv, dh, dtype, n_pre, rows, own):
    def inputs(seed):
        d = prefix_case(seed, n_pre, rows, own, H, Hkv, dh, dtype)
        return {**{name: t.cuda() for name, t in d.items()}, "cu_q": cu(rows), "cu_kv": cu(own)}

    def call(x):
        return (B.lazy_k_attention_prefix(x["q"], x["cu_q"], max(rows), x["k_pre"], x["v_pre"], x["k"], x["v"], x["kv_idx"],
                                          x["cu_kv"], max(own), H, Hkv, dh),)
    return inputs, call


def _verify_call(V, drafts):
    def inputs(seed):
        return {**{name: t.cuda() for name, t in verify_case(seed, drafts, V).items()}, "cu": cu(drafts)}

    def call(x):
        return B.lazy_k_verify(x["p"], x["draft"], x["cu"], max(drafts), x["u_accept"], x["u_sample"], q=x["q"])
    return inputs, call


CALLS = {
    "mass": _mass_call(8, 2, 128, BF16, [700, 1, 333], 0), "mass_split_keys": _mass_call(8, 8, 64, BF16, [5000, 40], 33),
    "mass_f32": _mass_call(4, 2, 64, F32, [150, 20], 0), "evict": _evict_call(2, 64, BF16, [500, 30], 100, 10),
    "step": _step_call(8, 2, 128, BF16, [300, 40, 0], 300), "step_long": _step_call(8, 1, 64, BF16, [2200], 2200),
    "step_f32": _step_call(4, 4, 64, F32, [60, 3], 60), "prefix": _prefix_call(8, 2, 128, BF16, 700, [2, 1, 3], [9, 150, 40]),
    "prefix_none": _prefix_call(8, 2, 64, BF16, 0, [1, 2], [200, 30]), "prefix_f32": _prefix_call(6, 2, 32, F32, 100, [2, 1], [9, 15]),
    "verify": _verify_call(5000, [3, 0, 5]),
}


@pytest.mark.parametrize("name", CALLS)
def test_captured_calls_take_new_inputs(name):
    """A captured call, replayed on other inputs in the same buffers, gives what the call itself gives."""
    inputs, call = CALLS[name]
    x = inputs(50)
    want = [t.clone() for t in call(inputs(51))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = call(x)
    for seed in (52, 51):
        for key, t in inputs(seed).items():
            x[key].copy_(t)
        graph.replay()
    torch.cuda.synchronize()
    B.lazy_device_status()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and len(got) == len(want)


def test_calls_at_once_on_two_streams():
    """Every operator on two streams at once, several times over, each with its own scratch: the same bits as alone."""
    for name, (inputs, call) in CALLS.items():
        want = [[t.clone() for t in call(inputs(seed))] for seed in (60, 61)]
        sets = [[inputs(seed) for _ in range(6)] for seed in (60, 61)]
        torch.cuda.synchronize()
        streams, got = (torch.cuda.Stream(), torch.cuda.Stream()), ([], [])
        for i in range(6):
            for k in range(2):
                with torch.cuda.stream(streams[k]):
                    got[k].append(call(sets[k][i]))
        torch.cuda.synchronize()
        B.lazy_device_status()
        for k in range(2):
            for out in got[k]:
                assert all(torch.equal(a, b) for a, b in zip(out, want[k])), name


# ------------------------------------------------------------------------------------------- far offsets
FAR = 2 ** 31 + 2 ** 24   # elements: rows at the end of such a buffer lie behind what 32 bits reach


def far_rows(t, pitch):
    """The rows of t at the end of a buffer of FAR elements, `pitch` apart; the first row lies at its start."""
    rows = FAR // pitch
    far = torch.zeros((rows, pitch), dtype=t.dtype, device="cuda")
    far[rows - t.shape[0]:, :t.shape[1]] = t.cuda()
    return far, rows - t.shape[0]


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_mass_and_evict_of_far_rows(dtype):
    H, Hkv, dh, n = 4, 2, 64, 90
    _, _, q, k = mass_case(70, [n], H, Hkv, dh, dtype, fused=False)
    v = randn(gen(71), n, Hkv * dh, dtype=dtype).cuda()
    want = B.lazy_k_attention_mass(q, k, cu([n]), n, H, Hkv, dh)
    wide = torch.cat([q, k, v], 1)
    far, first = far_rows(wide, 2 ** 21)
    table = cu([first, n])
    fq, fk, fv = far[:, :H * dh], far[:, H * dh:(H + Hkv) * dh], far[:, (H + Hkv) * dh:(H + 2 * Hkv) * dh]
    got = B.lazy_k_attention_mass(fq, fk, table, far.shape[0], H, Hkv, dh)
    e = weight_error(f64(q).reshape(n, H, dh), f64(k).reshape(n, Hkv, dh), dh) + n * H * 2.0 ** -24   # and of fp32 sums
    assert torch.all((got[:, first:] - want).abs() <= 2 * e * want)
    pos = torch.arange(far.shape[0], dtype=torch.int32).cuda()
    c = new_cache(2, 20, Hkv, dh, dtype)
    B.lazy_k_evict(fk, fv, pos, got, table, far.shape[0], 20, 5, **c)
    B.lazy_device_status()
    for h in range(Hkv):
        kept = R.kept_rows(got[h, first:].cpu().numpy(), n, 20, 5)
        assert (c["cpos"][1, h].cpu() - first).tolist() == kept
        assert torch.equal(c["kc"][1, :, h], k.view(n, Hkv, dh)[kept, h]) and torch.equal(c["vc"][1, :, h], v.view(n, Hkv, dh)[kept, h])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_prefix_and_verify_of_far_rows(dtype):
    H, Hkv, dh, rows, own = 4, 2, 64, [2, 1], [30, 70]
    d = prefix_case(72, 130, rows, own, H, Hkv, dh, dtype)
    clean = run_prefix(d, rows, own, H, Hkv, dh)
    far_k, first = far_rows(torch.nan_to_num(d["k"], posinf=0.0), 2 ** 21)
    far_v, _ = far_rows(torch.nan_to_num(d["v"], posinf=0.0), 2 ** 21)
    w = Hkv * dh
    got = B.lazy_k_attention_prefix(d["q"].cuda(), cu(rows), 2, d["k_pre"].cuda(), d["v_pre"].cuda(), far_k[:, :w], far_v[:, :w],
                                    d["kv_idx"].cuda() + first, cu(own), 70, H, Hkv, dh)
    assert torch.equal(got, clean)
    del far_v
    if dtype == F32:   # the last request's rows of the target lie far behind the first one's
        V, n = 40, far_k.shape[0] - 2
        x = verify_case(73, [1], V)
        far_k[:, :V] = 0.0
        far_k[-2:, :V] = x["p"].cuda()
        far_k[:-2, 0] = 1.0
        acc, tokens = B.lazy_k_verify(far_k[:, :V], x["draft"].cuda(), torch.tensor([0] * (n + 1) + [1], dtype=torch.int32).cuda(),
                                      1, x["u_accept"].cuda(), torch.cat([torch.zeros(n), x["u_sample"]]).cuda(), q=x["q"].cuda())
        assert (acc[-1].item(), tokens[-1, acc[-1].item()].item()) == R.verify(
            x["p"].numpy(), x["q"].numpy(), x["draft"].numpy(), x["u_accept"].numpy(), x["u_sample"][0].item())
        assert not torch.any(tokens[:-1, 0]) and not torch.any(acc[:-1])
    B.lazy_device_status()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_step_on_far_caches(dtype):
    """Many sequences, the last of which lies behind 2^31 elements."""
    H, Hkv, dh, budget, cap = 4, 2, 64, 40, 270
    c, new = step_case(74, [40], budget, H, Hkv, dh, dtype, cap=cap)
    S = FAR // (cap * Hkv * dh)
    many = {name: torch.zeros((S, *t.shape[1:]), dtype=t.dtype, device="cuda") for name, t in {**c, **new}.items()}
    for name, t in {**c, **new}.items():
        many[name][-1] = t[0].cuda()
    one = {name: t.cuda() for name, t in {**c, **new}.items()}
    want = B.lazy_k_evict_step(**one, n_heads=H, budget=budget, n_recent=3)
    got = B.lazy_k_evict_step(**many, n_heads=H, budget=budget, n_recent=3)
    B.lazy_device_status()
    _, m64, o64, amount, slots, gones, e = step_expected(c, new, H, budget, 3)
    for o, slot, gone in ((got[0][-1], got[1][-1], got[2][-1]), (want[0][0], want[1][0], want[2][0])):
        assert np.all(np.abs(f64(o).reshape(o64[0].shape) - o64[0]) <= e * amount[0] + half_step(dtype) * np.abs(o64[0]) * (1 + e))
        assert np.array_equal(slot.cpu().numpy(), slots[0]) and np.array_equal(gone.cpu().numpy(), gones[0])
    for name in ("kc", "vc"):
        assert torch.equal(many[name][-1, :40], one[name][0, :40])
    assert torch.equal(many["cpos"][-1, :, :40], one["cpos"][0, :, :40])
    assert same_weights(many["cmass"][-1:, :, :40].cpu().numpy().astype(np.float64), m64[:, :, :40], e)


# ------------------------------------------------------------------------------------------- together
def test_a_pruned_prompt_shared_by_requests_with_drafts():
    """As they are used: a prompt is weighed, cut to a budget, shared by three requests with drafted tokens, whose
    drafts are verified; then one request continues token by token on the cut cache.  On a side stream throughout."""
    H, Hkv, dh, n, budget, V = 8, 2, 128, 400, 96, 500
    g = gen(41)
    q, k, v = (randn(g, n, w * dh, dtype=BF16) for w in (H, Hkv, Hkv))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mass = B.lazy_k_attention_mass(q.cuda(), k.cuda(), cu([n]), n, H, Hkv, dh)
        c = new_cache(1, budget, Hkv, dh, BF16)
        B.lazy_k_evict(k.cuda(), v.cuda(), torch.arange(n, dtype=torch.int32).cuda(), mass, cu([n]), n, budget, 16, **c)
        rows, own = [3, 1, 4], [9, 1, 20]
        d = prefix_case(42, 0, rows, own, H, Hkv, dh, BF16)
        pre = {x: c[y][0].reshape(budget, Hkv * dh) for x, y in (("k_pre", "kc"), ("v_pre", "vc"))}
        dev = {x: t.cuda() for x, t in d.items()}
        o = B.lazy_k_attention_prefix(dev["q"], cu(rows), 4, pre["k_pre"], pre["v_pre"], dev["k"], dev["v"], dev["kv_idx"],
                                      cu(own), 20, H, Hkv, dh)
        w = torch.randn((V, H * dh), generator=g).to(BF16).cuda()
        p = torch.softmax(B.lazy_k_gemm(o, torch.nn.functional.pad(w, (0, 0, 0, 4))).float()[:, :V], -1)
        drafts = [2, 0, 3]
        draft = torch.tensor([int(p[0].argmax()), 7, int(p[4].argmax()), 1, 2], dtype=torch.int32)
        u, us = torch.rand(5, generator=g), torch.rand(3, generator=g)
        acc, tokens = B.lazy_k_verify(p, draft.cuda(), cu(drafts), 3, u.cuda(), us.cuda())
        new = dict(q=randn(g, 1, H * dh, dtype=BF16), k_new=randn(g, 1, Hkv * dh, dtype=BF16),
                   v_new=randn(g, 1, Hkv * dh, dtype=BF16), pos_new=torch.tensor([n], dtype=torch.int32))
        before = {x: t.cpu().clone() for x, t in c.items()}
        so, slot, gone = B.lazy_k_evict_step(**{x: t.cuda() for x, t in new.items()}, **c, n_heads=H, budget=budget,
                                             n_recent=16)
        B.lazy_device_status()
    # the cut: from the weights that came out (their own error is tested above)
    m = mass.cpu().numpy()
    for h in range(Hkv):
        assert before["cpos"][0, h].tolist() == R.kept_rows(m[h], n, budget, 16)
    ref = dict(d, **{x: t.cpu() for x, t in pre.items()})
    ref["k_pre"] = before["kc"][0].reshape(budget, -1)
    ref["v_pre"] = before["vc"][0].reshape(budget, -1)
    want, tol = prefix_expected(ref, rows, own, H, Hkv, dh)
    assert np.all(np.abs(f64(o).reshape(want.shape) - want) <= tol)
    pn, a = p.cpu().numpy(), 0
    for s, t in enumerate(drafts):
        got = R.verify(pn[a + s:a + s + t + 1], None, draft[a:a + t].numpy(), u[a:a + t].numpy(), us[s].item())
        assert (acc[s].item(), tokens[s, acc[s].item()].item()) == got
        a += t
    _, m64, so64, amount, slots, gones, e = step_expected(before, new, H, budget, 16)
    assert np.array_equal(slot.cpu().numpy(), slots) and np.array_equal(gone.cpu().numpy(), gones)
    assert np.all(np.abs(f64(so).reshape(so64.shape) - so64) <= e * amount + half_step(BF16) * np.abs(so64) * (1 + e))
    assert same_weights(c["cmass"].cpu().numpy().astype(np.float64), m64, e)
