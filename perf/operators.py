"""What is measured of the operators for serving from bounded and shared caches: their plain forms, the
calls a program makes of the library, and cases over the range in use.

  mass     accumulated attention weight of a prompt, per key/value head and key
  evict    a prompt's keys and values compacted to a budget by that weight, the newest kept regardless
  step     one token on such a cache: eviction, attention, accumulation
  prefix   attention of a batch of requests over one shared prefix and each request's own keys
  verify   drafted tokens accepted or replaced by the target's probabilities and given random numbers

`own` chooses between the plain form (False) and the library's calls (True).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _ints(text):
    return [int(t) for t in text.split(",")]


def _text(values):
    return ",".join(str(int(v)) for v in values)


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # heavy-hitter weights of one prompt of the mean length of the long-context suite, 7B shape
        dict(name="mass_prompt_3376", op="mass", dtype="bf16", n_heads=32, n_kv_heads=32, head_dim=128,
             lens="3376", window=0),
        # the same over the last 64 rows of a long prompt (observation window), grouped heads
        dict(name="mass_window64_16k", op="mass", dtype="bf16", n_heads=32, n_kv_heads=8, head_dim=128,
             lens="16384", window=64),
        # a packed batch of ragged prompts, grouped heads
        dict(name="mass_batch4_ragged", op="mass", dtype="bf16", n_heads=32, n_kv_heads=8, head_dim=128,
             lens="3309,1968,4079,2232", window=0),
        # the tiny fp32 decoder's shape, a few short prompts
        dict(name="mass_tiny_f32", op="mass", dtype="f32", n_heads=4, n_kv_heads=4, head_dim=64,
             lens="200,1,77", window=0),
        # a prompt's cache cut to 1024 slots after the prefill
        dict(name="evict_prompt_3376", op="evict", dtype="bf16", n_kv_heads=32, head_dim=128, lens="3376",
             budget=1024, recent=128),
        # a packed batch of long and short prompts cut to 2048 slots, grouped heads
        dict(name="evict_batch8_ragged", op="evict", dtype="bf16", n_kv_heads=8, head_dim=128,
             lens="16384,9001,4079,1968,3376,1,2585,7777", budget=2048, recent=256),
        # one request decoding on a full cache: the latency case
        dict(name="step_single_1024", op="step", dtype="bf16", n_heads=32, n_kv_heads=32, head_dim=128,
             lens="1024", budget=1024, recent=128),
        # a batch of requests, most of them at their budget
        dict(name="step_batch32_2048", op="step", dtype="bf16", n_heads=32, n_kv_heads=8, head_dim=128,
             lens=_text([2048] * 24 + [2047, 1500, 777, 1, 0, 300, 1024, 64]), budget=2048, recent=256),
        # four requests with four drafted tokens each behind a short shared prompt
        dict(name="prefix_drafts4_1000", op="prefix", dtype="bf16", n_heads=32, n_kv_heads=32, head_dim=128,
             n_prefix=1000, rows="5,5,5,5", own="40,133,5,261"),
        # a batch of requests behind a long shared prompt, one token each
        dict(name="prefix_batch64_16k", op="prefix", dtype="bf16", n_heads=32, n_kv_heads=8, head_dim=128,
             n_prefix=16384, rows=_text([1] * 64), own=_text([1 + (37 * i * i) % 500 for i in range(64)])),
        # one request's four drafted tokens
        dict(name="verify_single", op="verify", vocab=32000, drafts="4", drafted_probs=True),
        # a batch of requests, zero to seven drafted tokens each
        dict(name="verify_batch128", op="verify", vocab=32000, drafts=_text([(5 * i) % 8 for i in range(128)]),
             drafted_probs=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["mass", "evict", "step", "prefix", "verify"])
    if op == "verify":
        vocab = _log(rng, 1000, 128256)
        n = min(_log(rng, 1, 128), max(1, 4_000_000 // vocab))
        t = rng.randint(0, 8)
        return dict(op=op, vocab=vocab, drafts=_text(rng.randint(0, t) for _ in range(n)),
                    drafted_probs=rng.random() < 0.75)
    f32 = rng.random() < 0.2
    if f32:
        H, Hkv, dh = rng.choice([(4, 4, 64), (8, 2, 64), (4, 2, 128), (6, 2, 32)])
    else:
        H, Hkv, dh = rng.choice([(32, 32, 128), (32, 8, 128), (32, 8, 128), (8, 1, 128), (16, 4, 64), (8, 8, 64),
                                 (12, 4, 128), (8, 2, 96)])
    head = dict(op=op, dtype="f32" if f32 else "bf16")
    if op == "mass":
        top = 700 if f32 else 16384
        n = _log(rng, 1, 6)
        longest = _log(rng, 8, top)
        lens = [longest] + [_log(rng, 1, longest) for _ in range(n - 1)]
        window = rng.choice([0, 0, 1, _log(rng, 2, 300)])
        while n * H * longest * min(longest, window or longest) > 4 * 32 * 4079 ** 2 // 2:
            longest = longest * 2 // 3
            lens = [min(v, longest) for v in lens]
        return dict(head, n_heads=H, n_kv_heads=Hkv, head_dim=dh, lens=_text(lens), window=window)
    if op == "evict":
        n = _log(rng, 1, 8)
        longest = _log(rng, 1, 2000 if f32 else 16384)
        budget = _log(rng, 1, 2048)
        return dict(head, n_kv_heads=min(Hkv, 8) if n > 1 else Hkv, head_dim=dh,
                    lens=_text([longest] + [_log(rng, 1, longest) for _ in range(n - 1)]), budget=budget,
                    recent=min(budget, rng.choice([0, 1, budget // 4, budget // 2])))
    if op == "step":
        n = _log(rng, 1, 32)
        budget = max(2, min(_log(rng, 2, 1000 if f32 else 16384), 32 * 2048 * 8 * 128 // (n * Hkv * dh)))
        lens = [budget if rng.random() < 0.7 else rng.randint(0, budget) for _ in range(n)]
        return dict(head, n_heads=H, n_kv_heads=Hkv, head_dim=dh, lens=_text(lens), budget=budget,
                    recent=rng.choice([0, 1, budget // 8, budget // 2]))
    n = _log(rng, 1, 64)
    t = rng.choice([1, 1, rng.randint(2, 8)])
    rows = [rng.randint(1, t) for _ in range(n)]
    n_prefix = rng.choice([0, _log(rng, 1, 1500 if f32 else 16384)])
    n_prefix = min(n_prefix, 64 * 16384 * 32 // (sum(rows) * H))
    most = max(8, min(500, 64 * 500 * 8 // (n * Hkv)))
    return dict(head, n_heads=H, n_kv_heads=Hkv, head_dim=dh, n_prefix=n_prefix, rows=_text(rows),
                own=_text(r + _log(rng, 1, most) - 1 for r in rows))


# ------------------------------------------------------------------------------------------ work
def work(case):
    op = case["op"]
    if op == "verify":
        drafts = _ints(case["drafts"])
        # the drafted tokens' probabilities, one row of the target and, after a rejection, one of the draft model
        rows = sum(2 if d and case["drafted_probs"] else 1 for d in drafts)
        return {"bytes": 4.0 * case["vocab"] * rows + 16.0 * sum(drafts) + 8.0 * len(drafts),
                "flops": 2.0 * case["vocab"] * rows}
    eb = 2 if case["dtype"] == "bf16" else 4
    Hkv, dh = case["n_kv_heads"], case["head_dim"]
    if op == "evict":
        lens = _ints(case["lens"])
        kept = sum(min(n, case["budget"]) for n in lens)
        return {"bytes": kept * Hkv * (4.0 * dh * eb + 8) + sum(lens) * (4.0 * Hkv + 4), "flops": 0.0}
    H = case["n_heads"]
    if op == "mass":
        lens, w = _ints(case["lens"]), case["window"]
        rows = [min(n, w or n) for n in lens]
        pairs = sum(r * n - r * (r - 1) / 2.0 for r, n in zip(rows, lens))
        return {"bytes": eb * dh * (H * sum(rows) + Hkv * sum(lens)) + 4.0 * Hkv * sum(lens),
                "flops": 2.0 * pairs * H * dh}
    if op == "step":
        held = [min(n + 1, case["budget"]) for n in _ints(case["lens"])]
        return {"bytes": sum(held) * Hkv * (2.0 * dh * eb + 16) + len(held) * eb * dh * (2.0 * H + 4.0 * Hkv),
                "flops": 4.0 * sum(held) * H * dh}
    rows, keys = _ints(case["rows"]), _ints(case["own"])
    seen = sum(r * c - r * (r - 1) / 2.0 for r, c in zip(rows, keys)) + sum(rows) * case["n_prefix"]
    return {"bytes": 2.0 * eb * dh * Hkv * (case["n_prefix"] + sum(keys)) + 2.0 * eb * dh * H * sum(rows),
            "flops": 4.0 * seen * H * dh}


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _cu(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")


def _keys(g, n, Hkv, dh, along):
    """Keys with heavy hitters: a few lie far along the direction that the queries share."""
    weight = torch.exp(_randn(g, n, Hkv, 1)).clamp(max=16.0)
    return _randn(g, n, Hkv, dh) + 0.35 * math.sqrt(dh) * weight * along


def _queries(g, n, H, dh, along, Hkv):
    return _randn(g, n, H, dh) + along.repeat_interleave(H // Hkv, 0)


def _along(g, Hkv, dh):
    a = _randn(g, Hkv, dh)
    return a / a.norm(dim=-1, keepdim=True)


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    s = dict(case)
    if op == "verify":
        drafts, V = _ints(case["drafts"]), case["vocab"]
        n, total = len(drafts), sum(drafts)
        logits = 3.0 * _randn(g, total + n, V)
        # the draft model's distribution: near the target's at the same place
        at = torch.cat([torch.arange(d) + sum(drafts[:i]) + i for i, d in enumerate(drafts)]).cuda() if total else \
            torch.zeros(0, dtype=torch.int64, device="cuda")
        q = torch.softmax(logits[at] + 0.7 * _randn(g, total, V), -1)
        s["p"] = torch.softmax(logits, -1)
        s["draft"] = (torch.multinomial(q, 1, generator=g).view(-1) if total else at).to(torch.int32)
        s["q"] = q if case["drafted_probs"] else None
        s["cu"] = _cu(drafts)
        s["n"], s["max_draft"] = n, max(drafts)
        s["u_accept"] = torch.rand(total, generator=g, device="cuda")
        s["u_sample"] = torch.rand(n, generator=g, device="cuda")
        return s
    dt = DTYPES[case["dtype"]]
    Hkv, dh = case["n_kv_heads"], case["head_dim"]
    along = _along(g, Hkv, dh)
    if op == "mass" or op == "evict":
        lens = _ints(case["lens"])
        n = sum(lens)
        H = case["n_heads"] if op == "mass" else 0
        # one buffer as a fused projection leaves it: a row's queries (where they are used), keys and values
        row = torch.empty((n, (H + 2 * Hkv) * dh), dtype=dt, device="cuda")
        if H:
            row[:, :H * dh] = _queries(g, n, H, dh, along, Hkv).view(n, -1)
        row[:, H * dh:(H + Hkv) * dh] = _keys(g, n, Hkv, dh, along).view(n, -1)
        row[:, (H + Hkv) * dh:] = _randn(g, n, Hkv * dh)
        s["q"], s["k"], s["v"] = row[:, :H * dh], row[:, H * dh:(H + Hkv) * dh], row[:, (H + Hkv) * dh:]
        s["cu"], s["max_len"], s["n"], s["n_seqs"] = _cu(lens), max(lens), n, len(lens)
        if op == "evict":
            # weights over five decades, a tenth of the tokens never attended to (equal weights: lowest index first)
            mass = torch.exp(2.0 * _randn(g, Hkv, n))
            s["mass"] = torch.where(torch.rand((Hkv, n), generator=g, device="cuda") < 0.1, 0.0, mass)
            s["pos"] = torch.cat([torch.arange(v, dtype=torch.int32) for v in lens]).cuda()
            _new_cache(s, dt, len(lens), case["budget"] + 3, Hkv, dh)
        return s
    H = case["n_heads"]
    if op == "step":
        lens, budget = _ints(case["lens"]), case["budget"]
        B, cap = len(lens), budget + 1
        s["kc"] = _keys(g, B * cap, Hkv, dh, along).to(dt).view(B, cap, Hkv, dh)
        s["vc"] = _randn(g, B, cap, Hkv, dh).to(dt)
        s["cmass"] = torch.exp(2.0 * _randn(g, B, Hkv, cap))
        # slots hold positions in no order: evicted ones were written over by later tokens
        order = torch.rand((B, Hkv, cap), generator=g, device="cuda").argsort(-1).argsort(-1)
        held = torch.tensor(lens, dtype=torch.int32, device="cuda")[:, None].repeat(1, Hkv)
        s["clen"] = held
        s["cpos"] = (2 * order).to(torch.int32)
        s["pos_new"] = torch.full((B,), 2 * cap, dtype=torch.int32, device="cuda")
        s["q"] = _queries(g, B, H, dh, along, Hkv).to(dt).view(B, -1)
        s["k_new"] = _keys(g, B, Hkv, dh, along).to(dt).view(B, -1)
        s["v_new"] = _randn(g, B, Hkv * dh).to(dt)
        # the state after the step goes to buffers of its own, so that the step can be taken back
        s["mass_out"], s["pos_out"], s["len_out"] = s["cmass"].clone(), s["cpos"].clone(), held.clone()
        return s
    rows, keys = _ints(case["rows"]), _ints(case["own"])
    N, C, P = sum(rows), sum(keys), case["n_prefix"]
    s["kp"] = _keys(g, P, Hkv, dh, along).to(dt).view(P, Hkv * dh)
    s["vp"] = _randn(g, P, Hkv * dh).to(dt)
    # each request's own keys lie anywhere in one buffer of cache rows, named by a list of rows
    s["k"] = _keys(g, C + 5, Hkv, dh, along).to(dt).view(C + 5, Hkv * dh)
    s["v"] = _randn(g, C + 5, Hkv * dh).to(dt)
    s["kv_idx"] = torch.randperm(C + 5, generator=g, device="cuda")[:C].to(torch.int32)
    s["cu_kv"], s["max_kv"] = _cu(keys), max(keys)
    s["cu_q"], s["max_q"], s["n"] = _cu(rows), max(rows), N
    s["q"] = _queries(g, N, H, dh, along, Hkv).to(dt).view(N, -1)
    return s


def _new_cache(s, dt, n_seqs, cap, Hkv, dh):
    s["kc"] = torch.zeros((n_seqs, cap, Hkv, dh), dtype=dt, device="cuda")
    s["vc"] = torch.zeros((n_seqs, cap, Hkv, dh), dtype=dt, device="cuda")
    s["cmass"] = torch.zeros((n_seqs, Hkv, cap), device="cuda")
    s["cpos"] = torch.full((n_seqs, Hkv, cap), -1, dtype=torch.int32, device="cuda")
    s["clen"] = torch.zeros((n_seqs, Hkv), dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    return (_OWN if own else _PLAIN)[state["op"]](state)


def _own_mass(s):
    from paper_2407_14057_b200 import binding as B
    H, Hkv, dh = s["n_heads"], s["n_kv_heads"], s["head_dim"]
    if "scratch" not in s:
        s["scratch"] = B.lazy_k_attention_mass_scratch(s["n_seqs"], s["n"], s["max_len"], H, Hkv, s["window"])
        s["out"] = torch.empty((Hkv, s["n"]), device="cuda")
    return B.lazy_k_attention_mass(s["q"], s["k"], s["cu"], s["max_len"], H, Hkv, dh, s["window"],
                                   scratch=s["scratch"], out=s["out"])


def _own_evict(s):
    from paper_2407_14057_b200 import binding as B
    if "scratch" not in s:
        s["scratch"] = B.lazy_k_evict_scratch(s["n_seqs"], s["n_kv_heads"], s["budget"])
    B.lazy_k_evict(s["k"], s["v"], s["pos"], s["mass"], s["cu"], s["max_len"], s["budget"], s["recent"], s["kc"],
                   s["vc"], s["cmass"], s["cpos"], s["clen"], scratch=s["scratch"])
    return {name: s[name] for name in ("kc", "vc", "cmass", "cpos", "clen")}


def _own_step(s):
    from paper_2407_14057_b200 import binding as B
    if "scratch" not in s:
        n, cap, Hkv, dh = s["kc"].shape
        s["scratch"] = B.lazy_k_evict_step_scratch(n, s["n_heads"], Hkv, dh, s["budget"])
        s["out"] = (torch.empty_like(s["q"]), torch.empty((n, Hkv), dtype=torch.int32, device="cuda"),
                    torch.empty((n, Hkv), dtype=torch.int32, device="cuda"))
    o, slot, gone = B.lazy_k_evict_step(s["q"], s["k_new"], s["v_new"], s["pos_new"], s["kc"], s["vc"], s["cmass"],
                                        s["cpos"], s["clen"], s["n_heads"], s["budget"], s["recent"],
                                        mass_out=s["mass_out"], pos_out=s["pos_out"], len_out=s["len_out"],
                                        scratch=s["scratch"], out=s["out"])
    return {"o": o, "slot": slot, "gone": gone, "kc": s["kc"], "vc": s["vc"], "mass": s["mass_out"],
            "pos": s["pos_out"], "len": s["len_out"]}


def _own_prefix(s):
    from paper_2407_14057_b200 import binding as B
    H, Hkv, dh = s["n_heads"], s["n_kv_heads"], s["head_dim"]
    if "scratch" not in s:
        s["scratch"] = B.lazy_k_attention_prefix_scratch(s["n"], s["cu_q"].numel() - 1, s["max_q"], s["n_prefix"],
                                                         s["max_kv"], H, Hkv, dh)
        s["out"] = torch.empty_like(s["q"])
    return B.lazy_k_attention_prefix(s["q"], s["cu_q"], s["max_q"], s["kp"], s["vp"], s["k"], s["v"], s["kv_idx"],
                                     s["cu_kv"], s["max_kv"], H, Hkv, dh, scratch=s["scratch"], out=s["out"])


def _own_verify(s):
    from paper_2407_14057_b200 import binding as B
    if "out" not in s:
        s["out"] = (torch.empty(s["n"], dtype=torch.int32, device="cuda"),
                    torch.empty((s["n"], s["max_draft"] + 1), dtype=torch.int32, device="cuda"))
    return B.lazy_k_verify(s["p"], s["draft"], s["cu"], s["max_draft"], s["u_accept"], s["u_sample"], q=s["q"],
                           out=s["out"])


_OWN = {"mass": _own_mass, "evict": _own_evict, "step": _own_step, "prefix": _own_prefix, "verify": _own_verify}


# ------------------------------------------------------------------------------------------ plain forms
def _plain_mass(s):
    """mass[g, j] = sum over the last `window` rows i >= j and the heads of group g of softmax_j(q_i . k_j / sqrt(dh))."""
    H, Hkv, dh, L = s["n_heads"], s["n_kv_heads"], s["head_dim"], s["max_len"]
    G, S, n, dev = H // Hkv, s["n_seqs"], s["n"], "cuda"
    W = min(L, s["window"] or L)
    lo, lens = s["cu"][:-1].long(), (s["cu"][1:] - s["cu"][:-1]).long()
    j = torch.arange(L, device=dev)
    i = lens[:, None] - W + torch.arange(W, device=dev)                       # row inside its sequence, < 0: none
    key_rows = (lo[:, None] + j).clamp(max=n - 1)
    q_rows = (lo[:, None] + i.clamp(min=0)).clamp(max=n - 1)
    q = s["q"][q_rows.view(-1)].float().view(S, W, Hkv, G, dh).permute(0, 2, 1, 3, 4).reshape(S, Hkv, W * G, dh)
    k = s["k"][key_rows.view(-1)].float().view(S, L, Hkv, dh).permute(0, 2, 3, 1)
    x = torch.matmul(q, k).mul_(1.0 / math.sqrt(dh)).view(S, Hkv, W, G, L)
    seen = (j <= i[:, :, None]) & (i >= 0)[:, :, None]                          # [S, W, L]
    x = x.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    m = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(torch.isfinite(m), m, 0.0)).exp_()
    total = x.sum(-1, keepdim=True)
    x = x.mul_(torch.where(total > 0, 1.0 / total, 0.0))
    x = x.sum((2, 3))                                                            # [S, Hkv, L]
    seq = torch.repeat_interleave(torch.arange(S, device=dev), lens, output_size=n)
    return x[seq, :, torch.arange(n, device=dev) - lo[seq]].t().contiguous()


def _plain_evict(s):
    """Per sequence and head: the newest `recent` slots and the heaviest others up to `budget`, in slot order."""
    cu, L, S, n = s["cu"].long(), s["max_len"], s["n_seqs"], s["n"]
    Hkv, dh, dev = s["n_kv_heads"], s["head_dim"], "cuda"
    lo, lens = cu[:-1], cu[1:] - cu[:-1]
    keep = lens.clamp(max=s["budget"])
    j = torch.arange(L, device=dev)
    rows = (lo[:, None] + j).clamp(max=n - 1)
    m = s["mass"][:, rows].transpose(0, 1)                                       # [S, Hkv, L]
    m = torch.where((j >= lens[:, None] - s["recent"])[:, None], math.inf, m)
    m = torch.where((j < lens[:, None])[:, None], m, -math.inf)
    order = torch.sort(m, dim=-1, descending=True, stable=True)[1]
    most = min(L, s["budget"])
    chosen = torch.where(torch.arange(most, device=dev) < keep[:, None, None], order[..., :most], L).sort(-1)[0]
    there = chosen < L
    row = (lo[:, None, None] + chosen).clamp(max=n - 1)                          # [S, Hkv, most]
    si, hi, ti = torch.nonzero(there, as_tuple=True)
    k, v = s["k"].unflatten(1, (Hkv, dh)), s["v"].unflatten(1, (Hkv, dh))
    r = row[si, hi, ti]
    s["kc"][si, ti, hi] = k[r, hi]
    s["vc"][si, ti, hi] = v[r, hi]
    s["cmass"][si, hi, ti] = s["mass"][hi, r]
    s["cpos"][si, hi, ti] = s["pos"][r]
    s["clen"].copy_(keep[:, None].expand(S, Hkv))
    return {name: s[name] for name in ("kc", "vc", "cmass", "cpos", "clen")}


def _softmax(x, seen):
    x = x.masked_fill(~seen, -math.inf)
    m = x.amax(-1, keepdim=True)
    e = (x - torch.where(torch.isfinite(m), m, 0.0)).exp()
    total = e.sum(-1, keepdim=True)
    return e * torch.where(total > 0, 1.0 / total, 0.0)


def _plain_step(s):
    B, cap, Hkv, dh = s["kc"].shape
    H, budget, dev = s["n_heads"], s["budget"], "cuda"
    G = H // Hkv
    at = torch.arange(cap, device=dev)
    held = s["clen"][..., None]                                                  # every head has its own length
    # the lightest slot that is not among the newest `recent` positions; the lowest of equal ones
    free = (at < held) & (s["cpos"] < s["pos_new"][:, None, None] - s["recent"])
    weight = torch.where(free, s["cmass"], math.inf)
    victim = torch.where(weight == weight.amin(-1, keepdim=True), at, cap).amin(-1)
    full = s["clen"] >= budget
    slot = torch.where(full, victim, s["clen"].long())
    gone = torch.where(full, s["cpos"].gather(-1, slot[..., None]).squeeze(-1), -1)
    bi, hi = torch.arange(B, device=dev)[:, None], torch.arange(Hkv, device=dev)[None]
    s["kc"][bi, slot, hi] = s["k_new"].view(B, Hkv, dh)
    s["vc"][bi, slot, hi] = s["v_new"].view(B, Hkv, dh)
    length = torch.where(full, s["clen"], s["clen"] + 1)
    there = at < length[..., None]                                               # [B, Hkv, cap]
    k, v = s["kc"].float().permute(0, 2, 3, 1), s["vc"].float().permute(0, 2, 1, 3)
    x = torch.matmul(s["q"].float().view(B, Hkv, G, dh), k) * (1.0 / math.sqrt(dh))
    w = _softmax(x, there[:, :, None])
    o = torch.matmul(w, torch.where(there[..., None], v, 0.0))
    before = s["cmass"].scatter(-1, slot[..., None], 0.0)
    s["mass_out"].copy_(torch.where(there, before + w.sum(2), s["mass_out"]))
    s["pos_out"].copy_(torch.where(there, s["cpos"].scatter(-1, slot[..., None], s["pos_new"][:, None, None].expand(
        B, Hkv, 1)), s["pos_out"]))
    s["len_out"].copy_(length)
    return {"o": o.reshape(B, H * dh).to(s["q"].dtype), "slot": slot.to(torch.int32), "gone": gone.to(torch.int32),
            "kc": s["kc"], "vc": s["vc"], "mass": s["mass_out"], "pos": s["pos_out"], "len": s["len_out"]}


def _plain_prefix(s):
    H, Hkv, dh, N, P, C = s["n_heads"], s["n_kv_heads"], s["head_dim"], s["n"], s["n_prefix"], s["max_kv"]
    G, dev = H // Hkv, "cuda"
    cu_q, cu_kv = s["cu_q"].long(), s["cu_kv"].long()
    n_rows, n_own = cu_q[1:] - cu_q[:-1], cu_kv[1:] - cu_kv[:-1]
    seq = torch.repeat_interleave(torch.arange(n_rows.numel(), device=dev), n_rows, output_size=N)
    vis = (n_own - n_rows + 1)[seq] + torch.arange(N, device=dev) - cu_q[seq]    # own keys that a row sees
    at = torch.arange(C, device=dev)
    own_rows = s["kv_idx"].long()[(cu_kv[seq][:, None] + at).clamp(max=max(s["kv_idx"].numel() - 1, 0))]
    q = s["q"].float().view(N, Hkv, G, dh) * (1.0 / math.sqrt(dh))
    k = s["k"].float().view(-1, Hkv, dh)[own_rows]                                # [N, C, Hkv, dh]
    v = s["v"].float().view(-1, Hkv, dh)[own_rows]
    x_own = torch.matmul(q, k.permute(0, 2, 3, 1))                               # [N, Hkv, G, C]
    kp, vp = s["kp"].float().view(P, Hkv, dh), s["vp"].float().view(P, Hkv, dh)
    qh = q.permute(1, 0, 2, 3).reshape(Hkv, N * G, dh)
    x_pre = torch.matmul(qh, kp.permute(1, 2, 0)).view(Hkv, N, G, P).transpose(0, 1)
    seen = torch.cat([torch.ones((N, P), dtype=torch.bool, device=dev), at < vis[:, None]], 1)
    w = _softmax(torch.cat([x_pre, x_own], -1), seen[:, None, None])
    o = torch.matmul(w[..., P:], v.permute(0, 2, 1, 3))
    w_pre = w[..., :P].transpose(0, 1).reshape(Hkv, N * G, P)
    o = o + torch.matmul(w_pre, vp.transpose(0, 1)).view(Hkv, N, G, dh).transpose(0, 1)
    return o.reshape(N, H * dh).to(s["q"].dtype)


def _plain_verify(s):
    """Draft t of a sequence is accepted iff u_t q(x_t) < p(x_t) and all before it were; the token behind the
    accepted ones comes from max(p - q, 0) after a rejection, from p behind the last draft: the first id whose
    running sum exceeds u times the total."""
    p, q, n, T, V, dev = s["p"], s["q"], s["n"], s["max_draft"], s["vocab"], "cuda"
    cu = s["cu"].long()
    lens = cu[1:] - cu[:-1]
    t = torch.arange(T, device=dev)
    there = t < lens[:, None]
    at = (cu[:-1, None] + t).clamp(max=max(int(s["draft"].numel()) - 1, 0))
    if s["draft"].numel():
        x = s["draft"].long()[at]
        px = p[at + torch.arange(n, device=dev)[:, None], x].double()
        qx = q[at, x].double() if q is not None else torch.ones_like(px)
        ok = there & (s["u_accept"][at].double() * qx < px)
    else:
        x, ok = torch.zeros((n, T), dtype=torch.int64, device=dev), there
    accepted = ok.long().cumprod(1).sum(1)
    row = cu[:-1] + torch.arange(n, device=dev) + accepted
    r = p[row].double()
    rejected = accepted < lens
    if s["draft"].numel():
        back = (cu[:-1] + accepted).clamp(max=s["draft"].numel() - 1)
        if q is not None:
            less = q[back].double()
        else:
            less = torch.zeros_like(r).scatter_(1, s["draft"].long()[back][:, None], math.inf)
        r = torch.where(rejected[:, None], (r - less).clamp(min=0.0), r)
        r = torch.where(r.sum(1, keepdim=True) > 0, r, p[row].double())
    run_sum = r.cumsum(1)
    bar = s["u_sample"].double()[:, None] * run_sum[:, -1:]
    token = (run_sum <= bar).sum(1).clamp(max=V - 1)
    tokens = torch.full((n, T + 1), -1, dtype=torch.int64, device=dev)
    tokens[:, :T] = torch.where(t < accepted[:, None], x, -1)
    tokens = tokens.scatter(1, accepted[:, None], token[:, None])
    return accepted.to(torch.int32), tokens.to(torch.int32)


_PLAIN = {"mass": _plain_mass, "evict": _plain_evict, "step": _plain_step, "prefix": _plain_prefix,
          "verify": _plain_verify}


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """What run() returns, from the definitions, one sequence and head at a time; None for whole numbers."""
    op = case["op"]
    if op == "verify":
        return None  # whole numbers throughout
    s = prepare(case, seed)
    if op == "evict":
        Hkv, dh = s["n_kv_heads"], s["head_dim"]
        out = {name: s[name].double() for name in ("kc", "vc", "cmass")}
        mass = s["mass"].cpu().tolist()
        a = 0
        for b, n in enumerate(_ints(case["lens"])):
            old = n - min(n, case["recent"])
            for h in range(Hkv):
                heavy = sorted(range(old), key=lambda i: (-mass[h][a + i], i))[:min(n, case["budget"]) - (n - old)]
                at = torch.tensor(sorted(heavy) + list(range(old, n)), dtype=torch.int64, device="cuda") + a
                out["kc"][b, :len(at), h] = s["k"][at, h * dh:(h + 1) * dh].double()
                out["vc"][b, :len(at), h] = s["v"][at, h * dh:(h + 1) * dh].double()
                out["cmass"][b, h, :len(at)] = s["mass"][h, at].double()
            a += n
        return {**out, "cpos": None, "clen": None}
    H, Hkv, dh = s["n_heads"], s["n_kv_heads"], s["head_dim"]
    G, scale = H // Hkv, 1.0 / math.sqrt(dh)
    if op == "mass":
        out = torch.zeros((Hkv, s["n"]), dtype=torch.float64, device="cuda")
        a = 0
        for n in _ints(case["lens"]):
            first = n - min(n, case["window"] or n)
            for h in range(H):
                g = h // G
                for b in range(first, n, 2048):
                    e = min(n, b + 2048)
                    x = s["q"][a + b:a + e, h * dh:(h + 1) * dh].double() @ \
                        s["k"][a:a + e, g * dh:(g + 1) * dh].double().t() * scale
                    x = x.masked_fill(torch.ones((e - b, e), dtype=torch.bool, device="cuda").triu(b + 1), -math.inf)
                    out[g, a:a + e] += torch.softmax(x, -1).sum(0)
            a += n
        return out
    if op == "step":
        lens, budget = _ints(case["lens"]), case["budget"]
        o = torch.zeros((len(lens), H, dh), dtype=torch.float64, device="cuda")
        mass = s["mass_out"].double()
        for b, n in enumerate(lens):
            m = min(n + 1, budget)
            at = torch.full((Hkv,), n, dtype=torch.int64, device="cuda")
            if n >= budget:
                far = s["cpos"][b, :, :n] < s["pos_new"][b] - case["recent"]
                w = torch.where(far, s["cmass"][b, :, :n].double(), math.inf)
                at = (w <= w.amin(1, keepdim=True)).to(torch.uint8).argmax(1)
            heads = torch.arange(Hkv, device="cuda")
            k, v = s["kc"][b, :m].double(), s["vc"][b, :m].double()
            k[at, heads] = s["k_new"][b].double().view(Hkv, dh)
            v[at, heads] = s["v_new"][b].double().view(Hkv, dh)
            mass[b, heads, at] = 0.0
            w = torch.softmax(torch.einsum("hgd,mhd->hgm", s["q"][b].double().view(Hkv, G, dh), k) * scale, -1)
            o[b] = torch.einsum("hgm,mhd->hgd", w, v).reshape(H, dh)
            mass[b, :, :m] += w.sum(1)
        return {"o": o.view(len(lens), -1), "slot": None, "gone": None, "kc": None, "vc": None, "mass": mass,
                "pos": None, "len": None}
    o = torch.zeros((s["n"], H, dh), dtype=torch.float64, device="cuda")
    kp, vp = s["kp"].double().view(-1, Hkv, dh), s["vp"].double().view(-1, Hkv, dh)
    r = a = 0
    for t, c in zip(_ints(case["rows"]), _ints(case["own"])):
        idx = s["kv_idx"][a:a + c].long()
        k = torch.cat([kp, s["k"][idx].double().view(c, Hkv, dh)])
        v = torch.cat([vp, s["v"][idx].double().view(c, Hkv, dh)])
        x = torch.einsum("thgd,mhd->hgtm", s["q"][r:r + t].double().view(t, Hkv, G, dh), k) * scale
        hide = torch.ones((t, c), dtype=torch.bool, device="cuda").triu(c - t + 1)
        x[..., case["n_prefix"]:] = x[..., case["n_prefix"]:].masked_fill(hide, -math.inf)
        o[r:r + t] = torch.einsum("hgtm,mhd->thgd", torch.softmax(x, -1), v).reshape(t, H, dh)
        r, a = r + t, a + c
    return o.view(s["n"], -1)
