"""What is measured of the operators for serving from paged caches: their plain forms, the calls a program makes of the
library, and cases over the range in use.

  append    new rows' queries and keys rotated by their positions (each head normalised first, where the model does
            that), keys and values written to the pages of their sequences
  paged     attention of one or several new rows per sequence over a paged cache
  logprobs  log probabilities of given tokens, with the distribution's entropy, the token's rank and the top alternatives

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
        # one request's next token, 7B shape: the latency case of a decoder's layer
        dict(name="append_one_row", op="append", dtype="bf16", n_heads=32, n_kv_heads=32, head_dim=128, page=16,
             layout="slots", norms=False, past="1023", rows="1"),
        # a batch of requests, one token each, grouped heads, normalised heads
        dict(name="append_batch64_norms", op="append", dtype="bf16", n_heads=32, n_kv_heads=8, head_dim=128, page=16,
             layout="slots", norms=True, past=_text((97 * i * i) % 1500 for i in range(64)), rows=_text([1] * 64)),
        # a prompt of the mean length of the long-context suite, 7B shape
        dict(name="append_prompt_3376", op="append", dtype="bf16", n_heads=32, n_kv_heads=32, head_dim=128, page=16,
             layout="slots", norms=False, past="0", rows="3376"),
        # chunks of ragged prompts behind what is cached already, pages that hold a head's slots side by side
        dict(name="append_chunks_ragged", op="append", dtype="bf16", n_heads=32, n_kv_heads=8, head_dim=128, page=64,
             layout="heads", norms=True, past="0,4079,1,513,0", rows="4096,2585,777,1,1968"),
        # one request of 1024 tokens, 7B shape: the latency case
        dict(name="paged_one_1024", op="paged", dtype="bf16", n_heads=32, n_kv_heads=32, head_dim=128, page=16,
             layout="slots", rows="1", lens="1024"),
        # four requests with four drafted tokens each
        dict(name="paged_drafts4_ragged", op="paged", dtype="bf16", n_heads=32, n_kv_heads=8, head_dim=128, page=16,
             layout="slots", rows="5,5,3,5", lens="3376,1000,77,5"),
        # a ragged batch, one token each, page of 64 slots, a head's slots side by side
        dict(name="paged_batch32_ragged", op="paged", dtype="bf16", n_heads=32, n_kv_heads=8, head_dim=128, page=64,
             layout="heads", rows=_text([1] * 32), lens=_text([1 + (131 * i * i) % 4096 for i in range(32)])),
        # one request over a long context
        dict(name="paged_one_65536", op="paged", dtype="bf16", n_heads=32, n_kv_heads=8, head_dim=128, page=16,
             layout="slots", rows="1", lens="65536"),
        # a batch of long requests: the largest
        dict(name="paged_batch16_16k", op="paged", dtype="bf16", n_heads=32, n_kv_heads=8, head_dim=128, page=16,
             layout="slots", rows=_text([1] * 16), lens=_text([16384] * 8 + [16383, 9001, 16000, 12345, 14000, 16384, 7777, 16384])),
        # one row of logits and its five best alternatives: the latency case
        dict(name="logprobs_one_top5", op="logprobs", dtype="f32", vocab=32000, n=1, n_top=5),
        # a batch of requests over a large vocabulary
        dict(name="logprobs_batch64_top20", op="logprobs", dtype="bf16", vocab=128256, n=64, n_top=20),
        # every token of a prompt of the mean length of the long-context suite
        dict(name="logprobs_prompt_3376", op="logprobs", dtype="f32", vocab=32000, n=3376, n_top=5),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["append", "paged", "paged", "logprobs"])
    if op == "logprobs":
        vocab = _log(rng, 1000, 128256)
        n = _log(rng, 1, max(1, min(3376, 100_000_000 // vocab)))
        return dict(op=op, dtype=rng.choice(["f32", "bf16"]), vocab=vocab, n=n, n_top=rng.choice([0, 1, 5, 20, rng.randint(2, 32)]))
    f32 = rng.random() < 0.15
    if f32:
        H, Hkv, dh = rng.choice([(4, 4, 64), (8, 2, 64), (4, 2, 128), (6, 2, 32)])
    else:
        H, Hkv, dh = rng.choice([(32, 32, 128), (32, 8, 128), (32, 8, 128), (8, 1, 128), (16, 4, 64), (8, 8, 64),
                                 (12, 4, 128), (8, 2, 96), (28, 4, 128)])
    head = dict(op=op, dtype="f32" if f32 else "bf16", n_heads=H, n_kv_heads=Hkv, head_dim=dh,
                page=rng.choice([16, 16, 32, 64, 128, rng.randint(5, 100)]), layout=rng.choice(["slots", "heads"]))
    if op == "append":
        n = _log(rng, 1, 128)
        most = max(1, (9400 * 48 * 128) // (n * (H + 2 * Hkv) * dh * (2 if f32 else 1)))
        longest = 1 if rng.random() < 0.4 else _log(rng, 1, min(4096, most))
        past = [0 if rng.random() < 0.2 else _log(rng, 1, max(1, min(4096, 40_000 // n))) for _ in range(n)]
        return dict(head, norms=rng.random() < 0.5, past=_text(past),
                    rows=_text([longest] + [rng.randint(0, longest) if longest > 1 else 1 for _ in range(n - 1)]))
    n = _log(rng, 1, 64)
    t = rng.choice([1, 1, 1, rng.randint(2, 8)])
    rows = [rng.randint(1, t) for _ in range(n)]
    budget = 16 * 14000 * 8 * 128 // (8 if f32 else 1)
    longest = max(8, min(_log(rng, 8, 65536), budget // (n * Hkv * dh)))
    lens = [longest] + [longest if rng.random() < 0.3 else _log(rng, 1, longest) for _ in range(n - 1)]
    return dict(head, rows=_text(rows), lens=_text(max(a, b) for a, b in zip(lens, rows)))


# ------------------------------------------------------------------------------------------ work
def work(case):
    op = case["op"]
    eb = 2 if case["dtype"] == "bf16" else 4
    if op == "logprobs":
        n, V, k = case["n"], case["vocab"], case["n_top"]
        return {"bytes": n * (V * eb + 4.0 + 12.0 + 8.0 * k), "flops": 5.0 * n * V}
    H, Hkv, dh = case["n_heads"], case["n_kv_heads"], case["head_dim"]
    rows = _ints(case["rows"])
    if op == "append":
        n = sum(rows)
        return {"bytes": n * (2.0 * eb * dh * (H + 2 * Hkv) + 4),
                "flops": n * dh * (H + Hkv) * (7.0 if case["norms"] else 3.0)}
    lens = _ints(case["lens"])
    seen = sum(r * c - r * (r - 1) / 2.0 for r, c in zip(rows, lens))
    return {"bytes": 2.0 * eb * dh * Hkv * sum(lens) + 2.0 * eb * dh * H * sum(rows) + 4.0 * sum(-(-c // case["page"]) for c in lens),
            "flops": 4.0 * seen * H * dh}


# ------------------------------------------------------------------------------------------ inputs
EPS, THETA = 1e-6, 10000.0


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _i32(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def _cu(lens):
    return _i32(sum(lens[:i]) for i in range(len(lens) + 1))


def _pages(g, s, dt, lens, fill):
    """Pages of all sequences, anywhere in one pool of a few more, as [n_pages, page, n_kv_heads, head_dim]."""
    page, Hkv, dh = s["page"], s["n_kv_heads"], s["head_dim"]
    held = [-(-n // page) for n in lens]
    total, width = sum(held) + 3, max(held) + 2
    shape = (total, page, Hkv, dh) if s["layout"] == "slots" else (total, Hkv, page, dh)
    for name in ("k_pages", "v_pages"):
        pool = torch.empty(shape, dtype=dt, device="cuda")
        for a in range(0, total, 4096):
            pool[a:a + 4096] = _randn(g, *pool[a:a + 4096].shape) if fill else 0.0
        s[name] = pool if s["layout"] == "slots" else pool.transpose(1, 2)
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(held):
        table[i, :n] = order[at:at + n]
        at += n
    s["table"], s["kv_len"], s["max_kv"] = table, _i32(lens), max(lens)


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    dt = DTYPES[case["dtype"]]
    if case["op"] == "logprobs":
        n, V = case["n"], case["vocab"]
        # rows from flat to sure of themselves; the last ids of a padded vocabulary are never possible
        x = (1.0 + 3.0 * torch.rand((n, 1), generator=g, device="cuda")) * _randn(g, n, V)
        x[:, V - V // 200:] = -math.inf
        best = torch.randint(0, V - V // 200, (n,), generator=g, device="cuda")
        x[torch.arange(n, device="cuda"), best] += 12.0 * torch.rand(n, generator=g, device="cuda")
        other = torch.randint(0, V - V // 200, (n,), generator=g, device="cuda")
        s["tokens"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.7, best, other).to(torch.int32)
        s["logits"] = x.to(dt)
        return s
    H, Hkv, dh = case["n_heads"], case["n_kv_heads"], case["head_dim"]
    rows = _ints(case["rows"])
    n = sum(rows)
    # one token each: no table of lengths
    s["cu_q"], s["max_q"] = (None if rows == [1] * len(rows) else _cu(rows)), max(rows)
    s["row_lens"] = rows
    if case["op"] == "append":
        past = _ints(case["past"])
        lens = [a + b for a, b in zip(past, rows)]
        # one buffer as a fused projection leaves it
        row = torch.empty((n, (H + 2 * Hkv) * dh), dtype=dt, device="cuda")
        row[:] = _randn(g, n, (H + 2 * Hkv) * dh)
        s["q"], s["k"], s["v"] = row[:, :H * dh], row[:, H * dh:(H + Hkv) * dh], row[:, (H + Hkv) * dh:]
        # original positions of a pruned prompt's rows: ascending, with gaps
        s["pos"] = torch.cat([torch.arange(a, a + b, device="cuda") for a, b in zip(past, rows)]).mul(7).div(
            4, rounding_mode="floor").to(torch.int32)
        top = max(lens) * 7 // 4 + 1
        angle = torch.arange(top, dtype=torch.float64, device="cuda")[:, None] * \
            THETA ** (-2.0 / dh * torch.arange(dh // 2, dtype=torch.float64, device="cuda"))
        s["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
        s["g_q"] = (1.0 + 0.2 * _randn(g, dh)).to(dt) if case["norms"] else None
        s["g_k"] = (1.0 + 0.2 * _randn(g, dh)).to(dt) if case["norms"] else None
        _pages(g, s, dt, lens, fill=False)
        s["q_out"] = torch.empty((n, H * dh), dtype=dt, device="cuda")
        return s
    lens = _ints(case["lens"])
    _pages(g, s, dt, lens, fill=True)
    # heavy hitters: the queries of a key/value head share a direction, along which some keys lie far
    along = _randn(g, Hkv, dh)
    along = along / along.norm(dim=-1, keepdim=True)
    s["q"] = (_randn(g, n, H, dh) + along.repeat_interleave(H // Hkv, 0)).to(dt).view(n, H * dh)
    k = s["k_pages"]
    for a in range(0, k.shape[0], 4096):
        weight = torch.exp(_randn(g, *k[a:a + 4096].shape[:3], 1)).clamp(max=16.0)
        k[a:a + 4096] += (0.35 * math.sqrt(dh) * weight * along).to(dt)
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    return (_OWN if own else _PLAIN)[state["op"]](state)


def _own_append(s):
    from paper_2407_14057_b200 import binding as B
    B.lazy_k_paged_append(s["q"], s["k"], s["v"], s["pos"], s["rope"], s["k_pages"], s["v_pages"], s["table"], s["kv_len"],
                          cu_q=s["cu_q"], g_q=s["g_q"], g_k=s["g_k"], eps=EPS, q_out=s["q_out"])
    return s["q_out"], s["k_pages"], s["v_pages"]


def _own_paged(s):
    from paper_2407_14057_b200 import binding as B
    if "scratch" not in s:
        H, Hkv, dh = s["n_heads"], s["n_kv_heads"], s["head_dim"]
        s["scratch"] = B.lazy_k_attention_paged_scratch(s["q"].shape[0], s["kv_len"].numel(), s["max_q"], s["max_kv"], H, Hkv, dh)
        s["out"] = torch.empty_like(s["q"])
    return B.lazy_k_attention_paged(s["q"], s["k_pages"], s["v_pages"], s["table"], s["kv_len"], s["max_kv"], cu_q=s["cu_q"],
                                    max_q=s["max_q"], scratch=s["scratch"], out=s["out"])


def _own_logprobs(s):
    from paper_2407_14057_b200 import binding as B
    if "out" not in s:
        n, k = s["n"], s["n_top"]
        s["out"] = (torch.empty(n, device="cuda"), torch.empty(n, device="cuda"),
                    torch.empty(n, dtype=torch.int32, device="cuda"),
                    torch.empty((n, k), dtype=torch.int32, device="cuda"), torch.empty((n, k), device="cuda"))
    return B.lazy_k_token_logprobs(s["logits"], s["tokens"], s["n_top"], out=s["out"])


_OWN = {"append": _own_append, "paged": _own_paged, "logprobs": _own_logprobs}


# ------------------------------------------------------------------------------------------ plain forms
def _row_tables(s, n):
    """Sequence of every row, and the place in its sequence."""
    if s["cu_q"] is None:
        seq = torch.arange(n, device="cuda")
        return seq, s["kv_len"].long() - 1
    cu = s["cu_q"].long()
    count = cu[1:] - cu[:-1]
    seq = torch.repeat_interleave(torch.arange(count.numel(), device="cuda"), count, output_size=n)
    return seq, torch.arange(n, device="cuda") - cu[seq] + (s["kv_len"].long() - count)[seq]


def _rotated(x, gain, cs):
    """x [n, heads, dh]: each head normalised (where there is a gain), then pairs (i, i + dh / 2) rotated."""
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
    a, b = x.chunk(2, -1)
    c, d = cs[:, None, :, 0], cs[:, None, :, 1]
    return torch.cat([a * c - b * d, b * c + a * d], -1)


def _plain_append(s):
    H, Hkv, dh, page = s["n_heads"], s["n_kv_heads"], s["head_dim"], s["page"]
    n, dt = s["q"].shape[0], s["q"].dtype
    cs = s["rope"][s["pos"].long()]
    seq, slot = _row_tables(s, n)
    at = s["table"][seq, slot // page].long()
    s["k_pages"][at, slot % page] = _rotated(s["k"].unflatten(1, (Hkv, dh)), s["g_k"], cs).to(dt)
    s["v_pages"][at, slot % page] = s["v"].unflatten(1, (Hkv, dh))
    s["q_out"].copy_(_rotated(s["q"].unflatten(1, (H, dh)), s["g_q"], cs).reshape(n, H * dh))
    return s["q_out"], s["k_pages"], s["v_pages"]


def _plain_paged(s):
    H, Hkv, dh, page, L = s["n_heads"], s["n_kv_heads"], s["head_dim"], s["page"], s["max_kv"]
    n, G = s["q"].shape[0], H // Hkv
    seq, slot = _row_tables(s, n)
    j = torch.arange(L, device="cuda")
    o = torch.empty((n, Hkv, G, dh), device="cuda")
    # a sequence's rows side by side, a few sequences at a time
    T = s["max_q"]
    first = torch.tensor([sum(s["row_lens"][:i]) for i in range(len(s["row_lens"]))], device="cuda")
    count = torch.tensor(s["row_lens"], device="cuda")
    step = max(1, 2 ** 28 // (L * Hkv * max(dh, G * T)))
    for a in range(0, len(s["row_lens"]), step):
        b = min(len(s["row_lens"]), a + step)
        at = s["table"][a:b][:, j // page].clamp(min=0).long()
        k = s["k_pages"][at, j % page].float()                                       # [S, L, Hkv, dh]
        r = (first[a:b, None] + torch.arange(T, device="cuda")).clamp(max=n - 1)      # [S, T]
        there = torch.arange(T, device="cuda") < count[a:b, None]
        q = s["q"][r].float().view(b - a, T, Hkv, G, dh).permute(0, 2, 1, 3, 4).reshape(b - a, Hkv, T * G, dh)
        x = torch.matmul(q, k.permute(0, 2, 3, 1)).mul_(1.0 / math.sqrt(dh)).view(b - a, Hkv, T, G, L)
        x = x.masked_fill_(~(j <= slot[r][..., None])[:, None, :, None], -math.inf)
        x = x.sub_(x.amax(-1, keepdim=True)).exp_()
        x = x.mul_(1.0 / x.sum(-1, keepdim=True)).view(b - a, Hkv, T * G, L)
        v = s["v_pages"][at, j % page].float().masked_fill_((j >= s["kv_len"][a:b, None])[..., None, None], 0.0)
        y = torch.matmul(x, v.permute(0, 2, 1, 3)).view(b - a, Hkv, T, G, dh).transpose(1, 2)
        o[r[there]] = y[there]
    return o.view(n, H * dh).to(s["q"].dtype)


def _plain_logprobs(s):
    x, t, k = s["logits"].float(), s["tokens"].long(), s["n_top"]
    m = x.amax(1, keepdim=True)
    e = (x - m).exp()
    total = e.sum(1, keepdim=True)
    lse = m + total.log()
    given = x.gather(1, t[:, None])
    p = e / total
    entropy = -torch.where(p > 0, p * (x - lse), 0.0).sum(1)
    ids = torch.arange(x.shape[1], device="cuda")
    rank = ((x > given) | ((x == given) & (ids < t[:, None]))).sum(1)
    order = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :k]
    return ((given - lse).squeeze(1), entropy, rank.to(torch.int32), order.to(torch.int32), x.gather(1, order) - lse)


_PLAIN = {"append": _plain_append, "paged": _plain_paged, "logprobs": _plain_logprobs}


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """What run() returns, from the definitions, a sequence (or a few rows of logits) at a time; None for whole numbers."""
    s = prepare(case, seed)
    if case["op"] == "logprobs":
        n, k = case["n"], case["n_top"]
        logprob, entropy, top = [torch.empty(z, dtype=torch.float64, device="cuda") for z in ((n,), (n,), (n, k))]
        for a in range(0, n, 256):
            x = s["logits"][a:a + 256].double()
            lp = torch.log_softmax(x, 1)
            logprob[a:a + 256] = lp[torch.arange(len(x)), s["tokens"][a:a + 256].long()]
            entropy[a:a + 256] = torch.special.entr(lp.exp()).sum(1)
            top[a:a + 256] = lp.topk(k, 1)[0]
        return logprob, entropy, None, None, top
    H, Hkv, dh, page = case["n_heads"], case["n_kv_heads"], case["head_dim"], case["page"]
    rows = _ints(case["rows"])
    table = s["table"].cpu().tolist()
    if case["op"] == "append":
        out = [torch.empty((sum(rows), H, dh), dtype=torch.float64, device="cuda"), s["k_pages"].double(), s["v_pages"].double()]

        def turned(x, gain, cs):
            x = x.double()
            if gain is not None:
                x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * gain.double()
            z = torch.complex(x[..., :dh // 2], x[..., dh // 2:]) * torch.complex(cs[..., 0], cs[..., 1])[:, None]
            return torch.cat([z.real, z.imag], -1)

        a = 0
        for i, (old, new) in enumerate(zip(_ints(case["past"]), rows)):
            cs = s["rope"][s["pos"][a:a + new].long()].double()
            out[0][a:a + new] = turned(s["q"][a:a + new].view(new, H, dh), s["g_q"], cs)
            k = turned(s["k"][a:a + new].view(new, Hkv, dh), s["g_k"], cs)
            done = 0
            while done < new:
                p, at = divmod(old + done, page)
                m = min(page - at, new - done)
                out[1][table[i][p], at:at + m] = k[done:done + m]
                out[2][table[i][p], at:at + m] = s["v"][a + done:a + done + m].double().view(m, Hkv, dh)
                done += m
            a += new
        return out[0].view(-1, H * dh), out[1], out[2]
    o = torch.empty((sum(rows), H, dh), dtype=torch.float64, device="cuda")
    a = 0
    for i, (r, c) in enumerate(zip(rows, _ints(case["lens"]))):
        at = torch.tensor(table[i][:-(-c // page)], device="cuda")
        k = s["k_pages"][at].flatten(0, 1)[:c].double()
        v = s["v_pages"][at].flatten(0, 1)[:c].double()
        q = s["q"][a:a + r].double().view(r, Hkv, H // Hkv, dh)
        x = torch.einsum("thgd,jhd->thgj", q, k) / math.sqrt(dh)
        for t in range(r):
            x[t, :, :, c - r + t + 1:] = -math.inf
        o[a:a + r] = torch.einsum("thgj,jhd->thgd", torch.softmax(x, -1), v).reshape(r, H, dh)
        a += r
    return o.view(-1, H * dh)
