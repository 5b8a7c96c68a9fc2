"""Operators on paged caches and the log probabilities against their statements in 64 bits, through the public binding.

Tolerances (u = 2^-24, half a step of fp32).
append: a rotated element is two products and a sum of normalised elements; the normalisation's factor has the error of a sum
of dh squares (halved by the root), of the reciprocal root (4 u) and of three products; the table's entries are off by u.  So an
element is off by E (|a c| + |b s|) with E = (dh / 2 + 16) u, plus half a step of its own type.
attention: a logit is off by (dh + 4) 2 u S, S the largest |logit| that the norms allow; a weight takes that twice, plus 2^-19 for
the exponentials and the sums of a part, plus n / 16 * 4 u for a sum that runs through n keys 16 at a time.  An output is off by that
times sum w |v|, plus half a step of its type.
logprobs: x - m is off by u |x - m|, its product with log2(e) and the exponential by 2 u |x - m| + 2^-22 relative, a sum of V
positive terms by (V / 512 + 24) u; the logarithm and the differences that follow by 3 u of what they give.
"""
import numpy as np
import pytest
import torch

import paged_reference as R
from helpers import to_np
from paper_2407_14057_b200 import binding as B
from paper_2407_14057_b200 import build

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24
HEADS = [(4, 4, 128, BF16), (8, 2, 128, BF16), (8, 1, 64, BF16), (6, 2, 64, BF16), (5, 1, 128, BF16), (2, 2, 96, BF16),
         (4, 2, 256, BF16), (4, 4, 64, F32), (6, 2, 32, F32), (8, 2, 32, BF16), (12, 2, 96, BF16), (4, 1, 160, F32), (20, 1, 128, BF16),
         (2, 1, 224, BF16), (3, 3, 192, F32)]
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


def i32(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def f64(t):
    return to_np(t).astype(np.float64)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def reported(where=None):
    with pytest.raises(B.LazyError) as e:
        B.lazy_device_status()
    if where is not None:
        assert B.lazy_status_detail()[0] == where
    return e.value.status


class Pool:
    """Pages of a batch of sequences of `lens` tokens, anywhere in a pool; layout: slots, heads (a head's slots side by side) or wide
    (pages and slots with gaps between them)."""

    def __init__(self, g, lens, page, Hkv, dh, dtype, layout="slots", fill=None):
        held = [-(-n // page) for n in lens]
        n = sum(held) + 2
        order = torch.randperm(n, generator=g).tolist()
        self.table = np.full((len(lens), max(held + [1]) + 1), -5, dtype=np.int32)   # entries that are not to be read
        at = 0
        for s, h in enumerate(held):
            self.table[s, :h] = order[at:at + h]
            at += h
        self.page, self.lens = page, lens
        pools = []
        for _ in range(2):
            data = randn(g, n, page, Hkv, dh, dtype=dtype) if fill is None else torch.full((n, page, Hkv, dh), fill, dtype=dtype)
            if layout == "slots":
                p = data.cuda()
            elif layout == "heads":
                p = data.transpose(1, 2).contiguous().cuda().transpose(1, 2)
            else:
                wide = torch.full((n, page + 1, Hkv + 2, dh + 32), float("nan"), dtype=dtype, device="cuda")
                p = wide[:, :page, 1:Hkv + 1, 16:16 + dh]
                p.copy_(data)
            pools.append(p)
        self.k, self.v = pools
        wide = torch.full((len(lens), self.table.shape[1] + 3), 1 << 30, dtype=torch.int32, device="cuda")
        wide[:, :self.table.shape[1]] = torch.from_numpy(self.table)
        self.d_table = wide[:, :self.table.shape[1]]
        self.d_len = i32(lens)

    def args(self):
        return self.k, self.v, self.d_table, self.d_len

    def rows(self, s, n):
        """K and V of a sequence's first n tokens, [n, Hkv, dh] in 64 bits."""
        p, t = R.slots(self.table[s], self.page, n)
        return f64(self.k)[p, t], f64(self.v)[p, t]


# ------------------------------------------------------------------------------------------- the table
@pytest.mark.parametrize("max_pos,dh,theta", [(1, 32, 1e4), (5000, 128, 1e4), (70000, 96, 5e5)])
def test_rope_table(max_pos, dh, theta):
    t = f64(B.lazy_k_rope_table(max_pos, dh, theta))
    angle = np.arange(max_pos)[:, None] * np.float64(np.float32(theta)) ** (-2.0 * np.arange(dh // 2) / dh)
    # the angle is off by a few 2^-53 of itself
    assert np.all(np.abs(t[..., 0] - np.cos(angle)) <= U + 2.0 ** -50 * angle)
    assert np.all(np.abs(t[..., 1] - np.sin(angle)) <= U + 2.0 ** -50 * angle)


# ------------------------------------------------------------------------------------------- append
def append_case(seed, past, rows, heads, page, layout, norms, fused):
    H, Hkv, dh, dtype = heads
    g, n = gen(seed), sum(rows)
    lens = [a + b for a, b in zip(past, rows)]
    pool = Pool(g, lens, page, Hkv, dh, dtype, layout)
    x = [randn(g, n, w * dh, dtype=dtype) for w in (H, Hkv, Hkv)]
    if fused:
        row = torch.full((n, (H + 2 * Hkv) * dh + 64), float("nan"), dtype=dtype)
        at, views = 32, []
        for t in x:
            row[:, at:at + t.shape[1]] = t
            views.append((at, t.shape[1]))
            at += t.shape[1]
        row = row.cuda()
        dev = [row[:, a:a + w] for a, w in views]
    else:
        dev = [t.cuda() for t in x]
    pos = np.concatenate([np.sort(torch.randperm(3 * b + 5, generator=g)[:b].numpy()) + 2 * a for a, b in zip(past, rows)] +
                         [np.zeros(0, np.int64)]).astype(np.int32)
    gains = [(1.0 + 0.3 * torch.randn(dh, generator=g)).to(dtype) if norms else None for _ in range(2)]
    return pool, x, dev, pos, gains


def check_append(pool, x, pos, gains, past, rows, heads, table, eps, q_out, before, k_out=None):
    H, Hkv, dh, dtype = heads
    E, hs = (dh / 2 + 16) * U, half_step(dtype)
    want_k, want_v = f64(before[0]), f64(before[1])
    tol_k = np.zeros_like(want_k)
    t, gq, gk = f64(table), *[None if z is None else f64(z) for z in gains]
    q, k, v = [f64(z) for z in x]
    got = f64(q_out)
    r = 0
    for s, (a, b) in enumerate(zip(past, rows)):
        p, slot = R.slots(pool.table[s], pool.page, a + b)
        for i in range(b):
            c, sn = t[pos[r], :, 0], t[pos[r], :, 1]
            y, size = R.rotate(q[r].reshape(H, dh), gq, eps, c, sn)
            err = np.abs(got[r].reshape(H, dh) - y)
            assert np.all(err <= E * size + hs * (np.abs(y) + E * size)), (s, i, err.max())
            y, size = R.rotate(k[r].reshape(Hkv, dh), gk, eps, c, sn)
            want_k[p[a + i], slot[a + i]] = y
            tol_k[p[a + i], slot[a + i]] = E * size + hs * (np.abs(y) + E * size)
            want_v[p[a + i], slot[a + i]] = v[r].reshape(Hkv, dh)
            if k_out is not None:
                assert np.array_equal(f64(k_out[r]).reshape(Hkv, dh), f64(pool.k[int(p[a + i]), int(slot[a + i])]))
            r += 1
    assert np.all(np.abs(f64(pool.k) - want_k) <= tol_k)      # and what was not written is what it was
    assert np.array_equal(f64(pool.v), want_v)


@pytest.mark.parametrize("heads", HEADS, ids=IDS)
@pytest.mark.parametrize("past,rows,page,layout,norms", [
    ([0], [1], 16, "slots", False), ([15, 16, 17], [1, 1, 1], 16, "heads", True), ([0, 40, 3], [33, 0, 18], 16, "slots", True),
    ([5, 0], [20, 7], 7, "wide", False), ([100], [3], 64, "heads", False), ([0, 0, 9, 0], [0, 2, 1, 0], 1, "slots", True)])
def test_append(heads, past, rows, page, layout, norms):
    H, Hkv, dh, dtype = heads
    pool, x, dev, pos, gains = append_case(3 * len(past) + past[0] + rows[0] + page, past, rows, heads, page, layout, norms,
                                           fused=layout != "heads")
    table = B.lazy_k_rope_table(400, dh, 1e4)
    n = sum(rows)
    before = pool.k.clone(), pool.v.clone()
    wide = torch.full((n, H * dh + 16), -3.0, dtype=dtype, device="cuda")
    k_out = torch.empty((n, Hkv * dh), dtype=dtype, device="cuda") if norms else None
    one_each = rows == [1] * len(rows)
    B.lazy_k_paged_append(*dev, i32(pos), table, *pool.args(), cu_q=None if one_each else cu(rows),
                          g_q=None if gains[0] is None else gains[0].cuda(), g_k=None if gains[1] is None else gains[1].cuda(), eps=1e-5,
                          q_out=wide[:, :H * dh], k_out=k_out)
    B.lazy_device_status()
    assert torch.all(wide[:, H * dh:] == -3.0)
    check_append(pool, x, pos, gains, past, rows, heads, table, 1e-5, wide[:, :H * dh], before, k_out)


def test_append_normalises_queries_or_keys_alone():
    heads, past, rows = (4, 2, 128, BF16), [3], [9]
    for only in (0, 1):
        pool, x, dev, pos, gains = append_case(only, past, rows, heads, 16, "slots", True, True)
        gains[1 - only] = None
        table = B.lazy_k_rope_table(400, 128, 1e4)
        before = pool.k.clone(), pool.v.clone()
        gq, gk = [None if z is None else z.cuda() for z in gains]
        out = B.lazy_k_paged_append(*dev, i32(pos), table, *pool.args(), cu_q=cu(rows), g_q=gq, g_k=gk, eps=1e-6)
        check_append(pool, x, pos, gains, past, rows, heads, table, 1e-6, out, before)


def test_append_in_place_and_the_contiguous_call():
    """q and k rotated where they stand: the bits of the out-of-place call, and those that lazy_k_rope_kv gives."""
    heads, past, rows = (4, 4, 128, BF16), [0, 7], [50, 21]
    pool, x, dev, pos, _ = append_case(9, past, rows, heads, 16, "slots", False, True)
    table = B.lazy_k_rope_table(400, 128, 1e4)
    out = B.lazy_k_paged_append(*dev, i32(pos), table, *pool.args(), cu_q=cu(rows))
    k1, v1 = pool.k.clone(), pool.v.clone()
    qkv = torch.cat(x, 1).cuda()
    q, k, v = qkv[:, :512], qkv[:, 512:1024], qkv[:, 1024:]
    got = B.lazy_k_paged_append(q, k, v, i32(pos), table, *pool.args(), cu_q=cu(rows), q_out=q, k_out=k)
    assert got.data_ptr() == q.data_ptr() and torch.equal(got, out)
    assert torch.equal(pool.k, k1) and torch.equal(pool.v, v1)
    ref = torch.cat(x, 1).cuda()
    kc, vc = B.lazy_k_rope_kv(ref, i32(pos), 4, 128, 400, 1e4)
    assert torch.equal(kc, k) and torch.equal(ref[:, :512], q) and torch.equal(vc, v)
    B.lazy_device_status()


def test_append_many_sequences():
    """More than one level of the search for a row's sequence, empty ones among them; padded rows behind the last."""
    heads = (2, 1, 64, BF16)
    g = gen(31)
    rows = [int(v) for v in torch.randint(0, 3, (3000,), generator=g)]
    past = [int(v) for v in torch.randint(0, 5, (3000,), generator=g)]
    pool, x, dev, pos, gains = append_case(32, past, rows, heads, 4, "slots", False, False)
    n, pad = sum(rows), 37
    table = B.lazy_k_rope_table(64, 64, 1e4)
    before = pool.k.clone(), pool.v.clone()
    dev = [torch.cat([t, torch.full((pad, t.shape[1]), float("nan"), dtype=BF16, device="cuda")]) for t in dev]
    out = torch.full((n + pad, 128), -2.0, dtype=BF16, device="cuda")
    padded = i32(np.concatenate([pos, np.full(pad, 1 << 30, np.int32)]))
    B.lazy_k_paged_append(*dev, padded, table, *pool.args(), cu_q=cu(rows), q_out=out)
    B.lazy_device_status()
    assert torch.all(out[n:] == -2.0)
    check_append(pool, x, pos, gains, past, rows, heads, table, 0.0, out[:n], before)


def test_append_without_a_row_for_a_length_of_zero():
    heads = (2, 1, 64, BF16)
    pool, x, dev, pos, gains = append_case(5, [3, 5, 0], [1, 1, 1], heads, 4, "slots", False, False)
    pool.d_len[1] = 0
    table = B.lazy_k_rope_table(64, 64, 1e4)
    before = pool.k.clone(), pool.v.clone()
    out = torch.full((3, 128), -2.0, dtype=BF16, device="cuda")
    B.lazy_k_paged_append(*dev, i32(pos), table, *pool.args(), q_out=out)
    B.lazy_device_status()
    assert torch.all(out[1] == -2.0) and not torch.any(torch.all(out[[0, 2]] == -2.0, 1))
    assert int((pool.v != before[1]).flatten(1).any(1).sum()) == 2


def test_append_reports():
    """What the tables get wrong is reported, and only that row or sequence is left out."""
    heads, past, rows = (2, 2, 64, BF16), [6, 2], [3, 4]

    def run(change, where, status, skipped):
        pool, x, dev, pos, gains = append_case(8, past, rows, heads, 4, "slots", False, False)
        table = B.lazy_k_rope_table(64, 64, 1e4)
        out = B.lazy_k_paged_append(*dev, i32(pos), table, *pool.args(), cu_q=cu(rows))
        want = out.clone(), pool.k.clone(), pool.v.clone()
        pool2, *_ = append_case(8, past, rows, heads, 4, "slots", False, False)
        a = dict(pos=i32(pos), cu=cu(rows), table=pool2.d_table, len=pool2.d_len)
        change(a)
        out = torch.full_like(out, -2.0)
        B.lazy_k_paged_append(*dev, a["pos"], table, pool2.k, pool2.v, a["table"], a["len"], cu_q=a["cu"], q_out=out)
        assert reported(where) == status
        for r in range(7):
            assert torch.all(out[r] == -2.0) if r in skipped else torch.equal(out[r], want[0][r]), r
        return want, pool2, pool

    def put(name, at, value):
        def f(a):
            a[name][at] = value
        return f

    run(put("pos", 4, 64), 10, -3, {4})
    run(put("pos", 4, -1), 10, -3, {4})
    run(put("len", 1, 3), 20, -1, {3, 4, 5, 6})       # fewer tokens than rows
    run(put("len", 0, 17), 20, -1, {0, 1, 2})         # more than the table's pages hold
    run(put("len", 0, -4), 20, -1, {0, 1, 2})
    run(put("cu", 2, 9), 20, -1, {3, 4, 5, 6})        # rows that are not there
    run(put("cu", 0, -2), 20, -1, {0, 1, 2})
    for bad in (-1, 1 << 20):
        want, got, plain = run(put("table", (1, 1), bad), 20, -1, set())   # the rows are rotated, their slots not written
        page = int(plain.table[1, 1])
        fresh, *_ = append_case(8, past, rows, heads, 4, "slots", False, False)
        assert torch.equal(got.k[page], fresh.k[page]) and torch.equal(got.v[page], fresh.v[page])
        others = [p for p in range(got.k.shape[0]) if p != page]
        assert torch.equal(got.k[others], want[1][others]) and torch.equal(got.v[others], want[2][others])


# ------------------------------------------------------------------------------------------- attention
def attention_case(seed, rows, lens, heads, page, layout, scale=1.0):
    H, Hkv, dh, dtype = heads
    g, n = gen(seed), sum(rows)
    pool = Pool(g, lens, page, Hkv, dh, dtype, layout)
    q = (scale * torch.randn((n, H * dh), generator=g)).to(dtype)
    wide = torch.full((n, H * dh + 48), float("nan"), dtype=dtype)
    wide[:, 16:16 + H * dh] = q
    return pool, q, wide.cuda()[:, 16:16 + H * dh]


def check_attention(pool, q, rows, lens, heads, got, skip=(), there=None):
    H, Hkv, dh, dtype = heads
    qn, o = f64(q).reshape(-1, H, dh), f64(got).reshape(-1, H, dh)
    r = 0
    for s, (t, n) in enumerate(zip(rows, lens)):
        if s in skip or t == 0:
            r += t
            continue
        k, v = pool.rows(s, n)
        S = np.sqrt((qn[r:r + t] ** 2).sum(-1).max() * (k ** 2).sum(-1).max()) * dh ** -0.5
        E = 2 * (dh + 4) * 2 * U * S + 2.0 ** -19 + n / 16 * 4 * U
        for i in range(t):
            see = n - t + i + 1
            for h in range(H):
                g = h // (H // Hkv)
                y, size = R.attention_row(qn[r, h], k[:see, g], v[:see, g], None if there is None else there[s][:see])
                err = np.abs(o[r, h] - y)
                assert np.all(err <= E * size + half_step(dtype) * (np.abs(y) + E * size) + 1e-30), (s, i, h, err.max())
            r += 1


LENGTHS = [([1], [1], 16), ([1, 1, 1], [15, 16, 17], 16), ([1], [700], 64), ([1, 1], [1300, 3], 16), ([3, 0, 5], [3, 40, 130], 16),
           ([2, 1, 8], [65, 64, 300], 7), ([17, 1], [33, 1], 32), ([1] * 5, [1, 513, 64, 2, 255], 128), ([40], [100], 1)]


@pytest.mark.parametrize("heads", HEADS, ids=IDS)
@pytest.mark.parametrize("rows,lens,page", LENGTHS)
def test_attention_paged(heads, rows, lens, page):
    H, Hkv, dh, dtype = heads
    layout = ("slots", "heads", "wide")[(len(rows) + page + H) % 3]
    pool, q, dq = attention_case(11 * len(rows) + lens[0] + page, rows, lens, heads, page, layout)
    pool.k[int(pool.table[0, 0]), min(lens[0], page):] = float("nan")        # slots behind the last token
    pool.v[int(pool.table[0, 0]), min(lens[0], page):] = float("nan")
    one_each = rows == [1] * len(rows)
    n, w = sum(rows), H * dh
    out = torch.full((n + 1, w), -3.0, dtype=dtype, device="cuda")
    scratch = torch.full((B.lazy_k_attention_paged_scratch(n, len(rows), max(rows), max(lens), H, Hkv, dh).numel() + 1,), float("nan"),
                         device="cuda")
    B.lazy_k_attention_paged(dq, *pool.args(), max(lens), cu_q=None if one_each else cu(rows), max_q=max(rows), scratch=scratch[1:],
                             out=out[:n])
    B.lazy_device_status()
    assert torch.all(out[n] == -3.0)
    check_attention(pool, q, rows, lens, heads, out[:n])
    # loose bounds, and scratch from the call itself
    again = B.lazy_k_attention_paged(dq, *pool.args(), 1 << 30, cu_q=cu(rows), max_q=max(rows) + 9)
    check_attention(pool, q, rows, lens, heads, again)
    B.lazy_device_status()


@pytest.mark.parametrize("heads", [(32, 8, 128, BF16), (8, 8, 64, BF16), (4, 2, 64, F32), (2, 2, 256, BF16)])
@pytest.mark.parametrize("rows,lens", [([1, 1, 1], [9000, 1, 4097]), ([4, 1], [6001, 2500]), ([1], [20000])])
def test_attention_paged_long(heads, rows, lens):
    pool, q, dq = attention_case(len(rows) + lens[0], rows, lens, heads, 16, "slots")
    got = B.lazy_k_attention_paged(dq, *pool.args(), max(lens), cu_q=cu(rows), max_q=max(rows))
    B.lazy_device_status()
    check_attention(pool, q, rows, lens, heads, got)


def test_attention_paged_many_sequences():
    """More (sequence, head) pairs than run at once, lengths from one on, and padded rows behind the last sequence."""
    heads, g = (4, 4, 128, BF16), gen(41)
    rows = [int(v) for v in torch.randint(0, 4, (220,), generator=g)]
    lens = [max(t, int(v)) for t, v in zip(rows, torch.randint(1, 90, (220,), generator=g))]
    pool, q, dq = attention_case(42, rows, lens, heads, 16, "heads")
    n = sum(rows)
    padded = torch.cat([dq, torch.full((50, 512), float("nan"), dtype=BF16, device="cuda")])
    out = torch.full((n + 50, 512), -3.0, dtype=BF16, device="cuda")
    B.lazy_k_attention_paged(padded, *pool.args(), 90, cu_q=cu(rows), max_q=3, out=out)
    B.lazy_device_status()
    assert torch.all(out[n:] == -3.0)
    check_attention(pool, q, rows, lens, heads, out[:n])


def test_attention_paged_without_a_row_for_a_length_of_zero():
    heads, lens = (8, 2, 128, BF16), [100, 7, 60]
    pool, q, dq = attention_case(3, [1] * 3, lens, heads, 16, "slots")
    pool.d_len[1] = 0
    out = torch.full((3, 1024), -3.0, dtype=BF16, device="cuda")
    B.lazy_k_attention_paged(dq, *pool.args(), 100, out=out)
    B.lazy_device_status()
    assert torch.all(out[1] == -3.0)
    check_attention(pool, q, [1] * 3, lens, heads, out, skip=(1,))


@pytest.mark.parametrize("heads", [(8, 2, 128, BF16), (4, 4, 64, F32), (2, 2, 256, BF16), (12, 2, 96, BF16)])
def test_attention_paged_leaves_others_alone(heads):
    """NaN and infinities in pages of other sequences, in free pages and behind the last token change nothing, bit for bit."""
    H, Hkv, dh, dtype = heads
    rows, lens = [2, 1, 3], [70, 333, 41]
    pool, q, dq = attention_case(4, rows, lens, heads, 16, "slots")
    want = B.lazy_k_attention_paged(dq, *pool.args(), 400, cu_q=cu(rows), max_q=3)
    mine = set(pool.table[1, :-(-333 // 16)].tolist())
    for p in range(pool.k.shape[0]):
        if p not in mine:
            pool.k[p], pool.v[p] = float("nan"), float("inf")
    last = int(pool.table[1, 333 // 16])
    pool.k[last, 333 % 16:], pool.v[last, 333 % 16:] = float("inf"), float("nan")
    got = B.lazy_k_attention_paged(dq, *pool.args(), 400, cu_q=cu(rows), max_q=3)
    B.lazy_device_status()
    assert torch.equal(got[2], want[2])


@pytest.mark.parametrize("page", [1, 5, 16, 48, 64, 100])
@pytest.mark.parametrize("heads", [(28, 4, 128, BF16), (40, 2, 64, BF16), (8, 8, 96, BF16), (6, 2, 192, BF16), (9, 3, 128, F32)])
def test_attention_paged_page_sizes_and_columns(heads, page):
    """Pages that end inside a group of keys or hold several, heads and rows that do not divide a tile of columns; both launch shapes."""
    rows, lens = [1, 9, 3, 2], [64, 128, 3, 1500]
    pool, q, dq = attention_case(page, rows, lens, heads, page, "wide" if page == 48 else "heads")
    for bound in (1500, 1 << 20):
        got = B.lazy_k_attention_paged(dq, *pool.args(), bound, cu_q=cu(rows), max_q=9)
        B.lazy_device_status()
        check_attention(pool, q, rows, lens, heads, got)


@pytest.mark.parametrize("heads", [(8, 2, 128, BF16), (4, 4, 64, F32)])
def test_attention_paged_large_logits(heads):
    """Logits that grow along the keys by far more than the exponential's range, and that are all the same."""
    H, Hkv, dh, dtype = heads
    for lens in ([300], [5000]):
        pool, q, dq = attention_case(2, [1], lens, heads, 16, "slots")
        p, t = R.slots(pool.table[0], 16, lens[0])
        ramp = torch.linspace(-40.0, 40.0, lens[0])[:, None, None].expand(-1, Hkv, dh).to(dtype).cuda()
        for k, want_row in ((ramp, None), (torch.zeros_like(ramp), None), (-ramp, None)):
            pool.k[p.tolist(), t.tolist()] = k
            dq.fill_(1.0)
            got = B.lazy_k_attention_paged(dq, *pool.args(), lens[0])
            check_attention(pool, torch.ones_like(q), [1], lens, heads, got)
    B.lazy_device_status()


def test_attention_paged_shares_pages():
    """Sequences that share the pages of a prefix, and a page named twice by one sequence."""
    heads = (8, 2, 128, BF16)
    pool, q, dq = attention_case(8, [1, 1, 1], [100, 90, 64], heads, 16, "slots")
    pool.table[1, :4] = pool.table[0, :4]
    pool.table[2, 3] = pool.table[2, 0]
    table = torch.from_numpy(pool.table).cuda()
    got = B.lazy_k_attention_paged(dq, pool.k, pool.v, table, pool.d_len, 100)
    B.lazy_device_status()
    check_attention(pool, q, [1, 1, 1], [100, 90, 64], heads, got)


@pytest.mark.parametrize("heads", [(8, 2, 128, BF16), (4, 4, 64, F32)])
def test_attention_paged_infinite_values(heads):
    """A token's infinite value reaches the rows that see it, and no row before."""
    H, Hkv, dh, dtype = heads
    rows, lens = [4], [50]
    pool, q, dq = attention_case(6, rows, lens, heads, 16, "slots")
    want = f64(B.lazy_k_attention_paged(dq, *pool.args(), 50, cu_q=cu(rows), max_q=4)).reshape(4, H, dh)
    p, t = R.slots(pool.table[0], 16, 50)
    pool.v[int(p[48]), int(t[48]), :, 5] = float("inf")
    pool.v[int(p[49]), int(t[49]), :, 7] = float("nan")
    got = f64(B.lazy_k_attention_paged(dq, *pool.args(), 50, cu_q=cu(rows), max_q=4)).reshape(4, H, dh)
    assert np.array_equal(got[:2], want[:2])
    assert np.all(got[2:, :, 5] == np.inf) and np.all(np.isnan(got[3, :, 7])) and np.all(np.isfinite(got[2, :, 7]))


def test_attention_paged_reports():
    heads, rows, lens = (8, 2, 128, BF16), [2, 1, 3], [70, 333, 41]
    for impl in (heads, (4, 4, 64, F32)):
        pool, q, dq = attention_case(7, rows, lens, impl, 16, "slots")

        def run(cu_q, table, length, max_q=3, max_kv=400):
            out = torch.full((6, impl[0] * impl[2]), -3.0, dtype=impl[3], device="cuda")
            B.lazy_k_attention_paged(dq, pool.k, pool.v, table, length, max_kv, cu_q=cu_q, max_q=max_q, out=out)
            assert reported(20) == -1
            return out

        for name, at, value, skip in [("len", 1, 0, (1,)), ("len", 1, -7, (1,)), ("len", 2, 2, (2,)), ("len", 0, 401, (0,)),
                                      ("cu", 3, 7, (2,)), ("cu", 0, -1, (0,))]:
            a = dict(len=pool.d_len.clone(), cu=cu(rows))
            a[name][at] = value
            out = run(a["cu"], pool.d_table, a["len"])
            check_attention(pool, q, rows, lens, impl, out, skip=skip)
            first = [0, 2, 3, 6][skip[0]]
            assert torch.all(out[first:first + rows[skip[0]]] == -3.0), name
        out = run(cu(rows), pool.d_table, pool.d_len, max_kv=332)          # longer than declared
        assert torch.all(out[2] == -3.0)
        check_attention(pool, q, rows, lens, impl, out, skip=(1,))
        out = run(cu(rows), pool.d_table, pool.d_len, max_q=2)             # more rows than declared
        assert torch.all(out[3:] == -3.0)
        check_attention(pool, q, rows, lens, impl, out, skip=(2,))
        out = run(cu(rows), pool.d_table[:, :20], pool.d_len)              # more tokens than the table's pages hold
        check_attention(pool, q, rows, lens, impl, out, skip=(1,))
        for bad in (-1, 1 << 24):
            table = pool.d_table.clone()
            table[1, 3] = bad
            out = run(cu(rows), table, pool.d_len)
            there = [np.ones(n, bool) for n in lens]
            there[1][48:64] = False
            check_attention(pool, q, rows, lens, impl, out, there=there)
        table = torch.full_like(pool.d_table, -1)
        assert torch.all(run(cu(rows), table, pool.d_len) == 0)            # nothing to see


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pages_behind_32_bits(dtype):
    """Pages that lie further than 2^31 elements into the pool, written and read."""
    heads = (4, 2, 64, dtype)
    H, Hkv, dh, _ = heads
    page, stride = 16, 1_200_000_000
    flat = torch.empty(2 * stride + 16 * 128, dtype=dtype, device="cuda")
    pools = [torch.as_strided(flat, (3, page, Hkv, dh), (stride, 128, dh, 1), at) for at in (0, 0)]
    other = torch.empty(2 * stride + 16 * 128, dtype=dtype, device="cuda")
    pools[1] = torch.as_strided(other, (3, page, Hkv, dh), (stride, 128, dh, 1))
    g = gen(3)
    table, lens = i32([[2, 1]]), i32([30])
    rows = 30
    q, k, v = [randn(g, rows, w * dh, dtype=dtype) for w in (H, Hkv, Hkv)]
    rope = torch.zeros((40, dh // 2, 2), device="cuda")
    rope[..., 0] = 1.0     # no rotation
    pos = i32(list(range(30)))
    out = B.lazy_k_paged_append(q.cuda(), k.cuda(), v.cuda(), pos, rope, *pools, table, lens, cu_q=cu([rows]))
    B.lazy_device_status()
    assert torch.equal(out.cpu(), q)
    got = torch.cat([pools[0][2], pools[0][1]])[:30].reshape(30, -1).cpu()
    assert torch.equal(got, k)

    class Plain:
        def rows(self, s, n):
            return f64(k).reshape(30, Hkv, dh)[:n], f64(v).reshape(30, Hkv, dh)[:n]

    o = B.lazy_k_attention_paged(out, *pools, table, lens, 30, cu_q=cu([rows]), max_q=rows)
    B.lazy_device_status()
    check_attention(Plain(), q, [rows], [30], heads, o)


# ------------------------------------------------------------------------------------------- log probabilities
def check_logprobs(x, tokens, n_top, got):
    xs = f64(x)
    V = xs.shape[1]
    logprob, entropy, rank, ids, top = [to_np(t) for t in got]
    for r in range(xs.shape[0]):
        lp, H, rk, want_ids, want_top = R.logprobs(xs[r], int(tokens[r]), n_top)
        assert rank[r] == rk and list(ids[r]) == want_ids, (r, rank[r], rk, list(ids[r]), want_ids)
        if np.isnan(H):
            assert np.isnan(entropy[r])
            assert tokens[r] < 0 and logprob[r] == 0 or np.isnan(logprob[r])
            assert np.all(np.isnan(top[r]))
            continue
        d = xs[r] - xs[r].max()
        D = -d[d > -100].min()
        rel = 2.0 ** -22 + 4 * U * D + (V / 512 + 24) * U             # of an exponential, of the sum
        lse = np.log(np.sum(np.exp(d)))
        tol = rel + 3 * U * (lse + 1)
        for g, w in [(logprob[r], lp)] + list(zip(top[r], want_top)):
            assert g == w or abs(g - w) <= tol + 3 * U * abs(w), (r, g, w, tol)
        moment = -np.sum(np.where(np.exp(d) > 0, np.exp(d) * np.maximum(d, -1e4), 0)) / np.sum(np.exp(d))
        assert abs(entropy[r] - H) <= tol + 2 * rel * moment + 3 * U * (H + moment), (r, entropy[r], H)


def logits_case(seed, n, V, dtype, offset=0):
    g = gen(seed)
    x = (3.0 * torch.randn((n, V), generator=g)).to(dtype)
    wide = torch.full((n, V + offset + 3), float("nan"), dtype=dtype)
    wide[:, offset:offset + V] = x
    tokens = torch.randint(0, V, (n,), generator=g).to(torch.int32)
    tokens[::3] = x[::3].float().argmax(1).to(torch.int32)
    return x, tokens, wide.cuda()[:, offset:offset + V]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 17, 100, 255, 1000, 4095, 4097, 8191, 20000, 32000, 50257])
def test_logprobs(V, dtype):
    for offset, n_top in [(0, 0), (1, 1), (3, 5), (8, 20), (5, 64)]:
        n_top = min(n_top, V)
        x, tokens, dx = logits_case(V + offset, 4, V, dtype, offset)
        got = B.lazy_k_token_logprobs(dx, tokens.cuda(), n_top)
        B.lazy_device_status()
        check_logprobs(x, tokens, n_top, got)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_logprobs_of_a_large_vocabulary(dtype):
    x, tokens, _ = logits_case(1, 3, 262147, dtype)
    got = B.lazy_k_token_logprobs(x.cuda(), tokens.cuda(), 20)
    B.lazy_device_status()
    check_logprobs(x, tokens, 20, got)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_logprobs_of_many_rows(dtype):
    x, tokens, dx = logits_case(2, 700, 1003, dtype, 5)
    got = B.lazy_k_token_logprobs(dx, tokens.cuda(), 7)
    B.lazy_device_status()
    check_logprobs(x, tokens, 7, got)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V,k", [(40, 20), (5000, 5), (32000, 64), (70001, 20)])
def test_logprobs_orders_equal_logits_by_id(V, k, dtype):
    """Rows of one value, of few values, ascending, descending, and zeros of both signs."""
    g = gen(V)
    rows = [torch.zeros(V), torch.randint(0, 3, (V,), generator=g).float(), torch.arange(V).float(), -torch.arange(V).float(),
            torch.where(torch.rand(V, generator=g) < 0.5, 0.0, -0.0), torch.randint(0, 2, (V,), generator=g) * 1e-30,
            torch.full((V,), -7.5), (torch.arange(V) // 100).float()]
    x = torch.stack([r.float() for r in rows]).to(dtype)
    tokens = torch.tensor([0, V - 1, V // 2, 3, V // 3, 11, V - 2, V // 2], dtype=torch.int32)
    got = B.lazy_k_token_logprobs(x.cuda(), tokens.cuda(), k)
    B.lazy_device_status()
    check_logprobs(x, tokens, k, got)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V,k", [(33, 12), (5000, 5), (32000, 20)])
def test_logprobs_of_masked_and_odd_rows(V, k, dtype):
    """Masks of -infinity and of the type's lowest value that leave many, few, one or no id; infinities, NaN, tokens that are none."""
    g, low = gen(V + 1), torch.finfo(dtype).min
    x = (3.0 * torch.randn((14, V), generator=g)).to(dtype)
    x[0, V // 2:] = -float("inf")
    x[1] = torch.where(torch.rand(V, generator=g) < 3 / V, x[1], -float("inf"))
    x[2], x[2, V - 1] = -float("inf"), 2.0
    x[3] = -float("inf")
    x[4, 5:] = low
    x[5] = low
    x[6], x[6, V // 2] = low, 1.0
    x[7, V // 3] = float("nan")
    x[8, V // 4] = float("inf")
    x[9] = float("nan")
    x[10] = torch.finfo(dtype).max
    x[11, 1], x[11, V - 2] = torch.finfo(dtype).max, low
    tokens = torch.tensor([1, 2, V - 1, 0, 1, 3, V // 2, V // 3, V // 4, 0, V - 1, 1, -1, -100], dtype=torch.int32)
    got = B.lazy_k_token_logprobs(x.cuda(), tokens.cuda(), k)
    B.lazy_device_status()
    check_logprobs(x, tokens, k, got)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,V,k", [(300, 9000, 64), (900, 4099, 20), (1, 131072, 64), (40, 70000, 33), (2000, 300, 3)])
def test_logprobs_shapes_of_a_launch(n, V, k, dtype):
    """Rows to a CTA, rows in turn, rows to clusters: a few of them by the formula, others against themselves alone (two sums that are
    off by (V / 512 + 24) u each: 3.4e-5 for the largest)."""
    x, tokens, dx = logits_case(n, n, V, dtype, 2)
    got = B.lazy_k_token_logprobs(dx, tokens.cuda(), k)
    B.lazy_device_status()
    some = sorted({0, 1 % n, n // 2, n - 1})
    check_logprobs(x[some], tokens[some], k, [t[some] for t in got])
    for a in range(0, n, max(1, n // 3)):
        one = B.lazy_k_token_logprobs(dx[a:a + 1], tokens[a:a + 1].cuda(), k)
        assert torch.equal(one[3][0], got[3][a]) and torch.equal(one[2][0], got[2][a])
        assert torch.allclose(one[0][0], got[0][a], rtol=1e-5, atol=4e-5) and torch.allclose(one[1][0], got[1][a], rtol=1e-5, atol=4e-5)


def test_logprobs_report_a_token_that_is_not_there():
    x, tokens, dx = logits_case(4, 5, 1000, F32)
    tokens[2] = 1000
    got = B.lazy_k_token_logprobs(dx, tokens.cuda(), 3)
    assert reported(21) == -1
    tokens[2] = -1
    check_logprobs(x, tokens, 3, got)


def test_logprobs_without_every_output():
    x, tokens, dx = logits_case(4, 5, 1000, F32)
    dx = dx.contiguous()
    d = tokens.cuda()
    want = B.lazy_k_token_logprobs(dx, d, 3)
    outs = [torch.full_like(t, 77) for t in want]
    L, s = B.lib(), torch.cuda.current_stream().cuda_stream
    for given in ([0], [1], [2], [3, 4], [0, 2]):
        p = [outs[i].data_ptr() if i in given else None for i in range(5)]
        tok = d.data_ptr() if 0 in given or 2 in given else None
        assert L.lazy_k_token_logprobs(s, B.LAZY_F32, dx.data_ptr(), 1000, tok, 5, 1000, 3 if 3 in given else 0, *p) == 0
    B.lazy_device_status()
    for a, b in zip(outs, want):
        assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------- as they are used
def test_calls_check_their_tensors():
    heads, rows, lens = (4, 2, 64, BF16), [2], [20]
    pool, q, dq = attention_case(1, rows, lens, heads, 16, "slots")
    c = cu(rows)
    for bad in (dict(q=dq[:, :128]), dict(q=dq.float()), dict(k=pool.k.float()), dict(k=pool.k[:, :, :1]), dict(k=pool.k.transpose(2, 3)),
                dict(k=pool.k[..., ::2]), dict(table=pool.d_table.long()), dict(table=pool.d_table[0]), dict(len=pool.d_len.long()),
                dict(len=i32([20, 3])), dict(c=cu([2, 0])), dict(c=None), dict(q=dq.cpu())):
        a = dict(q=dq, k=pool.k, v=pool.v, table=pool.d_table, len=pool.d_len, c=c)
        a.update(bad)
        with pytest.raises((ValueError, B.LazyError)):
            B.lazy_k_attention_paged(a["q"], a["k"], a["v"], a["table"], a["len"], 20, cu_q=a["c"], max_q=2,
                                     scratch=torch.empty(1 << 16, device="cuda"),
                                     out=torch.empty((2, 256), dtype=BF16, device="cuda"))
    with pytest.raises(B.LazyError):
        B.lazy_k_attention_paged(dq, *pool.args(), 20, cu_q=c, max_q=2, scratch=torch.empty(1, device="cuda"))
    x = torch.zeros((2, 50), device="cuda")
    for args in ((x.half(), i32([0, 1]), 1), (x, i32([0]), 1), (x, i32([0, 1]).long(), 1), (x.t(), i32([0] * 50), 1)):
        with pytest.raises(ValueError):
            B.lazy_k_token_logprobs(*args)
    for n_top in (51, 65, -1):
        with pytest.raises((ValueError, B.LazyError, RuntimeError)):
            B.lazy_k_token_logprobs(x, i32([0, 1]), n_top)


def test_no_rows():
    heads = (4, 2, 64, BF16)
    pool, q, dq = attention_case(1, [2], [20], heads, 16, "slots")
    assert B.lazy_k_attention_paged(dq[:0], *pool.args(), 20, cu_q=cu([0]), max_q=1).shape == (0, 256)
    k = torch.empty((0, 128), dtype=BF16, device="cuda")
    rope = B.lazy_k_rope_table(8, 64, 1e4)
    B.lazy_k_paged_append(dq[:0], k, k, i32([]), rope, *pool.args(), cu_q=cu([0]))
    out = B.lazy_k_token_logprobs(torch.empty((0, 100), device="cuda"), i32([]), 3)
    assert out[3].shape == (0, 3)
    B.lazy_device_status()


@pytest.mark.parametrize("heads", [(8, 2, 128, BF16), (4, 4, 64, F32)])
def test_captured_and_replayed_on_new_inputs(heads):
    """Append, attention and log probabilities in one graph: replays see new rows, lengths, tables and logits."""
    H, Hkv, dh, dtype = heads
    lens = [100, 37, 260, 1]
    pool, x, dev, pos, _ = append_case(12, [n - 1 for n in lens], [1] * 4, heads, 16, "slots", False, False)
    fresh, x2, dev2, pos2, _ = append_case(13, [n - 1 for n in [90, 260, 1, 77]], [1] * 4, heads, 16, "slots", False, False)
    rope = B.lazy_k_rope_table(1024, dh, 1e4)
    d_pos, table = i32(pos), torch.zeros((4, 18), dtype=torch.int32, device="cuda")
    k_pages, v_pages = torch.zeros((64, 16, Hkv, dh), dtype=dtype, device="cuda"), torch.zeros((64, 16, Hkv, dh), dtype=dtype, device="cuda")
    q_out, o = torch.empty_like(dev[0]), torch.empty_like(dev[0])
    scratch = B.lazy_k_attention_paged_scratch(4, 4, 1, 288, H, Hkv, dh)
    logits = torch.randn((4, 5000), generator=gen(1)).cuda()
    tokens, out = i32([1, 2, 3, 4]), [torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), i32([0] * 4),
                                      torch.empty((4, 3), dtype=torch.int32, device="cuda"), torch.empty((4, 3), device="cuda")]
    length = pool.d_len.clone()

    def load(p):
        k_pages[:p.k.shape[0]], v_pages[:p.v.shape[0]] = p.k, p.v
        table.zero_()
        table[:, :p.table.shape[1]] = p.d_table
        length.copy_(p.d_len)

    def step():
        B.lazy_k_paged_append(*dev, d_pos, rope, k_pages, v_pages, table, length, q_out=q_out)
        B.lazy_k_attention_paged(q_out, k_pages, v_pages, table, length, 288, scratch=scratch, out=o)
        B.lazy_k_token_logprobs(logits, tokens, 3, out=out)

    load(pool)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for p, z, ps, seed in ((pool, dev, pos, 1), (fresh, dev2, pos2, 2)):
        load(p)
        for a, b in zip(dev, [t.clone() for t in z]):
            a.copy_(b)
        d_pos.copy_(i32(ps))
        logits.copy_(torch.randn((4, 5000), generator=gen(seed)))
        graph.replay()
        got = [t.clone() for t in [q_out, o, k_pages, v_pages] + out]
        load(p)
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, [q_out, o, k_pages, v_pages] + out):
            assert torch.equal(a, b)
    B.lazy_device_status()
    del graph


def test_two_streams_at_once():
    heads, rows = (8, 2, 128, BF16), [1] * 6
    cases = [attention_case(20 + i, rows, [300 + 97 * i, 1, 50, 1000, 700, 64], heads, 16, "slots") for i in range(2)]
    logits = [logits_case(30 + i, 20, 32000, F32) for i in range(2)]
    want = [B.lazy_k_attention_paged(dq, *pool.args(), 1200).clone() for pool, _, dq in cases]
    want_lp = [B.lazy_k_token_logprobs(dx, t.cuda(), 5) for _, t, dx in logits]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                pool, _, dq = cases[i]
                got[i].append((B.lazy_k_attention_paged(dq, *pool.args(), 1200), B.lazy_k_token_logprobs(logits[i][2], logits[i][1].cuda(), 5)))
    torch.cuda.synchronize()
    for i in range(2):
        for o, lp in got[i]:
            assert torch.equal(o, want[i]) and all(torch.equal(a, b) for a, b in zip(lp, want_lp[i]))
    B.lazy_device_status()


def test_a_prompt_then_tokens_from_pages():
    """A prompt's rows cached in pages and attended there as lazy_k_attention attends them in place; then tokens one by one and drafts
    together, which see what they would have seen together; then logits, their log probabilities, and the drafts' check."""
    H, Hkv, dh, n, extra, V = 4, 4, 128, 150, 6, 1000
    g, d = gen(50), 512
    qkv = randn(g, n + extra, 3 * d, dtype=BF16).cuda()
    pos = torch.arange(0, 2 * (n + extra), 2, dtype=torch.int32, device="cuda")     # a pruned prompt's positions have gaps
    rope = B.lazy_k_rope_table(400, dh, 1e4)
    full = qkv.clone()
    kc, vc = B.lazy_k_rope_kv(full, pos, H, dh, 400, 1e4)
    want = B.lazy_k_attention(full, 3 * d, kc, vc, d, cu([n + extra]), n + extra, n + extra, H, dh)
    pages = [torch.zeros((20, 16, Hkv, dh), dtype=BF16, device="cuda") for _ in range(2)]
    table = torch.randperm(20, generator=g)[None].to(torch.int32).cuda()
    parts = [q[:n] for q in (qkv[:, :d], qkv[:, d:2 * d], qkv[:, 2 * d:])]
    got = []

    def feed(a, b):
        length = i32([b])
        q = B.lazy_k_paged_append(qkv[a:b, :d], qkv[a:b, d:2 * d], qkv[a:b, 2 * d:], pos[a:b], rope, *pages, table, length, cu_q=cu([b - a]))
        got.append(B.lazy_k_attention_paged(q, *pages, table, length, b, cu_q=cu([b - a]), max_q=b - a))

    feed(0, n)
    feed(n, n + 1)
    feed(n + 1, n + 2)
    feed(n + 2, n + extra)      # a token and three drafts
    o = torch.cat(got)
    assert len(parts) == 3 and o.shape == want.shape
    # both round an output once, and a weight to bf16 in the prompt's kernel: 2^-8 of sum w |v| each
    assert torch.max(torch.abs(o.float() - want.float())).item() <= 3 * 2.0 ** -8 * vc.abs().max().item()
    head = randn(g, V, d, dtype=BF16).cuda()
    logits = B.lazy_k_gemm(o[n + 2:].contiguous(), head)
    draft = logits.float().argmax(1)[:3].to(torch.int32)
    lp, entropy, rank, ids, top = B.lazy_k_token_logprobs(logits, torch.cat([draft, i32([-1])]), 4)
    check_logprobs(logits.cpu(), torch.cat([draft, i32([-1])]).cpu(), 4, (lp, entropy, rank, ids, top))
    assert torch.all(rank[:3] == 0) and torch.equal(ids[:3, 0], draft) and torch.equal(top[:3, 0], lp[:3])
    p = torch.softmax(logits.float(), -1)
    u = 0.999 * lp[:3].exp()                                                        # below the probability: accepted
    accepted, tokens = B.lazy_k_verify(p, draft, i32([0, 3]), 3, u, torch.tensor([0.0], device="cuda"))
    assert accepted.item() == 3 and torch.equal(tokens[0, :3], draft)
    B.lazy_device_status()


# ------------------------------------------------------------------------------------------- mixed batches
@pytest.mark.parametrize("heads", [(8, 2, 128, BF16), (4, 4, 64, BF16), (4, 2, 64, F32), (2, 1, 256, BF16)])
def test_attention_paged_of_a_mixed_batch(heads):
    """A long chunk behind cached tokens among single tokens, with scratch of the size asked for and no more."""
    H, Hkv, dh, dtype = heads
    rows = [1] * 20 + [1100, 0] + [1] * 9
    lens = [1 + 97 * i % 700 for i in range(20)] + [1500, 40] + [2000, 1, 16, 17, 300, 5, 64, 1024, 33]
    pool, q, dq = attention_case(60, rows, lens, heads, 16, "slots")
    floats = B.lazy_k_attention_paged_scratch(sum(rows), len(rows), 1100, 2000, H, Hkv, dh).numel()
    assert floats * 4 < 16 << 20
    scratch = torch.full((floats + 64,), float("nan"), device="cuda")
    scratch[floats:] = 7.0
    got = B.lazy_k_attention_paged(dq, *pool.args(), 2000, cu_q=cu(rows), max_q=1100, scratch=scratch[:floats])
    B.lazy_device_status()
    assert torch.all(scratch[floats:] == 7.0)
    check_attention(pool, q, rows, lens, heads, got)


@pytest.mark.parametrize("heads", [(1, 1, 32, BF16), (3, 3, 32, BF16), (1, 1, 96, BF16), (5, 5, 64, BF16), (2, 1, 128, BF16)])
@pytest.mark.parametrize("lens", [[700], [3000], [130, 1, 2000]])
def test_attention_paged_few_outputs_to_a_cluster(heads, lens):
    """A column or two: a few lanes of one warp write the cluster's parts, and the others wait; the same bits every time."""
    rows = [1] * len(lens)
    pool, q, dq = attention_case(lens[0] + heads[0], rows, lens, heads, 16, "slots")
    got = B.lazy_k_attention_paged(dq, *pool.args(), max(lens))
    B.lazy_device_status()
    check_attention(pool, q, rows, lens, heads, got)
    for _ in range(20):
        assert torch.equal(B.lazy_k_attention_paged(dq, *pool.args(), max(lens)), got)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V,k", [(9001, 1), (20011, 3), (50257, 33), (131075, 7)])
def test_logprobs_lists_of_odd_sizes_in_clusters(V, k, dtype):
    x, tokens, dx = logits_case(V, 3, V, dtype, 1)
    got = B.lazy_k_token_logprobs(dx, tokens.cuda(), k)
    B.lazy_device_status()
    check_logprobs(x, tokens, k, got)
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(B.lazy_k_token_logprobs(dx, tokens.cuda(), k), got))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [3, 640])
def test_logprobs_of_parts_that_end_anywhere_in_a_round(n, dtype):
    """The last 16 bytes of a row belong to any lane and load of a round, in a row to a CTA and in rows in turn, the rest of which is not
    there; among masks of -infinity and of the type's lowest value."""
    per = 16 // dtype.itemsize
    for V in [per * (128 * u + t) + per - 1 for u, t in [(0, 1), (0, 31), (0, 33), (1, 0), (3, 127), (5, 64), (7, 32), (7, 127), (8, 0), (8, 1)]]:
        x, tokens, dx = logits_case(V + n, n, V, dtype, V % 5)
        x[1, V // 3:], x[2, :V // 2] = -float("inf"), torch.finfo(dtype).min
        dx.copy_(x)
        got = B.lazy_k_token_logprobs(dx, tokens.cuda(), 4)
        B.lazy_device_status()
        check_logprobs(x[:3], tokens[:3], 4, [t[:3] for t in got])
        check_logprobs(x[-1:], tokens[-1:], 4, [t[-1:] for t in got])


@pytest.mark.parametrize("bounds", [[0, 4, 2], [3, 0, 7], [0, 7, 7, 5], [0, 0, 7, 9], [0, 7, -1, 7], [2, 1, 2, 7]])
def test_append_reports_boundaries_that_no_row_leads_to(bounds):
    """Boundaries that do not ascend or leave the rows are reported wherever they are; nothing outside the sequences' slots is written."""
    heads, n = (2, 2, 64, BF16), len(bounds) - 1
    pool, x, dev, pos, _ = append_case(8, [6] * n, [7] * n, heads, 4, "slots", False, False)
    dev = [t[:7] for t in dev]
    rope = B.lazy_k_rope_table(64, 64, 1e4)
    before = pool.k.clone()
    B.lazy_k_paged_append(*dev, i32(list(range(7))), rope, *pool.args(), cu_q=i32(bounds))
    assert reported(20) == -1
    free = [p for p in range(before.shape[0]) if p not in set(pool.table.ravel().tolist())]
    assert free and torch.equal(pool.k[free], before[free])


# ------------------------------------------------------------------------------------------- large and odd numbers
@pytest.mark.parametrize("offset", [9.9e6, -9.9e6, 1e7, -1e7, 1.1e7, -1.1e7, 3e7, -3e7, 2.0 ** 24 + 2, -1e12, 1e30])
@pytest.mark.parametrize("n,V", [(3, 300), (2, 40001), (600, 1003)])
def test_logprobs_of_rows_far_from_zero(n, V, offset):
    """Logits that differ by a few around a large number, either side of the size from which a row is summed from the differences: the
    rounding of the largest logit's product with log2(e), up to half a unit there, must not show."""
    g = gen(V)
    step = max(1.0, float(np.spacing(np.float32(abs(offset)))))
    level = torch.floor(13.0 * torch.rand((n, V), generator=g) ** 3)          # few large ones
    level[0] = 2.0 * (torch.arange(V) % 7 == 3)
    x = (offset + step * level.double()).float()
    x[1, V // 2:] = -float("inf")
    tokens = torch.randint(0, V // 2, (n,), generator=g).to(torch.int32)
    got = B.lazy_k_token_logprobs(x.cuda(), tokens.cuda(), 9)
    B.lazy_device_status()
    some = sorted({0, 1, n // 2, n - 1})
    check_logprobs(x[some], tokens[some], 9, [t[some] for t in got])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,V", [(2, 500), (3, 32001)])
def test_logprobs_tells_the_smallest_numbers_apart(n, V, dtype):
    """Numbers below the smallest normal one are neither zero nor equal."""
    g = gen(n)
    x = torch.zeros((n, V), dtype=dtype)
    raw = torch.int16 if dtype == BF16 else torch.int32
    x.view(raw).copy_(torch.randint(0, 100, (n, V), generator=g).to(raw))
    x[1] = -x[1]
    tokens = torch.randint(0, V, (n,), generator=g).to(torch.int32)
    got = B.lazy_k_token_logprobs(x.cuda(), tokens.cuda(), 20)
    B.lazy_device_status()
    check_logprobs(x, tokens, 20, got)


@pytest.mark.parametrize("heads", [(8, 2, 128, BF16), (12, 2, 96, BF16), (4, 4, 64, F32), (2, 2, 256, BF16)])
@pytest.mark.parametrize("length", [50, 3000])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_attention_paged_of_keys_that_are_not_finite(heads, length, bad):
    """A key's infinity makes its logit one: all of the row is NaN, or the key has no weight; a NaN is the whole row's.  Rows that do not
    see it have the bits that they have without."""
    H, Hkv, dh, dtype = heads
    rows, lens, at, col = [4], [length], length - 3, 5
    pool, q, dq = attention_case(length + H, rows, lens, heads, 16, "slots")
    want = f64(B.lazy_k_attention_paged(dq, *pool.args(), length, cu_q=cu(rows), max_q=4)).reshape(4, H, dh)
    k, v = pool.rows(0, length)
    p, t = R.slots(pool.table[0], 16, length)
    pool.k[int(p[at]), int(t[at]), :, col] = bad
    got = f64(B.lazy_k_attention_paged(dq, *pool.args(), length, cu_q=cu(rows), max_q=4)).reshape(4, H, dh)
    B.lazy_device_status()
    qn = f64(q).reshape(4, H, dh)
    assert np.array_equal(got[0], want[0])
    others = np.arange(length) != at
    S = np.sqrt((qn ** 2).sum(-1).max() * (k ** 2).sum(-1).max()) * dh ** -0.5
    E = 2 * (dh + 4) * 2 * U * S + 2.0 ** -19 + length / 16 * 4 * U
    seen = set()
    for i in range(1, 4):
        for h in range(H):
            if np.isnan(bad) or qn[i, h, col] * bad > 0:
                assert np.all(np.isnan(got[i, h])), (i, h)
                seen.add("nan")
            else:
                g, see = h // (H // Hkv), length - 4 + i + 1
                y, size = R.attention_row(qn[i, h], k[:see, g], v[:see, g], others[:see])
                assert np.all(np.abs(got[i, h] - y) <= E * size + half_step(dtype) * (np.abs(y) + E * size)), (i, h)
                seen.add("left out")
    assert seen == {"nan"} if np.isnan(bad) else seen == {"nan", "left out"}


@pytest.mark.parametrize("heads", [(8, 2, 128, BF16), (4, 4, 64, F32), (2, 2, 256, BF16)])
def test_attention_paged_of_a_row_without_a_finite_logit(heads):
    """Where every logit is -infinity no key has weight: zeros, as for a row that sees no page."""
    H, Hkv, dh, dtype = heads
    for length in (1, 40, 2500):
        pool, q, dq = attention_case(length, [1], [length], heads, 16, "slots")
        dq.fill_(1.0)
        pool.k[..., 3] = -float("inf")
        assert torch.all(B.lazy_k_attention_paged(dq, *pool.args(), length) == 0)
    B.lazy_device_status()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_paged_of_nearly_2_to_31_tokens(dtype):
    """A table that names one page 2046 times and another last, whose keys outweigh all before: the last range of keys ends behind 2^31 by
    the bounds.  Every token of the last page has the same weight and value: o is that value, off by the sums of weights alone, at most
    2^20 / 8 terms one after the other in either."""
    page, dh = 1 << 20, 32
    k, v = [torch.zeros((2, page, 1, dh), dtype=dtype, device="cuda") for _ in range(2)]
    k[1] = 4.0
    want = (1.0 + torch.arange(dh) / 16).to(dtype)
    v[1] = want.cuda()
    table = torch.zeros((1, 2048), dtype=torch.int32, device="cuda")
    table[0, 2046] = 1
    q = torch.ones((1, dh), dtype=dtype, device="cuda")
    got = B.lazy_k_attention_paged(q, k, v, table, i32([2047 * page]), 2 ** 31 - 1)
    B.lazy_device_status()
    # a token of the others weighs e^-22.6 as much: 2046 times that is 3.2e-7
    assert torch.all(torch.abs(got[0].cpu().double() - want.double()) <= (2.0 ** 17 * 2 * U + 1e-6 + half_step(dtype)) * want.double())
