"""Refusals of the operators on paged caches and of the log probabilities: every check answers before the device is touched."""
import ctypes as C
import glob
import math
import os
import random

import pytest
import torch

from paper_2407_14057_b200 import binding, build

BADARG, CAPACITY = -1, -3
X = 1 << 30   # an aligned non-null address that no call below gets to use

PAGES = dict(k=X, v=X, page_stride=2048, slot_stride=128, head_stride=64, n_pages=4, page_size=16, table=X, table_pages=3, ld_table=3,
             len=X)
APPEND = dict(stream=None, dtype=0, q=X, ldq=256, k=X, v=X, ldkv=128, pos=X, rope=X, max_pos=64, g_q=X, g_k=X, eps=1e-6, cu_q=X,
              n_rows=2, n_seqs=1, pages=PAGES, H=4, Hkv=2, dh=64, q_out=X, ldq_out=256, k_out=X, ldk_out=128)
PAGED = dict(stream=None, dtype=0, q=X, ldq=256, cu_q=X, n_rows=2, n_seqs=1, max_q=2, pages=PAGES, max_kv=40, H=4, Hkv=2, dh=64,
             scratch=X, floats=1 << 24, o=X)
LOGPROBS = dict(stream=None, dtype=0, logits=X, ld=100, tokens=X, n_rows=2, vocab=100, n_top=5, logprob=X, entropy=X, rank=X, top_id=X,
                top_logprob=X)
HEADS = [dict(H=0), dict(H=4, Hkv=3), dict(Hkv=-1), dict(dh=48), dict(dh=0), dict(dh=288), dict(dtype=2), dict(dtype=-1)]
BAD_PAGES = [dict(k=None), dict(v=None), dict(table=None), dict(len=None), dict(k=X + 8), dict(v=X + 2), dict(page_stride=2047),
             dict(slot_stride=4), dict(head_stride=1), dict(page_stride=-8), dict(slot_stride=-128), dict(head_stride=-64),
             dict(n_pages=-1), dict(page_size=0), dict(page_size=-16), dict(table_pages=-1), dict(ld_table=2)]


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def refuse(fn, base, want, **change):
    args = dict(base, **change)
    assert set(args) == set(base)
    if isinstance(args.get("pages"), dict):
        args["pages"] = C.byref(binding.lazy_pages(*args["pages"].values()))
    assert fn(*args.values()) == want, change


def test_rope_table_refuses(lib):
    f = lib.lazy_k_rope_table
    for args in [(None, 4, 64, 1e4), (X + 4, 4, 64, 1e4), (X, -1, 64, 1e4), (X, 4, 63, 1e4), (X, 4, 0, 1e4), (X, 4, 64, 0.0),
                 (X, 4, 64, -1.0), (X, 4, 64, math.nan)]:
        assert f(None, *args) == BADARG, args
    assert f(None, X, 1 << 26, 128, 1e4) == CAPACITY
    assert f(None, None, 0, 64, 1e4) == 0


def test_append_refuses(lib):
    f = lib.lazy_k_paged_append
    pointers = [{k: None} for k in ("q", "k", "v", "pos", "rope", "q_out", "pages")]
    for change in HEADS + pointers + [dict(q=X + 8), dict(k=X + 2), dict(v=X + 8), dict(q_out=X + 8), dict(k_out=X + 8), dict(g_q=X + 8),
                                      dict(g_k=X + 4), dict(rope=X + 8), dict(ldq=255), dict(ldq=252), dict(ldkv=124), dict(ldkv=130),
                                      dict(ldq_out=248), dict(ldk_out=120), dict(n_rows=-1), dict(n_seqs=-1), dict(n_seqs=0),
                                      dict(max_pos=-1), dict(eps=-1.0), dict(eps=math.nan), dict(cu_q=None)]:
        refuse(f, APPEND, BADARG, **change)
    for change in BAD_PAGES:
        refuse(f, APPEND, BADARG, pages=dict(PAGES, **change))
    refuse(f, APPEND, CAPACITY, H=65536, Hkv=2)
    refuse(f, APPEND, CAPACITY, n_rows=(1 << 30) + 1)
    refuse(f, APPEND, CAPACITY, n_seqs=2 ** 31 - 1)
    refuse(f, APPEND, 0, n_rows=0, q=None, k=None, v=None, pages=None)


def test_attention_paged_refuses(lib):
    f = lib.lazy_k_attention_paged
    pointers = [{k: None} for k in ("q", "scratch", "o", "pages")]
    for change in HEADS + pointers + [dict(q=X + 8), dict(o=X + 8), dict(ldq=248), dict(ldq=257), dict(n_rows=-1), dict(n_seqs=-1),
                                      dict(n_seqs=0), dict(max_q=0), dict(max_q=-1), dict(max_kv=-1), dict(cu_q=None)]:
        refuse(f, PAGED, BADARG, **change)
    for change in BAD_PAGES:
        refuse(f, PAGED, BADARG, pages=dict(PAGES, **change))
    refuse(f, PAGED, CAPACITY, floats=0)
    refuse(f, PAGED, CAPACITY, n_rows=65536)
    refuse(f, PAGED, CAPACITY, n_seqs=65536)
    refuse(f, PAGED, CAPACITY, n_rows=65535, max_q=1 << 30, H=65535, Hkv=1, ldq=65535 * 64, floats=1 << 60)
    refuse(f, PAGED, 0, n_rows=0)
    g = lib.lazy_k_attention_paged_scratch_floats
    assert g(2, 1, 2, 40, 4, 3, 64) == 0 and g(-1, 1, 2, 40, 4, 2, 64) == 0 and g(2, 1, 2, -1, 4, 2, 64) == 0
    assert g(2, 1, 2, 40, 4, 2, 64) > 0


def test_logprobs_refuses(lib):
    f = lib.lazy_k_token_logprobs
    for change in [dict(logits=None), dict(tokens=None), dict(tokens=None, rank=None), dict(top_id=None), dict(top_logprob=None),
                   dict(logits=X + 1), dict(dtype=1, logits=X + 2), dict(dtype=3), dict(ld=99), dict(vocab=0), dict(n_rows=-1),
                   dict(n_top=-1), dict(n_top=65), dict(vocab=4), dict(ld=(1 << 30), vocab=-1)]:
        refuse(f, LOGPROBS, BADARG, **change)
    refuse(f, LOGPROBS, CAPACITY, ld=1 << 31, vocab=(1 << 30) + 1)
    refuse(f, LOGPROBS, CAPACITY, n_rows=2 ** 31 - 1)
    refuse(f, LOGPROBS, 0, n_rows=0, logits=None)


def _sizes(rng, top):
    return max(1, min(top, int(round(2 ** rng.uniform(0, math.log2(top))))))


def test_scratch_for_the_largest_serves_every_smaller_call(lib):
    """The size asked for a shape is at least that of every shape that is no larger in anything."""
    rng = random.Random(5)
    f = lib.lazy_k_attention_paged_scratch_floats
    for _ in range(20000):
        H, Hkv, dh = rng.choice([(32, 32, 128), (32, 8, 128), (8, 1, 128), (16, 4, 64), (12, 4, 128), (8, 2, 96), (4, 2, 256), (40, 1, 64),
                                 (6, 2, 32), (150, 1, 32), (200, 200, 64)])
        n_seqs, max_q, max_kv = _sizes(rng, 300), _sizes(rng, 20), _sizes(rng, 200000)
        rows = rng.randint(1, n_seqs * max_q)
        a = f(rows, n_seqs, max_q, max_kv, H, Hkv, dh)
        s, t = rng.randint(1, n_seqs), rng.randint(1, max_q)
        less = (rng.randint(1, min(rows, s * t)), s, t, rng.randint(1, max_kv), H, Hkv, dh)
        assert f(*less) <= a, (rows, n_seqs, max_q, max_kv, less)


@pytest.mark.parametrize("heads", [(32, 8, 128), (32, 32, 64), (8, 1, 128), (32, 8, 256)])
def test_scratch_of_a_mixed_batch(lib, heads):
    """A chunk among single tokens, a server's ordinary step: parts of keys that are not split need no place."""
    f = lib.lazy_k_attention_paged_scratch_floats
    for n_seqs, chunk in [(64, 512), (64, 4096), (256, 8192), (2000, 30000)]:
        assert f(n_seqs - 1 + chunk, n_seqs, chunk, 32768, *heads) * 4 < 16 << 20, (n_seqs, chunk)
        refuse(lib.lazy_k_attention_paged, PAGED, CAPACITY, n_rows=n_seqs - 1 + chunk, n_seqs=n_seqs, max_q=chunk, floats=0)


def test_scratch_of_mixed_batches_serves_smaller_calls(lib):
    """As above, where the largest call's keys are not split and a smaller one's are."""
    rng = random.Random(6)
    f = lib.lazy_k_attention_paged_scratch_floats
    for _ in range(20000):
        H, Hkv, dh = rng.choice([(32, 8, 128), (8, 1, 128), (16, 4, 64), (4, 2, 256), (40, 1, 64), (12, 2, 192)])
        n_seqs, max_q, max_kv = _sizes(rng, 3000), _sizes(rng, 20000), _sizes(rng, 200000)
        rows = min(65535, n_seqs - 1 + max_q)
        s, t, r, L = _sizes(rng, n_seqs), _sizes(rng, max_q), _sizes(rng, rows), _sizes(rng, max_kv)
        assert f(r, s, t, L, H, Hkv, dh) <= f(rows, n_seqs, max_q, max_kv, H, Hkv, dh), (rows, n_seqs, max_q, max_kv, r, s, t, L)


@pytest.mark.parametrize("heads", [(32, 8, 128), (4, 2, 256), (1, 1, 64), (65535, 1, 64), (65535, 65535, 32)])
def test_scratch_with_bounds_that_bind_nothing(lib, heads):
    """Any numbers serve as bounds, the largest among them."""
    f, most = lib.lazy_k_attention_paged_scratch_floats, 2 ** 31 - 1
    for n_rows, n_seqs, max_q in [(1, 1, 1), (4, 4, most), (65535, 65535, most), (most, most, most)]:
        want = f(min(n_rows, 65535), min(n_seqs, 65535), min(max_q, 65535), 1 << 30, *heads)
        for max_kv in (1 << 30, most - 300, most - 127, most - 126, most):
            assert f(n_rows, n_seqs, max_q, max_kv, *heads) == want < 1 << 24, (n_rows, n_seqs, max_q, max_kv)


def test_cluster_barriers_find_the_warp_together():
    """The .aligned forms are undefined for a warp whose lanes are apart: each stands right behind a barrier that joins them."""
    found = 0
    for path in sorted(glob.glob(os.path.join(os.path.dirname(build.__file__), "csrc", "*.cu*"))):
        with open(path) as f:
            code = [line.split("//")[0].strip() for line in f]
        for i, line in enumerate(code):
            if "barrier.cluster." in line and ".aligned" in line and "barrier.cluster.arrive" not in code[i - 1]:
                before = code[i - 1] if code[i - 1].startswith("__sync") else None
                if before is None:   # at the head of a function: its callers have the barrier
                    assert os.path.basename(path) == "tc_pair.cuh" and code[i - 1].endswith("{"), (path, i + 1)
                found += 1
    assert found >= 4


def test_rope_table_checks_its_output():
    t = torch.empty
    for out in (t(4, 32, 2), t(4, 32, 4)[..., :2], t(4, 16, 2), t((4, 32, 2), dtype=torch.float64)):
        with pytest.raises(ValueError):
            binding.lazy_k_rope_table(4, 64, 1e4, out=out)


def test_rope_table_refuses_another_devices_output(monkeypatch):
    class There:
        """As much of a tensor on device 1 as is looked at."""
        dtype, is_cuda = torch.float32, True
        numel, is_contiguous, get_device = (lambda self: 256), (lambda self: True), (lambda self: 1)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="current CUDA device"):
        binding.lazy_k_rope_table(4, 64, 1e4, out=There())
