"""Refusals of the operators on bounded and shared caches: every check answers before the device is touched."""
import ctypes as C
import math
import random

import pytest

from paper_2407_14057_b200 import binding, build

BADARG, CAPACITY = -1, -3
X = 1 << 30   # an aligned non-null address that no call below gets to use


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


MASS = dict(stream=None, dtype=0, q=X, ldq=256, k=X, ldkv=128, cu=X, n_seqs=1, max_len=8, n_total=8, H=4, Hkv=2,
            dh=64, window=0, scratch=X, floats=32, mass=X)
EVICT = dict(stream=None, dtype=0, k=X, v=X, ldkv=128, pos=X, mass=X, cu=X, n_seqs=1, max_len=8, n_total=8, Hkv=2,
             dh=64, budget=4, recent=2, scratch=X, ints=8, kc=X, vc=X, cmass=X, cpos=X, clen=X, cap=4)
STEP = dict(stream=None, dtype=0, q=X, ldq=256, k_new=X, v_new=X, ld_new=128, pos_new=X, kc=X, vc=X, cap=5, mass_in=X,
            mass_out=X, pos_in=X, pos_out=X, len_in=X, len_out=X, n_seqs=1, H=4, Hkv=2, dh=64, budget=4, recent=2,
            scratch=X, floats=1 << 20, o=X, slot=X, gone=X)
PREFIX = dict(stream=None, dtype=0, q=X, ldq=256, cu_q=X, n_rows=2, n_seqs=1, max_q=2, k_pre=X, v_pre=X, ld_pre=128,
              n_pre=3, k=X, v=X, ldkv=128, kv_rows=9, kv_idx=X, cu_kv=X, n_kv=2, max_kv=2, H=4, Hkv=2, dh=64,
              scratch=X, floats=1 << 20, o=X)
VERIFY = dict(stream=None, p=X, ldp=10, q=X, ldq=10, draft=X, cu=X, n_seqs=1, n_draft=1, max_draft=1, vocab=10,
              u_accept=X, u_sample=X, n_accept=X, tokens=X)


def refuse(fn, base, want, **change):
    args = dict(base, **change)
    assert set(args) == set(base)
    assert fn(*args.values()) == want, change


HEADS = [dict(H=0), dict(H=4, Hkv=3), dict(Hkv=-1), dict(dh=48), dict(dh=0), dict(dh=288), dict(dtype=2), dict(dtype=-1)]


def test_attention_mass_refuses(lib):
    f = lib.lazy_k_attention_mass
    for change in HEADS + [dict(q=None), dict(k=None), dict(cu=None), dict(scratch=None), dict(mass=None),
                           dict(q=X + 8), dict(k=X + 2), dict(ldq=248), dict(ldq=260), dict(ldkv=127), dict(ldkv=132),
                           dict(n_seqs=-1), dict(n_total=-1), dict(max_len=-1), dict(max_len=0), dict(window=-1)]:
        refuse(f, MASS, BADARG, **change)
    refuse(f, MASS, CAPACITY, floats=0)
    refuse(f, MASS, CAPACITY, n_seqs=65536)
    refuse(f, MASS, 0, n_seqs=0)
    refuse(f, MASS, 0, n_total=0, q=None, k=None, mass=None)
    assert lib.lazy_k_attention_mass_scratch_floats(1, 8, 8, 4, 3, 0) == 0


def test_evict_refuses(lib):
    f = lib.lazy_k_evict
    for change in [c for c in HEADS if "H" not in c] + \
            [dict(k=None), dict(v=None), dict(pos=None), dict(mass=None), dict(cu=None), dict(scratch=None), dict(kc=None),
             dict(vc=None), dict(cmass=None), dict(cpos=None), dict(clen=None), dict(k=X + 4), dict(vc=X + 8),
             dict(ldkv=120), dict(ldkv=129), dict(budget=0), dict(recent=-1), dict(recent=5), dict(cap=3),
             dict(n_seqs=-1), dict(max_len=-1), dict(max_len=0), dict(n_total=-1)]:
        refuse(f, EVICT, BADARG, **change)
    refuse(f, EVICT, CAPACITY, ints=7)
    refuse(f, EVICT, CAPACITY, n_seqs=65536, ints=1 << 40)
    refuse(f, EVICT, 0, n_seqs=0)
    assert lib.lazy_k_evict_scratch_ints(1, 2, 0) == 0


def test_evict_step_refuses(lib):
    f = lib.lazy_k_evict_step
    pointers = [dict([(k, None)]) for k in STEP if STEP[k] == X]
    for change in HEADS + pointers + [dict(q=X + 8), dict(k_new=X + 8), dict(kc=X + 8), dict(o=X + 8), dict(ldq=248),
                                      dict(ld_new=120), dict(ld_new=130), dict(budget=0), dict(recent=4), dict(recent=-1),
                                      dict(cap=3), dict(n_seqs=-1)]:
        refuse(f, STEP, BADARG, **change)
    refuse(f, STEP, CAPACITY, floats=0)
    refuse(f, STEP, 0, n_seqs=0)
    assert lib.lazy_k_evict_step_scratch_floats(1, 4, 2, 64, 0) == 0
    assert lib.lazy_k_evict_step_scratch_floats(1, 4, 3, 64, 4) == 0


def test_attention_prefix_refuses(lib):
    f = lib.lazy_k_attention_prefix
    pointers = [dict([(k, None)]) for k in PREFIX if PREFIX[k] == X]
    for change in HEADS + pointers + [dict(q=X + 8), dict(k_pre=X + 8), dict(v=X + 8), dict(o=X + 8), dict(ldq=248),
                                      dict(ld_pre=120), dict(ldkv=130), dict(n_rows=-1), dict(n_pre=-1), dict(n_kv=-1),
                                      dict(max_kv=-1), dict(kv_rows=-1), dict(kv_rows=0), dict(max_q=0), dict(n_seqs=0)]:
        refuse(f, PREFIX, BADARG, **change)
    refuse(f, PREFIX, CAPACITY, floats=0)
    refuse(f, PREFIX, CAPACITY, n_rows=65536)
    refuse(f, PREFIX, 0, n_rows=0)
    assert lib.lazy_k_attention_prefix_scratch_floats(2, 1, 2, 3, 2, 4, 3, 64) == 0
    assert lib.lazy_k_attention_prefix_scratch_floats(2, 1, 2, 2 ** 31 - 1, 2 ** 31 - 1, 4, 2, 64) == 0
    refuse(f, PREFIX, CAPACITY, n_pre=2 ** 31 - 1)


def test_verify_refuses(lib):
    f = lib.lazy_k_verify
    pointers = [dict([(k, None)]) for k in VERIFY if VERIFY[k] == X and k != "q"]
    for change in pointers + [dict(ldp=9), dict(ldq=9), dict(vocab=0), dict(n_seqs=-1), dict(n_draft=-1),
                              dict(max_draft=-1), dict(max_draft=0x7fffffff)]:
        refuse(f, VERIFY, BADARG, **change)
    refuse(f, VERIFY, CAPACITY, n_seqs=(1 << 24) + 1)
    refuse(f, VERIFY, 0, n_seqs=0)


def test_attention_mass_scratch_of_a_loose_bound(lib):
    """max_len beyond all rows asks for no more than their number does."""
    f = lib.lazy_k_attention_mass_scratch_floats
    for window in (0, 1, 20):
        for n_seqs, n_total in ((1, 8), (3, 5000), (2, 60000)):
            for heads in ((4, 2), (32, 8), (8, 8)):
                want = f(n_seqs, n_total, n_total, *heads, window)
                assert want > 0
                for bound in (n_total + 1, 10 ** 8, 2 ** 31 - 100, 2 ** 31 - 1):
                    assert f(n_seqs, n_total, bound, *heads, window) == want


def _sizes(rng, top):
    return max(1, min(top, int(round(2 ** rng.uniform(0, math.log2(top))))))


SCRATCH_HEADS = [(32, 32, 128), (32, 8, 128), (8, 1, 128), (16, 4, 64), (12, 4, 128), (8, 2, 96), (4, 2, 256), (40, 1, 64),
                 (6, 2, 32), (150, 1, 32), (200, 200, 64)]


def test_scratch_for_the_largest_serves_every_smaller_call(lib):
    """The size asked for a shape is at least that of every shape that is no larger in anything."""
    rng = random.Random(3)
    for _ in range(20000):
        H, Hkv, dh = rng.choice(SCRATCH_HEADS)
        n_seqs, longest, window = _sizes(rng, 300), _sizes(rng, 20000), rng.choice([0, 1, _sizes(rng, 400)])
        total = rng.randint(longest, n_seqs * longest)
        a = lib.lazy_k_attention_mass_scratch_floats(n_seqs, total, longest, H, Hkv, window)
        less = (rng.randint(1, n_seqs), rng.randint(1, total), rng.randint(1, longest), H, Hkv,
                rng.randint(1, window) if window else rng.choice([0, rng.randint(1, 400)]))
        assert lib.lazy_k_attention_mass_scratch_floats(*less) <= a, (n_seqs, total, longest, window, less)
        budget = _sizes(rng, 20000)
        a = lib.lazy_k_evict_step_scratch_floats(n_seqs, H, Hkv, dh, budget)
        less = (rng.randint(1, n_seqs), H, Hkv, dh, rng.randint(1, budget))
        assert lib.lazy_k_evict_step_scratch_floats(*less) <= a, (n_seqs, budget, less)
        assert lib.lazy_k_evict_scratch_ints(less[0], Hkv, less[4]) <= lib.lazy_k_evict_scratch_ints(n_seqs, Hkv, budget)
        max_q, max_kv, n_pre = _sizes(rng, 20), rng.choice([0, _sizes(rng, 3000)]), rng.choice([0, _sizes(rng, 30000)])
        rows = rng.randint(1, n_seqs * max_q)
        a = lib.lazy_k_attention_prefix_scratch_floats(rows, n_seqs, max_q, n_pre, max_kv, H, Hkv, dh)
        s, t = rng.randint(1, n_seqs), rng.randint(1, max_q)
        less = (rng.randint(1, min(rows, s * t)), s, t, rng.randint(0, n_pre), rng.randint(0, max_kv), H, Hkv, dh)
        assert lib.lazy_k_attention_prefix_scratch_floats(*less) <= a, (rows, n_seqs, max_q, n_pre, max_kv, less)


def test_scratch_of_a_batch_that_shrinks(lib):
    """One that fills a lane group of its own needs more parts than the next larger one: asked for either, it has room."""
    f = lib.lazy_k_attention_prefix_scratch_floats
    sizes = [f(n, n, 1, 16384, 500, 32, 8, 128) for n in range(1, 200)]
    assert sizes == sorted(sizes) and sizes[-1] < 4 * sizes[63]


def test_verify_refuses_more_rows_than_an_index_reaches(lib):
    """p has n_draft + n_seqs rows."""
    f = lib.lazy_k_verify
    for n_draft, n_seqs in ((2 ** 31 - 1, 1), (2 ** 31 - 1, 1 << 24), (2 ** 31 - 5, 6)):
        refuse(f, VERIFY, CAPACITY, n_draft=n_draft, n_seqs=n_seqs)
