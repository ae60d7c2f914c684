"""How a decode step over the 8-bit cache is cut, and that it fits the workspace (host only; the planner is called directly, a call
to an entry point would need a GPU)."""
import ctypes as C
import math
import random

import pytest

from paper_2506_06266_amd import binding as cb


class _Plan(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("n_rb", "n_parts", "n_ranges", "n_cuts", "cut")] + [(n, C.c_long) for n in ("n_shared_wg", "n_wg", "slots")]


NAME = "_ZN4cart17cache_decode_planERK22cart_cache_decode_descRK10cart_cachePK18cart_cache_segment"


def arguments(B, Hq, Hkv, D, own, segs):
    desc = cb.CacheDecodeDesc(B=B, Hq=Hq, n_shared=len(segs), max_blocks=-(-own // 64), max_own_len=own, dtype=cb.CART_BF16, softmax_scale=0.0)
    cache = cb.CacheStruct(n_blocks=9, Hkv=Hkv, D=D, format=0)
    return desc, cache, (cb.CacheSegment * max(len(segs), 1))(*[cb.CacheSegment(0x1000, p) for p in segs])


def plan(*sizes):
    f = C.CDLL(cb.LIB_PATH)[NAME]
    f.restype = _Plan
    desc, cache, segs = arguments(*sizes)
    return f(C.byref(desc), C.byref(cache), segs)


def workspace(*sizes):
    desc, cache, segs = arguments(*sizes)
    return cb.load().cart_cache_decode_workspace(C.byref(desc), C.byref(cache), segs)


def drawn(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    Hq, Hkv = rng.choice([(32, 8), (24, 8), (8, 2), (4, 1), (16, 16), (28, 4), (32, 1), (34, 2), (64, 8), (1, 1)])
    own = rng.choice([0, log(1, 200), log(1, 200000)])
    segs = [rng.choice([0, log(1, 300), log(1, 100000)]) for _ in range(rng.choice([0, 1, 1, 2, 8]))]
    return log(1, 4096), Hq, Hkv, rng.choice([64, 128]), own, segs


@pytest.mark.parametrize("seed", range(4))
def test_every_key_has_its_place(seed):
    rng = random.Random(seed)
    forms = set()
    for _ in range(2000):
        B, Hq, Hkv, D, own, segs = sizes = drawn(rng)
        p, steps = plan(*sizes), sum(-(-s // 32) for s in segs)
        every = steps + -(-own // 32)
        row = Hq * (4 * D + 12)
        if p.n_cuts:
            assert (p.n_cuts - 1) * p.cut < max(every, 1) <= p.n_cuts * p.cut and p.n_wg == B * Hkv * p.n_cuts, sizes
            assert p.slots == (B * p.n_cuts if p.n_cuts > 1 else 0), sizes
        else:
            per = 32 if B * (Hq // Hkv) > 16 else 16
            assert Hq // Hkv <= 16 and p.n_rb == -(-B * (Hq // Hkv) // per) and 1 <= p.n_parts <= -(-steps // 4), sizes
            assert p.n_shared_wg == p.n_rb * p.n_parts * Hkv and (p.n_ranges > 0) == (own > 0), sizes
            # the workgroups hold the ranges; range r and request b have slot n_parts B + r + b
            assert (p.n_wg - p.n_shared_wg) * 4 >= p.n_ranges * Hkv and p.slots >= p.n_parts * B + (p.n_ranges + B - 1 if own else 0), sizes
        assert p.slots * row <= workspace(*sizes), sizes
        forms.add((p.n_cuts > 0) + (p.n_cuts > 1))
    assert forms == {0, 1, 2}


@pytest.mark.parametrize("seed", range(4))
def test_a_larger_call_has_no_smaller_workspace(seed):
    rng = random.Random(100 + seed)
    for _ in range(2000):
        B, Hq, Hkv, D, own, segs = drawn(rng)
        less = (rng.randint(1, B), Hq, Hkv, D, rng.randint(0, own), [rng.randint(0, s) for s in segs][:rng.randint(0, len(segs))])
        assert workspace(*less) <= workspace(B, Hq, Hkv, D, own, segs), (less, (B, own, segs))
