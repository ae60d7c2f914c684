"""What the 8-bit cache's entry points refuse, at the C ABI and in the binding, before anything is launched (host only)."""
import ctypes as C
import sys

import pytest
import torch

from paper_2506_06266_amd import binding as cb

P = 0x1000


@pytest.fixture(scope="module")
def lib():
    return cb.load()


def cache(**kw):
    return cb.CacheStruct(**{**dict(n_blocks=9, Hkv=2, D=128, format=0, k=P, v=P, k_scale=P, v_scale=P), **kw})


def rows(**kw):
    return cb.CacheRows(**{**dict(T=6, B=3, max_blocks=4, dtype=cb.CART_BF16, k_row_stride=256, k_head_stride=128, v_row_stride=256,
                                  v_head_stride=128), **kw})


BAD_CACHES = [(dict(n_blocks=0), 2), (dict(Hkv=0), 2), (dict(D=0), 2), (dict(D=96), 3), (dict(D=256), 3), (dict(format=2), 3),
              (dict(n_blocks=2 ** 31 - 1, Hkv=2 ** 20), 2), (dict(k=None), 1), (dict(v=None), 1), (dict(k_scale=None), 1), (dict(v_scale=None), 1),
              (dict(k=P + 8), 6), (dict(v=P + 1), 6), (dict(k_scale=P + 2), 6)]
BAD_ROWS = [(dict(T=-1), 2), (dict(B=0), 2), (dict(max_blocks=0), 2), (dict(dtype=7), 3), (dict(k_row_stride=-256), 2),
            (dict(k_head_stride=4), 6), (dict(v_row_stride=257), 6), (dict(dtype=cb.CART_F32, v_head_stride=2), 6), (dict(v_row_stride=1 << 50), 2)]


@pytest.mark.parametrize("name", ["cart_cache_write", "cart_cache_read"])
def test_rows_are_refused(lib, name):
    f = getattr(lib, name)
    call = lambda c, r, k=P, v=P, cu=P, first=P, table=P: f(C.byref(c) if c else None, C.byref(r) if r else None, k, v, cu, first, table, None)
    for kw, status in BAD_CACHES:
        assert call(cache(**kw), rows()) == status, kw
    for kw, status in BAD_ROWS:
        assert call(cache(), rows(**kw)) == status, kw
    assert call(None, rows()) == 1 and call(cache(), None) == 1
    assert call(cache(), rows(), k=None) == 1 and call(cache(), rows(), v=None) == 1 and call(cache(), rows(), table=None) == 1
    assert call(cache(), rows(), k=P + 8) == 6 and call(cache(), rows(), table=P + 2) == 6 and call(cache(), rows(), cu=P + 1) == 6
    assert call(cache(), rows(T=7), cu=None) == 2               # 7 rows of 3 requests
    # more wavefronts than a launch counts
    assert call(cache(), rows(B=2 ** 30, T=1)) == 2 and call(cache(Hkv=2 ** 20), rows(B=2 ** 10 + 1, T=1)) == 2
    if name == "cart_cache_read":
        for kw in (dict(k_row_stride=0), dict(k_head_stride=0), dict(v_row_stride=0), dict(v_head_stride=0)):
            assert call(cache(), rows(**kw)) == 2, kw
    # no row at all: nothing to launch, nothing to point to
    assert call(cache(), rows(T=0), k=None, v=None) == 0 and call(cache(), rows(T=0), k=None, v=None, cu=None, first=None, table=None) == 0


def test_decode_is_refused(lib):
    def desc(**kw):
        return cb.CacheDecodeDesc(**{**dict(B=3, Hq=8, n_shared=0, max_blocks=4, max_own_len=200, dtype=cb.CART_BF16, softmax_scale=0.0), **kw})

    def call(d, c=None, q=P, shared=None, table=P, cu=P, o=P, lse=P, ws=P, n=1 << 40):
        c = c or cache()
        return lib.cart_cache_decode(C.byref(d) if d else None, C.byref(c), q, shared, table, cu, o, lse, ws, n, None)

    for kw, status in BAD_CACHES:
        assert call(desc(), cache(**kw)) == status, kw
    for kw, status in [(dict(B=0), 2), (dict(Hq=0), 2), (dict(Hq=7), 2), (dict(Hq=66), 3), (dict(n_shared=-1), 2), (dict(n_shared=9), 2),
                       (dict(max_blocks=-1), 2), (dict(max_own_len=-1), 2), (dict(max_own_len=257), 2), (dict(dtype=cb.CART_F32), 3),
                       (dict(softmax_scale=-1.0), 2), (dict(softmax_scale=float("nan")), 2), (dict(softmax_scale=float("inf")), 2),
                       (dict(max_blocks=2 ** 31 - 1, max_own_len=2 ** 30 + 1), 2), (dict(n_shared=1), 1), (dict(B=2 ** 30 + 1), 2),
                       (dict(B=2 ** 30, Hq=8), 2)]:
        assert call(desc(**kw)) == status, kw
        assert lib.cart_cache_decode_workspace(C.byref(desc(**kw)), C.byref(cache()), None) == 0, kw
    assert call(None) == 1 and call(desc(), q=None) == 1 and call(desc(), o=None) == 1 and call(desc(), table=None) == 1 and call(desc(), cu=None) == 1
    assert call(desc(), q=P + 8) == 6 and call(desc(), o=P + 8) == 6 and call(desc(), ws=P + 8) == 6 and call(desc(), lse=P + 2) == 6
    seg = lambda blocks, p: (cb.CacheSegment * 1)(cb.CacheSegment(blocks, p))
    assert call(desc(n_shared=1), shared=seg(P, -1)) == 2 and call(desc(n_shared=1), shared=seg(P, 2 ** 30 + 1)) == 2
    assert call(desc(n_shared=1), shared=seg(None, 1)) == 1 and call(desc(n_shared=1), shared=seg(P + 2, 1)) == 6
    # a workspace that is too small, wherever one is needed
    big = desc(B=64, max_blocks=2048, max_own_len=131072)
    need = lib.cart_cache_decode_workspace(C.byref(big), C.byref(cache()), None)
    if need:
        assert call(big, n=need - 1) == 4 and call(big, ws=None, n=need) == 4


# ---- the binding --------------------------------------------------------------------------------
def tensors(n=5, Hkv=2, D=128, dtype=torch.float8_e4m3fn):
    z = torch.zeros(n, Hkv, 64, D, dtype=torch.uint8).view(dtype)
    return (z, z.clone(), torch.ones(n, Hkv), torch.ones(n, Hkv))


I32 = dict(dtype=torch.int32)
TABLE = torch.zeros(3, 2, **I32)
X, Q = torch.zeros(6, 2, 128, dtype=torch.bfloat16), torch.zeros(3, 4, 128, dtype=torch.bfloat16)
CU = torch.zeros(4, **I32)


def write(cache=None, k=X, v=X, table=TABLE, **kw):
    return cb.cart_cache_write(cache or tensors(), k, v, table, **kw)


def read(cache=None, k=X, v=X, table=TABLE, **kw):
    return cb.cart_cache_read(cache or tensors(), k, v, table, **kw)


def decode(cache=None, q=Q, shared=(), table=TABLE, cu=CU, n=100, **kw):
    return cb.cart_cache_decode(q, cache or tensors(), list(shared), table, cu, n, **kw)


def test_host_tensors_are_refused():
    for call in (write, read, decode):
        with pytest.raises(ValueError, match="device tensors"):
            call()


def test_caches_are_refused():
    k, v, ks, vs = tensors()
    for call in (write, read, decode):
        for bad in ((k, v, ks), None, 3, (k, v, ks, None), (k, v, ks, vs, vs), (k.view(torch.uint8), v.view(torch.uint8), ks, vs), (k.half(), v, ks, vs)):
            with pytest.raises((TypeError, ValueError)):
                call(cache=bad) if bad else (cb.cart_cache_write(bad, X, X, TABLE) if call is not decode else cb.cart_cache_decode(Q, bad, [], TABLE, CU, 100))
        for bad in ((k[0], v[0], ks, vs), (k[:, :, :32], v[:, :, :32], ks, vs), (k, v[:4], ks, vs), (k, v.view(torch.int8), ks, vs), (k, v, ks[:4], vs),
                    (k, v, ks.half(), vs), (k, v, ks, vs[:, :1])):
            with pytest.raises(ValueError, match="^(?!tensors handed)"):
                call(cache=bad)


@pytest.mark.parametrize("call", [write, read])
def test_rows_are_refused_by_the_binding(call):
    for kw in (dict(k=X[0]), dict(k=X[:, :1], v=X[:, :1]), dict(k=X[:, :, :64], v=X[:, :, :64]), dict(v=X[:5]), dict(v=X.float()), dict(table=TABLE[0])):
        with pytest.raises((ValueError, TypeError)):
            call(**kw)
    for kw in (dict(k=X.half(), v=X.half()), dict(k=None), dict(table=None), dict(first=[0, 0, 0])):
        with pytest.raises(TypeError):
            call(**kw)


def test_decode_arguments_are_refused_by_the_binding():
    seg = torch.zeros(2, **I32)
    for kw in (dict(q=Q[0]), dict(q=Q.half()), dict(shared=[seg]), dict(shared=[(seg,)]), dict(shared=[(None, 3)]), dict(n=2.5), dict(n="3"),
               dict(scale="1"), dict(table=TABLE[:2])):
        with pytest.raises((TypeError, ValueError)):
            decode(**kw)
    with pytest.raises(TypeError, match="list"):
        cb.cart_cache_decode(Q, tensors(), None, TABLE, CU, 100)


def test_refused_calls_keep_no_references():
    c = tensors()
    held = [*c, X, Q, TABLE, CU]
    before = [sys.getrefcount(t) for t in held]
    for _ in range(50):
        for call in (write, read, decode):
            with pytest.raises(ValueError):
                call(cache=c)
    assert [sys.getrefcount(t) for t in held] == before
