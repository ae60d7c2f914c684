"""The 8-bit cache on the GPU against the fp64 oracle: writing, reading back, the decode step over it, and a run of them together.

Writing and reading are exact: magnitudes are compared as they are, scales are powers of two, and codes are rounded once, so the
codes' values and the scales have to be equal to the oracle's, bit for bit.

Decode, per element: the weights are rounded to bf16 once (2^-8 of each at most: size = sum_j w_j |v_j| is what that moves), the
output once (2^-8); a score is a sum of D products in fp32 (each of the D additions 2^-24 of sum_d |q_d k_d| = reach), its
exponent's arithmetic and the exponential another few 2^-24 of it and of 1, and the sums over the keys and their joins
in fp32 stay below 2^-18 for the lengths here.  So
  |o - o_ref| <= 2^-8 (1 + 2^-7) |o_ref| + (2^-8 (1 + 2^-7) + 2 d + 2^-18) size + 2^-104,
  |lse - lse_ref| <= d + 2^-20 (1 + |lse_ref|)
with d = (D + 16) 2^-24 (reach + 1).  (2^-104: a weight is at most 1, and one whose product with its value's scale is below
2^-126, the smallest normal number of fp32 and bf16, may be lost; 2^13 of them times a code below 2^9 are below that.)"""
import math

import numpy as np
import pytest
import torch

from oracle import cartridge_oracle as orc
from paper_2506_06266_amd import binding as cb

pytestmark = pytest.mark.gpu
TYPES = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}
FMT = list(TYPES)
STALE = 0x7F                # NaN in e4m3


def rand(*sizes, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*sizes, generator=g) * torch.exp2(spread * torch.randn(*sizes[:-1], 1, generator=g))


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


class Both:
    """A cache on the GPU and the oracle's copy; codes nobody wrote are NaN in e4m3, and their scales NaN."""

    def __init__(self, n_blocks, Hkv, D, fmt):
        self.fmt, self.sizes = fmt, (n_blocks, Hkv, D)
        self.ref = [[np.full((n_blocks, Hkv, 64, D), STALE, np.uint8), np.full((n_blocks, Hkv), np.nan)] for _ in range(2)]
        c = cb.cache_empty(n_blocks, Hkv, D, TYPES[fmt])
        for t in c[:2]:
            t.view(torch.uint8).fill_(STALE)
        for t in c[2:]:
            t.fill_(math.nan)
        self.gpu = c

    def write(self, k, v, table, first, lens, **kw):
        cu = offsets(lens)
        for ref, x in zip(self.ref, (k, v)):
            orc.cache_write(*ref, x[:cu[-1]].double().numpy(), table, first, cu, self.fmt)
        cb.cart_cache_write(self.gpu, k.cuda(), v.cuda(), i32(table), first=i32(first), cu_rows=i32(cu), **kw)

    def equal(self):
        means = orc.cache_meaning(self.fmt)
        for w in (0, 1):
            codes, scale = self.gpu[w].view(torch.uint8).cpu().numpy(), self.gpu[2 + w].cpu().double().numpy()
            assert np.array_equal(scale, self.ref[w][1], equal_nan=True)
            known = ~np.isnan(scale)[:, :, None, None]          # (a NaN scale's codes mean nothing)
            assert np.array_equal(np.where(known, means[codes], 0), np.where(known, means[self.ref[w][0]], 0), equal_nan=True)

    def decode_ref(self, q, shared, table, lens, scale=None):
        return orc.cache_decode(q.double().numpy(), *self.ref[0], *self.ref[1], shared, table, offsets(lens), self.fmt, scale)


def check_decode(o, lse, ref, D):
    o_ref, lse_ref, size, reach = ref
    o, lse = o.double().cpu().numpy().reshape(o_ref.shape), lse.double().cpu().numpy().reshape(lse_ref.shape)
    none, some = lse_ref == -np.inf, np.isfinite(lse_ref)
    assert np.array_equal(lse == -np.inf, none) and (o[none] == 0).all()
    assert np.array_equal(np.isnan(lse), np.isnan(lse_ref)) and np.array_equal(np.isnan(o), np.isnan(o_ref))
    d = (D + 16) * 2.0 ** -24 * (reach + 1)
    r = 2.0 ** -8 * (1 + 2.0 ** -7)
    assert (np.abs(o - o_ref)[some] <= (r * np.abs(o_ref) + (r + 2 * d[..., None] + 2.0 ** -18) * size + 2.0 ** -104)[some]).all()
    assert (np.abs(lse[some] - lse_ref[some]) <= (d + 2.0 ** -20 * (1 + np.abs(lse_ref)))[some]).all()


# ---- writing and reading ------------------------------------------------------------------------
LENGTHS = {
    "one token": ([0], [1]),
    "a block": ([0], [64]),
    "a block and one": ([0], [65]),
    "one short of a block": ([0], [63]),
    "steps": ([0, 63, 64, 5, 190], [1] * 5),
    "ragged": ([0, 63, 64, 127, 1, 130], [200, 1, 64, 66, 63, 129]),
    "empty ones": ([10, 0, 70, 0, 3], [0, 5, 0, 0, 61]),
    "nobody": ([4, 0], [0, 0]),
    "many": (list(range(0, 140, 1)), [(7 * i) % 90 for i in range(140)]),
}


def layout(first, lens, spare=2, seed=0):
    """A table over blocks in disorder: (table with -1 behind a request's blocks, blocks in the pool)."""
    need = [-(-(f + n) // 64) for f, n in zip(first, lens)]
    ids = np.random.RandomState(seed).permutation(sum(need) + spare)
    table, at = np.full((len(need), max(max(need), 1)), -1, np.int64), 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, sum(need) + spare


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("Hkv,D", [(8, 128), (1, 64), (3, 128)])
@pytest.mark.parametrize("name", LENGTHS)
def test_rows_in_and_out(name, Hkv, D, dtype, fmt):
    print("case rows", name, Hkv, D, dtype, fmt, flush=True)
    first, lens = LENGTHS[name]
    table, n_blocks = layout(first, lens, seed=len(name))
    c = Both(n_blocks, Hkv, D, fmt)
    T = sum(lens)
    # what stood before `first`: rows of other magnitudes, so that some scales grow
    before = rand(sum(first), Hkv, D, seed=1).to(dtype)
    c.write(before, before.flip(0), table, [0] * len(first), first)
    x = rand(T + 3, Hkv, D, seed=2, spread=3.0).to(dtype)
    y = rand(T + 3, Hkv, D, seed=3, spread=3.0).to(dtype)
    c.write(x, y, table, first, lens)
    torch.cuda.synchronize()
    c.equal()
    out = [torch.full((T + 3, Hkv, D), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    cb.cart_cache_read(c.gpu, *out, i32(table), first=i32(first), cu_rows=i32(offsets(lens)))
    torch.cuda.synchronize()
    for w in (0, 1):
        want = torch.from_numpy(orc.cache_read(*c.ref[w], table, first, offsets(lens), fmt))
        assert torch.equal(out[w][:T].cpu().double(), want)         # (exact in bf16 too)
        assert (out[w][T:] == 7.0).all()                            # behind the last request


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_rows_of_equal_number_and_any_strides(fmt, dtype):
    Hkv, D, B, n = 5, 128, 3, 70
    first = [0, 3, 60]
    table, n_blocks = layout(first, [n] * B)
    c = Both(n_blocks, Hkv, D, fmt)
    c.write(*(rand(63, Hkv, D, seed=s).to(dtype) for s in (4, 5)), table, [0] * B, first)
    # k: a slice of a joint projection; v: head first
    joint = rand(B * n, 3 * Hkv, D, seed=6).to(dtype).cuda()
    heads = rand(Hkv, B * n, D, seed=7).to(dtype).cuda()
    k, v = joint[:, Hkv:2 * Hkv], heads.transpose(0, 1)
    for ref, x in zip(c.ref, (k, v)):
        orc.cache_write(*ref, x.cpu().double().numpy(), table, first, offsets([n] * B), fmt)
    cb.cart_cache_write(c.gpu, k, v, i32(table), first=i32(first))
    torch.cuda.synchronize()
    c.equal()
    out_joint, out_heads = torch.full_like(joint, 9.0), torch.full_like(heads, 9.0)
    r = cb.cart_cache_read(c.gpu, out_joint[:, Hkv:2 * Hkv], out_heads.transpose(0, 1), i32(table), first=i32(first))
    torch.cuda.synchronize()
    assert r[0].data_ptr() == out_joint[:, Hkv:].data_ptr()
    want = [torch.from_numpy(orc.cache_read(*c.ref[w], table, first, offsets([n] * B), fmt)) for w in (0, 1)]
    assert torch.equal(out_joint[:, Hkv:2 * Hkv].cpu().double(), want[0]) and torch.equal(out_heads.transpose(0, 1).cpu().double(), want[1])
    assert (out_joint[:, :Hkv] == 9.0).all() and (out_joint[:, 2 * Hkv:] == 9.0).all()
    # without `first`: from token 0 on
    d = Both(n_blocks, Hkv, D, fmt)
    cb.cart_cache_write(d.gpu, k, v, i32(table))
    for ref, x in zip(d.ref, (k, v)):
        orc.cache_write(*ref, x.cpu().double().numpy(), table, [0] * B, offsets([n] * B), fmt)
    torch.cuda.synchronize()
    d.equal()


@pytest.mark.parametrize("fmt", FMT)
def test_tokens_one_at_a_time(fmt):
    """130 steps of 3 requests: growing magnitudes (every block's scale grows several times), shrinking, and both."""
    B, Hkv, D, n = 3, 2, 64, 130
    table, n_blocks = layout([0] * B, [n] * B)
    c = Both(n_blocks, Hkv, D, fmt)
    ramp = torch.stack([torch.linspace(-9, 5, n), torch.linspace(5, -9, n), 4 * torch.sin(torch.arange(n) * 0.7)], 1)
    for t in range(n):
        x, y = ((rand(B, Hkv, D, seed=100 * w + t, spread=0.3) * torch.exp2(ramp[t])[:, None, None]).bfloat16() for w in (1, 2))
        for ref, r in zip(c.ref, (x, y)):
            orc.cache_write(*ref, r.double().numpy(), table, [t] * B, offsets([1] * B), fmt)
        cb.cart_cache_write(c.gpu, x.cuda(), y.cuda(), i32(table), first=i32([t] * B))
    torch.cuda.synchronize()
    c.equal()


@pytest.mark.parametrize("fmt", FMT)
def test_magnitudes_at_the_borders(fmt):
    """Largest magnitudes at, and one fp32 step to either side of, qmax times a power of two; zeros, the smallest and largest numbers,
    halves between codes."""
    q = orc.CACHE_QMAX[fmt]
    tops = [q, np.nextafter(np.float32(q), np.float32(0)), np.nextafter(np.float32(q), np.float32(1e9)), 0.0, 1e-45, 1.2e-38, 2.0 ** -64, q * 2.0 ** -64,
            q * 2.0 ** -64 * (1 + 2.0 ** -23), 2.0 ** 126.99, np.nextafter(np.float32(2.0 ** 127), np.float32(0)), 1.0, 3.0e-20]
    B, Hkv, D = len(tops), 2, 64
    g = torch.Generator().manual_seed(8)
    means = orc.cache_meaning(fmt)
    values = np.unique(means[np.abs(means) <= q])
    halves = torch.from_numpy((values[1:] + values[:-1]) / 2)
    x = halves[torch.randint(0, len(halves), (B * 3, Hkv, D), generator=g)] / q / 1.1
    x = (x.view(B, 3, Hkv, D) * torch.tensor([float(t) for t in tops], dtype=torch.float64)[:, None, None, None]).float()
    x[:, 1, :, 5] = torch.tensor([float(t) for t in tops])[:, None]
    x[:, 2, 1, 7] = -torch.tensor([float(t) for t in tops])
    x = x.view(B * 3, Hkv, D)
    table, n_blocks = layout([0] * B, [3] * B)
    c = Both(n_blocks, Hkv, D, fmt)
    c.write(x, -x, table, [0] * B, [3] * B)
    torch.cuda.synchronize()
    c.equal()
    out = [torch.empty(B * 3, Hkv, D, device="cuda") for _ in range(2)]
    cb.cart_cache_read(c.gpu, *out, i32(table))
    torch.cuda.synchronize()
    assert torch.isfinite(out[0]).all() and torch.equal(out[0].cpu().double(), torch.from_numpy(orc.cache_read(*c.ref[0], table, [0] * B, offsets([3] * B), fmt)))


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, 2.0 ** 127])
def test_what_is_not_finite_is_seen(fmt, bad):
    """One value of K of one token and head: the scale of its block and head is NaN, its rows read as NaN, later rows too, until the
    block is begun anew; nothing else changes."""
    B, Hkv, D = 2, 3, 128
    table, n_blocks = layout([0] * B, [100] * B)
    c = Both(n_blocks, Hkv, D, fmt)
    x, y = rand(180, Hkv, D, seed=9).bfloat16(), rand(180, Hkv, D, seed=10).bfloat16()
    x[90 + 70, 1, 17] = bad                                  # request 1, block 1, head 1
    c.write(x, y, table, [0, 0], [90, 90])
    c.write(x[:2], y[:2], table, [90, 90], [1, 1])           # a row behind it
    torch.cuda.synchronize()
    c.equal()
    assert np.isnan(c.gpu.k_scale.cpu().numpy()[table[1, 1]]).tolist() == [False, True, False]
    out = [torch.empty(182, Hkv, D, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    cb.cart_cache_read(c.gpu, *out, i32(table))
    nan = torch.isnan(out[0]).cpu()
    want = torch.zeros_like(nan)
    want[91 + 64:, 1] = True
    assert torch.equal(nan, want) and not torch.isnan(out[1]).any()
    q = rand(B, 6, D, seed=11, spread=0).bfloat16()
    o, lse = cb.cart_cache_decode(q.cuda(), c.gpu, [], i32(table), i32([0, 91, 182]), 91)
    heads = torch.zeros(B, 6, dtype=torch.bool)
    heads[1, 2:4] = True
    assert torch.equal(torch.isnan(o).any(-1).cpu(), heads) and torch.equal(torch.isnan(o).all(-1).cpu(), heads)
    c.write(x[:64], y[:64], table[1:], [64], [64])           # begun anew
    torch.cuda.synchronize()
    c.equal()
    assert not np.isnan(c.gpu.k_scale.cpu().numpy()[table[1, 1]]).any()


@pytest.mark.parametrize("fmt", FMT)
def test_tokens_without_a_block(fmt):
    """Ids outside the pool, sequences past the table, a negative `first`: not written, read as 0, not attended."""
    Hkv, D, n = 2, 128, 150
    c = Both(6, Hkv, D, fmt)
    good = np.array([[0, 1, 2], [3, 4, 5]])
    x, y = rand(2 * n, Hkv, D, seed=12).bfloat16(), rand(2 * n, Hkv, D, seed=13).bfloat16()
    c.write(x, y, good, [0, 0], [n, n])
    table = np.array([[0, 2 ** 31 - 1, 2], [3, 6, -7]])
    c.write(y, x, table, [20, -1], [n, n])                   # request 0 reaches block 1, which it has not; request 1 is nowhere
    torch.cuda.synchronize()
    c.equal()
    first, lens = [30, -5, 100], [n, 3, n]
    table3 = np.array([[0, 2 ** 31 - 1, 2], [0, 1, 2], [3, 6, -7]])
    out = [torch.full((2 * n + 3, Hkv, D), 5.0, device="cuda") for _ in range(2)]
    cb.cart_cache_read(c.gpu, *out, i32(table3), first=i32(first), cu_rows=i32(offsets(lens)))
    torch.cuda.synchronize()
    for w in (0, 1):
        # (tokens 170 .. of request 0 were never written: NaN on both sides in e4m3)
        assert np.array_equal(out[w].cpu().double().numpy(), orc.cache_read(*c.ref[w], table3, first, offsets(lens), fmt), equal_nan=True)
    q = rand(2, 4, D, seed=14, spread=0).bfloat16()
    nowhere = np.array([[-1, 6, 7], [3, 6, 5]])
    seg = [np.array([5, -1, 4]), np.array([-2])]
    # (block 5 has 22 rows: with 64 of them attended the rest is what nobody wrote, NaN on both sides in e4m3)
    for shared in ([], [(seg[0], 140), (seg[1], 64)], [(np.array([4, -1, 3]), 190), (seg[1], 64)]):
        got = cb.cart_cache_decode(q.cuda(), c.gpu, [(i32(b), p) for b, p in shared], i32(nowhere), i32([0, n, 2 * n]), n)
        check_decode(*got, c.decode_ref(q, shared, nowhere, [n, n]), D)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_large_calls_are_their_requests_calls(D, dtype, fmt):
    """More than 100 MB of rows in one call, and a few requests at a time: the same codes, scales and rows."""
    Hkv, B = 8, 30
    T = 110000000 // (2 * Hkv * D * dtype.itemsize)
    cuts = sorted(np.random.RandomState(D).randint(0, T, B - 1).tolist())
    cu = [0] + cuts + [T]
    lens = [b - a for a, b in zip(cu, cu[1:])]
    first = [(13 * i) % 100 for i in range(B)]
    table, n_blocks = layout(first, lens, seed=D)
    g = torch.Generator(device="cuda").manual_seed(D)
    x, y = (torch.randn(T, Hkv, D, generator=g, device="cuda").mul_(torch.exp2(2 * torch.randn(T, Hkv, 1, generator=g, device="cuda"))).to(dtype) for _ in range(2))
    caches = []
    for per in (B, 7):
        c = cb.cache_empty(n_blocks, Hkv, D, TYPES[fmt])
        for t in c[:2]:
            t.view(torch.uint8).zero_()
        for t in c[2:]:
            t.fill_(2.0 ** -64)
        out = [torch.empty_like(x), torch.empty_like(y)]
        for i in range(0, B, per):
            j = min(i + per, B)
            rows, where = slice(cu[i], cu[j]), dict(first=i32(first[i:j]), cu_rows=i32(np.array(cu[i:j + 1]) - cu[i]))
            cb.cart_cache_write(c, x[rows], y[rows], i32(table[i:j]), **where)
            cb.cart_cache_read(c, out[0][rows], out[1][rows], i32(table[i:j]), **where)
        caches.append((*[t.view(torch.uint8) for t in c], *out))
    for a, b in zip(*caches):
        assert torch.equal(a, b)
    # and they are the rows that went in: half a step is 2^-4 of a value (e4m3) or half a scale (i8), which is at most twice the largest / 127
    for z, back in zip((x, y), caches[0][4:]):
        assert ((back.float() - z.float()).abs() <= 2.0 ** -4 * z.float().abs() + z.float().abs().max() / 127).all()


# ---- decode -------------------------------------------------------------------------------------
def filled(lens, seg_p, Hkv, D, fmt, seed=0, k_std=1.0):
    """A cache with the requests' tokens and the segments' in it."""
    table, n_own = layout([0] * len(lens), lens, spare=sum(-(-p // 64) for p in seg_p) + 1, seed=seed)
    used = set(table[table >= 0].tolist())
    free = [i for i in range(n_own) if i not in used]
    c = Both(n_own, Hkv, D, fmt)
    k, v = rand(sum(lens), Hkv, D, seed=seed + 1, spread=0.7) * k_std, rand(sum(lens), Hkv, D, seed=seed + 2)
    c.write(k, v, table, [0] * len(lens), lens)
    shared = []
    for i, p in enumerate(seg_p):
        blocks, free = np.array(free[:-(-p // 64)], dtype=np.int64), free[-(-p // 64):]
        if p:
            c.write(rand(p, Hkv, D, seed=seed + 10 + i) * k_std, rand(p, Hkv, D, seed=seed + 30 + i), blocks[None], [0], [p])
        shared.append((blocks, p))
    return c, table, shared


def run_decode(c, q, shared, table, lens, **kw):
    got = cb.cart_cache_decode(q.cuda(), c.gpu, [(i32(b), p) for b, p in shared], i32(table), i32(offsets(lens)), max(max(lens), 0), **kw)
    torch.cuda.synchronize()
    return got


DECODE = {
    "one token": ([1], []),
    "edges": ([1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 0], []),
    "no own tokens": ([0, 0, 0], [70]),
    "none at all": ([0, 0], []),
    "some": ([0, 5, 0, 300], []),
    "segments": ([7, 0, 64], [1, 64, 0, 33, 129, 31, 65, 200]),
    "many requests": ([(11 * i) % 70 for i in range(150)], [100]),
    "long and short": ([3000, 1, 2, 900], [500]),
    "a cartridge": ([40] * 5, [2500]),
}


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("Hq,Hkv,D", [(32, 8, 128), (3, 1, 128), (4, 4, 64), (8, 2, 64)])
@pytest.mark.parametrize("name", DECODE)
def test_decode(name, Hq, Hkv, D, fmt):
    print("case decode", name, Hq, Hkv, D, fmt, flush=True)
    lens, seg_p = DECODE[name]
    c, table, shared = filled(lens, seg_p, Hkv, D, fmt, seed=len(name))
    q = rand(len(lens), Hq, D, seed=77, spread=0.5).bfloat16()
    o, lse = run_decode(c, q, shared, table, lens)
    check_decode(o, lse, c.decode_ref(q, shared, table, lens), D)
    again = run_decode(c, q, shared, table, lens)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])          # run to run


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("Hq,Hkv,D", [(16, 1, 128), (17, 1, 128), (32, 1, 128), (64, 2, 64), (5, 5, 128), (14, 2, 128)])
def test_decode_head_layouts(Hq, Hkv, D, fmt):
    lens, seg_p = [100, 0, 33, 700], [64, 90]
    c, table, shared = filled(lens, seg_p, Hkv, D, fmt, seed=Hq)
    q = rand(len(lens), Hq, D, seed=78, spread=0.5).bfloat16()
    check_decode(*run_decode(c, q, shared, table, lens), c.decode_ref(q, shared, table, lens), D)


@pytest.mark.parametrize("fmt", FMT)
def test_decode_of_scores_far_apart(fmt):
    """Weights from 1 to 0: one key far above the others, first, last or in between; rising and falling scores; all equal."""
    Hkv, D, n = 1, 128, 300
    lens = [n] * 6
    table, n_blocks = layout([0] * 6, lens)
    c = Both(n_blocks, Hkv, D, fmt)
    u = rand(1, Hkv, D, seed=15, spread=0)[0]
    size = torch.zeros(6, n)
    size[0, 0] = size[1, n - 1] = size[2, 150] = 40.0
    size[3] = torch.linspace(-20, 20, n)
    size[4] = torch.linspace(20, -20, n)
    k = (size.view(-1, 1, 1) * u / D ** 0.5 + 0.01 * rand(6 * n, Hkv, D, seed=16, spread=0)).bfloat16()
    k[5 * n:] = k[5 * n]
    v = rand(6 * n, Hkv, D, seed=17)
    c.write(k.float(), v, table, [0] * 6, lens)
    for scale in (0.0, 1.0):                # (1: scores of several hundred)
        q = (u * torch.ones(6, 4, 1)).bfloat16()
        check_decode(*run_decode(c, q, [], table, lens, scale=scale), c.decode_ref(q, [], table, lens, scale or None), D)


@pytest.mark.parametrize("fmt", FMT)
def test_decode_of_scores_below_the_smallest_number(fmt):
    """A softmax scale and keys whose product fp32 does not hold: equal weights, also beside keys that do not exist."""
    lens = [40, 1, 64, 0, 130]
    c, table, shared = filled(lens, [70], 2, 128, fmt, seed=8, k_std=2.0 ** -70)
    q = rand(5, 8, 128, seed=9, spread=0.5).bfloat16()
    check_decode(*run_decode(c, q, shared, table, lens, scale=1e-30), c.decode_ref(q, shared, table, lens, 1e-30), 128)


@pytest.mark.parametrize("fmt", FMT)
def test_decode_takes_scales_that_are_no_powers_of_two(fmt):
    c, table, shared = filled([200, 31], [70], 2, 128, fmt, seed=3)
    g = torch.Generator().manual_seed(4)
    for w in (0, 1):
        f = torch.rand(c.gpu[2 + w].shape, generator=g) + 0.5
        c.gpu[2 + w].mul_(f.cuda())
        c.ref[w][1] = c.gpu[2 + w].cpu().double().numpy()
    q = rand(2, 8, 128, seed=5, spread=0.5).bfloat16()
    check_decode(*run_decode(c, q, shared, table, [200, 31]), c.decode_ref(q, shared, table, [200, 31]), 128)


@pytest.mark.parametrize("fmt", FMT)
def test_rows_past_the_bound_are_not_attended_and_outputs_stay_in_place(fmt):
    lens, bound = [300, 20, 100], 70
    c, table, shared = filled(lens, [90], 2, 128, fmt, seed=6)
    q = rand(3, 8, 128, seed=7, spread=0.5).bfloat16().cuda()
    o, lse = torch.full((5, 8, 128), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full((5, 8), 3.0, device="cuda")
    got = cb.cart_cache_decode(q, c.gpu, [(i32(shared[0][0]), 90)], i32(table), i32(offsets(lens)), bound, o=o[1:4], lse=lse[1:4])
    torch.cuda.synchronize()
    assert got[0].data_ptr() == o[1:].data_ptr() and (o[[0, 4]] == 3).all() and (lse[[0, 4]] == 3).all()
    check_decode(o[1:4], lse[1:4], c.decode_ref(q.cpu(), shared, table, [min(n, bound) for n in lens]), 128)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (32, 1, 64), (32, 8, 128), (24, 1, 128)])
@pytest.mark.parametrize("lens", [[100, 0, 33, 700, 64], [300]], ids=["five", "one"])
@pytest.mark.parametrize("seg_p", [[], [2500]], ids=["alone", "behind"])
def test_a_bound_far_above_the_lengths(seg_p, lens, Hq, Hkv, D, fmt):
    """33 MB of codes by the bound, a table as wide, a few tokens."""
    c, table, shared = filled(lens, seg_p, Hkv, D, fmt, seed=Hq + D)
    wide = np.full((len(lens), -(-33000000 // (len(lens) * Hkv * D * 64))), -1)
    wide[:, :table.shape[1]] = table
    q = rand(len(lens), Hq, D, seed=79, spread=0.5).bfloat16()
    o, lse = cb.cart_cache_decode(q.cuda(), c.gpu, [(i32(b), p) for b, p in shared], i32(wide), i32(offsets(lens)), 64 * wide.shape[1])
    check_decode(o, lse, c.decode_ref(q, shared, table, lens), D)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,P", [(4, 20000), (4, 19999), (16, 8000), (19, 7990)])
def test_long_segments_by_their_own(B, P, D, fmt):
    """Segments far longer than the requests, that list their blocks several times; the bound at the lengths and far above them."""
    Hq, Hkv, lens = 32, 8, [(67 * i) % 300 for i in range(B)]
    c, table, shared = filled(lens, [1280, 100], Hkv, D, fmt, seed=B + D)
    many = [(np.tile(shared[0][0], -(-P // 1280)), P), shared[1]]
    q = rand(B, Hq, D, seed=80, spread=0.5).bfloat16()
    ref = c.decode_ref(q, many, table, lens)
    check_decode(*run_decode(c, q, many, table, lens), ref, D)
    wide = np.full((B, -(-33000000 // (B * Hkv * D * 64))), -1)
    wide[:, :table.shape[1]] = table
    check_decode(*cb.cart_cache_decode(q.cuda(), c.gpu, [(i32(b), p) for b, p in many], i32(wide), i32(offsets(lens)), 64 * wide.shape[1]), ref, D)


@pytest.mark.parametrize("B,P,Hq,Hkv", [(63, 4000, 16, 8), (64, 4000, 16, 8), (65, 4000, 16, 8), (130, 2500, 8, 4), (4100, 1500, 4, 1)])
def test_ranges_over_many_requests(B, P, Hq, Hkv):
    """Where a range begins is found in one, two or three trips; requests without tokens at either end and in between."""
    lens = [0, 0] + [(37 * i) % 71 * (i % 5 > 0) for i in range(B - 4)] + [0, 0]
    c, table, shared = filled(lens, [640], Hkv, 64, "e4m3", seed=B)
    many = [(np.tile(shared[0][0], -(-P // 640)), P)]
    q = rand(B, Hq, 64, seed=81, spread=0.5).bfloat16()
    check_decode(*run_decode(c, q, many, table, lens), c.decode_ref(q, many, table, lens), 64)


def test_blocks_past_four_gigabytes():
    """Codes whose offset passes 2^32 bytes; the scales' offsets do not."""
    Hkv, D, n_blocks = 8, 128, 70000
    cache = cb.cache_empty(n_blocks, Hkv, D)
    for t in cache[:2]:
        t[:100].view(torch.uint8).zero_()
    cache.k_scale.fill_(1.0), cache.v_scale.fill_(1.0)
    lens = [130, 64]
    table = np.array([[69999, 0, 66001], [65537, 1, 2]])
    k, v = rand(194, Hkv, D, seed=18).bfloat16().cuda(), rand(194, Hkv, D, seed=19).bfloat16().cuda()
    cb.cart_cache_write(cache, k, v, i32(table), cu_rows=i32(offsets(lens)))
    out = cb.cart_cache_read(cache, torch.empty_like(k), torch.empty_like(v), i32(table), cu_rows=i32(offsets(lens)))
    small = cb.cache_empty(6, Hkv, D)
    table2 = np.array([[0, 1, 2], [3, 4, 5]])
    cb.cart_cache_write(small, k, v, i32(table2), cu_rows=i32(offsets(lens)))
    for w in (0, 1):
        for b in range(2):
            for j in range(-(-lens[b] // 64)):
                m = min(64, lens[b] - 64 * j)
                a, z = cache[w][table[b, j], :, :m], small[w][table2[b, j], :, :m]
                assert torch.equal(a.view(torch.uint8), z.view(torch.uint8)) and torch.equal(cache[2 + w][table[b, j]], small[2 + w][table2[b, j]])
    again = cb.cart_cache_read(small, torch.empty_like(k), torch.empty_like(v), i32(table2), cu_rows=i32(offsets(lens)))
    assert torch.equal(out[0], again[0]) and torch.equal(out[1], again[1])
    q = rand(2, 32, D, seed=20, spread=0).bfloat16().cuda()
    a = cb.cart_cache_decode(q, cache, [(i32([69999]), 64)], i32(table), i32(offsets(lens)), 130)
    b = cb.cart_cache_decode(q, small, [(i32([0]), 64)], i32(table2), i32(offsets(lens)), 130)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- together -----------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FMT)
def test_a_server_answers_with_a_cartridge(fmt):
    """A cartridge is loaded; read back for the attention over two prompts; their keys and values are written; tokens are generated."""
    Hq, Hkv, D, P, S, steps = 8, 2, 128, 150, 40, 30
    blocks = -(-(S + steps) // 64)
    c = cb.cache_empty(3 + 2 * blocks, Hkv, D, TYPES[fmt])
    cart_blocks = i32([[2 + 2 * blocks, 0, 1]])
    table = i32(np.arange(2, 2 + 2 * blocks).reshape(2, blocks))
    z_k, z_v = rand(Hkv, P, D, seed=21).cuda(), rand(Hkv, P, D, seed=22).cuda()
    cb.cart_cache_write(c, z_k.transpose(0, 1), z_v.transpose(0, 1), cart_blocks)
    y_k, y_v = (torch.empty(Hkv, P, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cb.cart_cache_read(c, y_k.transpose(0, 1), y_v.transpose(0, 1), cart_blocks)
    q, k, v = (rand(2, S, h, D, seed=23 + h, spread=0.3).bfloat16().cuda() for h in (Hq, Hkv, Hkv + 1))
    v = v[:, :, :Hkv].contiguous()
    o, lse = cb.cart_attn_fwd(q, k, v, y_k, y_v)
    f64 = lambda t: t.double().cpu().numpy()
    o_ref, lse_ref = orc.attn_fwd(f64(q), f64(k), f64(v), f64(y_k), f64(y_v))
    assert np.abs(f64(o) - o_ref).max() <= 2e-2 * np.abs(o_ref).max()
    cb.cart_cache_write(c, k.flatten(0, 1), v.flatten(0, 1), table)
    shared = [(cart_blocks[0], P)]
    for t in range(steps):
        n = S + t
        q1, k1, v1 = (rand(2, h, D, seed=200 + 10 * t + h, spread=0.5).bfloat16().cuda() for h in (Hq, Hkv, Hkv + 1))
        cb.cart_cache_write(c, k1, v1[:, :Hkv].contiguous(), table, first=i32([n, n]))
        o, lse = cb.cart_cache_decode(q1, c, shared, table, i32([0, n + 1, 2 * n + 2]), n + 1)
        if t % 10 == 9:
            # the 16-bit decode over what the cache holds, and the oracle
            own = [torch.empty(2 * n + 2, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            cb.cart_cache_read(c, *own, table)
            o16, lse16 = cb.cart_decode(q1, y_k, y_v, *own, i32([0, n + 1, 2 * n + 2]), n + 1)
            torch.cuda.synchronize()
            codes = [x.view(torch.uint8).cpu().numpy() for x in c[:2]]
            ref = orc.cache_decode(f64(q1), codes[0], f64(c.k_scale), codes[1], f64(c.v_scale), [(cart_blocks[0].cpu().numpy(), P)],
                                   table.cpu().numpy(), [0, n + 1, 2 * n + 2], fmt)
            check_decode(o, lse, ref, D)
            check_decode(o16, lse16, ref, D)


def test_steps_replay_from_a_graph():
    """A step (write, decode, read) captured twice with one workspace; replayed with eager work between; requests that grow from replay to
    replay."""
    B, Hq, Hkv, D = 5, 8, 2, 128
    cap = 64 * 3
    table = i32(np.random.RandomState(2).permutation(3 * B).reshape(B, 3))
    c = cb.cache_empty(3 * B + 4, Hkv, D)
    cart = i32([3 * B, 3 * B + 1, 3 * B + 2, 3 * B + 3])
    z = rand(200, Hkv, D, seed=30).bfloat16().cuda()
    cb.cart_cache_write(c, z, z.flip(0).contiguous(), cart[None])
    lens = [7, 60, 63, 64, 120]
    x = rand(sum(lens), Hkv, D, seed=31).bfloat16().cuda()
    cb.cart_cache_write(c, x, x.flip(0).contiguous(), table, cu_rows=i32(offsets(lens)))
    first, cu = i32(lens), i32(offsets([n + 1 for n in lens]))
    q, k, v = torch.zeros(B, Hq, D, dtype=torch.bfloat16, device="cuda"), *(torch.zeros(B, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    o, lse, back = torch.empty_like(q), torch.empty(B, Hq, device="cuda"), [torch.empty_like(k), torch.empty_like(v)]
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def step(cache, o, lse, back):
        cb.cart_cache_write(cache, k, v, table, first=first)
        cb.cart_cache_decode(q, cache, [(cart, 200)], table, cu, cap, o=o, lse=lse, workspace=ws)
        cb.cart_cache_read(cache, *back, table, first=first)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cb.Cache(*(t.clone() for t in c)), o, lse, back)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    second = cb.Cache(*(t.clone() for t in c))
    outs = [(o, lse, back), (torch.empty_like(o), torch.empty_like(lse), [torch.empty_like(k), torch.empty_like(v)])]
    graphs = []
    for cache, out in zip((c, second), outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(cache, *out)
        graphs.append(g)
    eager = cb.Cache(*(t.clone() for t in c))
    for i in range(4):
        q.copy_(rand(B, Hq, D, seed=40 + i, spread=0.5)), k.copy_(rand(B, Hkv, D, seed=50 + i)), v.copy_(rand(B, Hkv, D, seed=60 + i))
        first.copy_(torch.tensor([n + i for n in lens])), cu.copy_(torch.tensor(offsets([n + i + 1 for n in lens])))
        want = (torch.empty_like(o), torch.empty_like(lse), [torch.empty_like(k), torch.empty_like(v)])
        step(eager, *want)
        torch.cuda.synchronize()
        ws.fill_(255)                       # NaN
        for g, cache, got in zip(graphs, (c, second), outs):
            got[0].zero_(), got[1].zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and all(torch.equal(a, b) for a, b in zip(got[2], want[2]))
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(cache, eager))


def test_on_a_stream_of_its_own():
    c, table, shared = filled([300, 20, 1000], [90], 2, 128, "e4m3", seed=8)
    q = rand(3, 8, 128, seed=9, spread=0.5).bfloat16().cuda()
    seg, t, cu = [(i32(shared[0][0]), 90)], i32(table), i32(offsets([300, 20, 1000]))
    want = cb.cart_cache_decode(q, c.gpu, seg, t, cu, 1000)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = cb.cart_cache_decode(q, c.gpu, seg, t, cu, 1000, stream=side)
    k = torch.empty(1320, 2, 128, device="cuda")
    v = torch.empty_like(k)
    cb.cart_cache_read(c.gpu, k, v, t, cu_rows=cu, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(k.cpu().double(), torch.from_numpy(orc.cache_read(*c.ref[0], table, [0] * 3, offsets([300, 20, 1000]), "e4m3")))
