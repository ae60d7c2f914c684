"""The 8-bit key/value cache, timed operator by operator: writing rows into it, reading them back, and the decode step over it.

The cache of one layer is a pool of blocks of 64 tokens, `k` and `v` [n_blocks, Hkv, 64, D] in e4m3 or int8, with a scale
for each block and head, `k_scale` and `v_scale` [n_blocks, Hkv]; a request owns the blocks that its row of `table`
[B, max_blocks] names, in order.  A scale is the smallest power of two, 2^-64 at least, that brings the largest magnitude
of the block's rows into the codes' range (127 for int8, 448 for e4m3); code = round(x / scale), half to even.  Rows that
land behind others in a block raise its scale where they need it, and the codes before them are rounded again.

Shapes come from the library's own decode and training configurations and lie around them.
"""
from __future__ import annotations

import math
import random

import torch

own = False         # True: run() calls the library's entry points; False: the same in elementary operations

BLOCK = 64
MIN_SCALE = 2.0 ** -64
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
# the codes' largest magnitude as fraction and exponent, 0.5 <= fraction < 1
LARGEST = {"e4m3": (0.875, 9), "i8": (0.9921875, 7)}
HEADS = [(32, 8), (32, 8), (24, 8), (8, 2), (16, 16), (8, 1)]


def _decode(name, B, Hq, Hkv, P, n_shared, base, min_len, max_len, len_seed, fmt, D=128):
    return {"name": name, "kind": "decode", "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "P": P, "n_shared": n_shared, "base": base,
            "min_len": min_len, "max_len": max_len, "len_seed": len_seed, "fmt": fmt}


def _rows(name, kind, B, Hkv, base, min_len, max_len, len_seed, fmt, dtype, layout="rows", D=128):
    return {"name": name, "kind": kind, "B": B, "Hkv": Hkv, "D": D, "base": base, "min_len": min_len, "max_len": max_len,
            "len_seed": len_seed, "fmt": fmt, "dtype": dtype, "layout": layout}


def listed():
    return [
        # ---- decode over the cache --------------------------------------------------------------
        # a nearly idle server: four requests on one cartridge, latency is what counts
        _decode("decode_few", 4, 32, 8, 2048, 1, 0, 1, 150, 5003, "e4m3"),
        # a full server: 128 requests share one cartridge
        _decode("decode_shared", 128, 32, 8, 8192, 1, 0, 1, 1024, 5001, "e4m3"),
        # every request brings its own cartridge of 2048 slots, first in its blocks, behind a small shared one
        _decode("decode_private", 128, 32, 8, 2048, 1, 2048, 1, 1024, 5001, "i8"),
        # long histories without a cartridge (the comparison workload: 8 requests of 131072 tokens)
        _decode("decode_long", 8, 32, 8, 0, 0, 0, 131072, 131072, 5005, "e4m3"),
        # three composed cartridges that end inside a block, odd numbers of requests and tokens, three query heads a group
        _decode("decode_composed", 23, 24, 8, 5003, 3, 0, 1, 777, 5007, "i8"),
        # ---- writing ----------------------------------------------------------------------------
        # one generated token of each of 128 requests, behind up to 1024 others
        _rows("write_step", "write", 128, 8, 1024, 1, 1, 5001, "e4m3", "bf16"),
        # a trained cartridge is loaded: fp32 vectors [Hkv,p,D]
        _rows("write_cartridge", "write", 1, 8, 0, 8192, 8192, 5011, "i8", "f32", "heads"),
        # 64 prompts of 64 .. 1024 tokens, behind cartridges and turns that ended anywhere
        _rows("write_prompts", "write", 64, 8, 200, 64, 1024, 5013, "e4m3", "bf16"),
        # the largest training batch's worth of tokens (64 x 2048)
        _rows("write_large", "write", 64, 8, 0, 2048, 2048, 5015, "i8", "bf16"),
        # ---- reading back -----------------------------------------------------------------------
        # a cartridge for the attention over a prompt: [Hkv,p,D]
        _rows("read_cartridge", "read", 1, 8, 0, 8192, 8192, 5011, "e4m3", "bf16", "heads"),
        # two short histories for inspection, odd lengths from odd places, fp32
        _rows("read_few", "read", 2, 8, 70, 33, 201, 5017, "i8", "f32"),
        # 128 requests' histories of 1 .. 2048 tokens
        _rows("read_many", "read", 128, 8, 0, 1, 2048, 5019, "i8", "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    fmt, D = rng.choice(["e4m3", "i8"]), rng.choice([128, 128, 128, 64])
    u = rng.random()
    most = max(work(c)["bytes"] for c in listed())
    if u < 0.5:
        # one request to a full server; no, one or several shared cartridges, some with one per request; short and
        # long histories
        while True:
            Hq, Hkv = rng.choice(HEADS)
            n_shared = rng.choice([0, 1, 1, 1, 3])
            B, hi = _log(rng, 1, 256), _log(rng, 1, 131072)
            c = _decode("", B, Hq, Hkv, _log(rng, 128, 8192) if n_shared else 0, n_shared, _log(rng, 128, 2048) if rng.random() < 0.25 else 0,
                        rng.randint(1, hi), hi, rng.randrange(10000), fmt, D)
            # (the plain form pads to the longest request)
            if B * (hi + c["base"]) <= 2 ** 20 and work(c)["bytes"] <= most:
                break
    else:
        # one token of each of a server's requests, prompts, cartridges; to a pool's worth of rows
        while True:
            kind = "write" if u < 0.8 else "read"
            Hkv = rng.choice(HEADS)[1]
            one = rng.random()
            if one < 0.3:
                c = _rows("", kind, _log(rng, 1, 512), Hkv, _log(rng, 1, 4096), 1, 1, rng.randrange(10000), fmt, rng.choice(["bf16", "bf16", "f32"]), "rows", D)
            elif one < 0.5:
                p = _log(rng, 128, 8192)
                c = _rows("", kind, 1, Hkv, 0, p, p, rng.randrange(10000), fmt, rng.choice(["bf16", "f32"]), "heads", D)
            else:
                hi = _log(rng, 16, 8192)
                c = _rows("", kind, _log(rng, 1, 256), Hkv, rng.choice([0, _log(rng, 1, 4096)]), rng.randint(1, hi), hi, rng.randrange(10000), fmt,
                          rng.choice(["bf16", "bf16", "f32"]), "rows", D)
            if c["B"] * (c["base"] + c["max_len"]) <= 2 ** 19 and work(c)["bytes"] <= most / 4:
                break
    del c["name"]
    return c


# ---- inputs -------------------------------------------------------------------------------------
def _lengths(case, seed=None):
    """The case's lengths; a seed deals them out in another order (their sum stays)."""
    g = torch.Generator().manual_seed(case["len_seed"])
    lens = torch.randint(case["min_len"], case["max_len"] + 1, (case["B"],), generator=g)
    if seed is None:
        return lens
    return lens[torch.randperm(case["B"], generator=torch.Generator().manual_seed(seed))]


def _offsets(lens):
    cu = torch.zeros(lens.numel() + 1, dtype=torch.int32)
    cu[1:] = torch.cumsum(lens, 0).to(torch.int32)
    return cu.cuda()


def _values(sizes, g):
    """Keys or values: normal, with a factor for each vector (the last dimension) that spreads over a few octaves."""
    x = torch.randn(sizes, generator=g, device="cuda")
    return x.mul_(torch.exp2(0.5 * torch.randn(*sizes[:-1], 1, generator=g, device="cuda")))


def _scale_for(amax, fmt):
    f, e = torch.frexp(amax)
    fraction, exponent = LARGEST[fmt]
    e = e - exponent + (f > fraction).to(e.dtype)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.zeros_like(amax)).clamp(min=MIN_SCALE)


def _codes(x, fmt):
    return x.round().to(torch.int8) if fmt == "i8" else x.to(torch.float8_e4m3fn)


def _filled(n_blocks, Hkv, D, fmt, g):
    """Codes and scales of a pool all of whose blocks hold rows."""
    x = _values((n_blocks, Hkv, BLOCK, D), g)
    s = _scale_for(x.abs().amax((2, 3)), fmt)
    return _codes(x / s[:, :, None, None], fmt), s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    B, Hkv, D, fmt = case["B"], case["Hkv"], case["D"], case["fmt"]
    lens = _lengths(case, seed)
    if case["kind"] == "decode":
        lens = lens + case["base"]                                  # the request's own cartridge comes first in its blocks
        before = torch.zeros(B, dtype=torch.int64)
        n, P = case["n_shared"], case["P"]
        cuts = [P * i // n for i in range(n + 1)] if n else [0]
        parts = [b - a for a, b in zip(cuts, cuts[1:])]
    else:
        # rows before the ones of this call: any number up to `base`
        before = torch.randint(0, case["base"] + 1, (B,), generator=host)
        parts = []
    used = (before + lens + BLOCK - 1) // BLOCK
    seg = [-(-p // BLOCK) for p in parts]
    # as many for every seed; some blocks belong to nobody
    n_blocks = (int(lens.sum()) + B * (0 if case["kind"] == "decode" else case["base"])) // BLOCK + B + sum(seg) + 3
    ids = torch.randperm(n_blocks, generator=host).to(torch.int32)  # a pool that has been in use for a while
    max_blocks = int(used.max())
    table = torch.full((B, max_blocks), -1, dtype=torch.int32)
    mine = torch.arange(max_blocks)[None] < used[:, None]
    table[mine] = ids[:int(used.sum())]
    at = torch.tensor([int(used.sum())] + seg).cumsum(0).tolist()
    shared = [(ids[a:a + m].cuda(), p) for a, m, p in zip(at, seg, parts)]
    k, k_scale = _filled(n_blocks, Hkv, D, fmt, g)
    v, v_scale = _filled(n_blocks, Hkv, D, fmt, g)
    st = {"case": case, "cache": (k, v, k_scale, v_scale), "table": table.cuda(), "cu": _offsets(lens)}
    if case["kind"] == "decode":
        q = torch.randn(B, case["Hq"], D, generator=g, device="cuda").to(torch.bfloat16)
        return {**st, "q": q, "shared": shared, "max_len": int(lens.max())}
    T = int(lens.sum())
    st["first"] = before.to(torch.int32).cuda()
    st["rows"] = T
    # equal numbers of rows need no offsets
    st["even"] = case["min_len"] == case["max_len"]
    if case["kind"] == "write":
        sizes = (Hkv, T, D) if case["layout"] == "heads" else (T, Hkv, D)
        st["k"], st["v"] = (_values(sizes, g).to(TORCH[case["dtype"]]) for _ in range(2))
    return st


# ---- one pass -----------------------------------------------------------------------------------
def run(st):
    case = st["case"]
    if own:
        return _own(st)
    if case["kind"] == "decode":
        return _plain_decode(st)
    return _plain_write(st) if case["kind"] == "write" else _plain_read(st)


def _own(st):
    from paper_2506_06266_amd import binding as cart
    case, cache = st["case"], st["cache"]
    if case["kind"] == "decode":
        return cart.cart_cache_decode(st["q"], cache, st["shared"], st["table"], st["cu"], st["max_len"])
    heads, cu = case["layout"] == "heads", None if st["even"] else st["cu"]
    if case["kind"] == "write":
        k, v = (st["k"].transpose(0, 1), st["v"].transpose(0, 1)) if heads else (st["k"], st["v"])
        cart.cart_cache_write(cache, k, v, st["table"], first=st["first"], cu_rows=cu)
        return cache
    sizes = (case["Hkv"], st["rows"], case["D"]) if heads else (st["rows"], case["Hkv"], case["D"])
    k, v = (torch.empty(sizes, dtype=TORCH[case["dtype"]], device="cuda") for _ in range(2))
    cart.cart_cache_read(cache, k.transpose(0, 1) if heads else k, v.transpose(0, 1) if heads else v, st["table"], first=st["first"], cu_rows=cu)
    return k, v


def _where(st):
    """The request, the block, the row in it and the position of each row of the call."""
    t = torch.arange(st["rows"], dtype=torch.int32, device="cuda")
    b = torch.searchsorted(st["cu"][1:], t, right=True)
    pos = (st["first"][b] + t - st["cu"][b]).long()
    return b, st["table"][b, pos // BLOCK].long(), pos % BLOCK, pos


def _plain_write(st):
    b, block, row, pos = _where(st)
    first = st["first"][b].long()
    touched, at = torch.unique(block, return_inverse=True)
    # rows of each touched block that were there before: of a request's first one only
    kept = torch.where(pos // BLOCK == first // BLOCK, first % BLOCK, torch.zeros_like(first))
    kept = torch.zeros_like(touched).scatter_reduce_(0, at, kept, "amax")
    k, v, k_scale, v_scale = st["cache"]
    heads = st["case"]["layout"] == "heads"
    _plain_write_one(st["k"].transpose(0, 1) if heads else st["k"], k, k_scale, st["case"]["fmt"], touched, at, row, kept)
    _plain_write_one(st["v"].transpose(0, 1) if heads else st["v"], v, v_scale, st["case"]["fmt"], touched, at, row, kept)
    return st["cache"]


def _plain_write_one(x, codes, scale, fmt, touched, at, row, kept):
    x = x.float()
    amax = torch.zeros(touched.numel(), x.shape[1], device="cuda")
    amax.scatter_reduce_(0, at[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
    before = torch.where(kept[:, None] > 0, scale[touched], torch.full_like(amax, MIN_SCALE))
    s = torch.maximum(_scale_for(amax, fmt), before)
    held = codes.view(torch.uint8)[touched].view(codes.dtype).float()
    stays = (torch.arange(BLOCK, device="cuda") < kept[:, None])[:, None, :, None]
    held = torch.where(stays, held * (before / s)[:, :, None, None], held)
    held[at, :, row] = x / s[at][:, :, None]
    codes.view(torch.uint8)[touched] = _codes(held, fmt).view(torch.uint8)
    scale[touched] = s


def _plain_read(st):
    _, block, row, _ = _where(st)
    k, v, k_scale, v_scale = st["cache"]
    dtype, heads = TORCH[st["case"]["dtype"]], st["case"]["layout"] == "heads"
    out_k = (k.view(torch.uint8)[block, :, row].view(k.dtype).float() * k_scale[block][:, :, None]).to(dtype)
    out_v = (v.view(torch.uint8)[block, :, row].view(v.dtype).float() * v_scale[block][:, :, None]).to(dtype)
    return (out_k.transpose(0, 1).contiguous(), out_v.transpose(0, 1).contiguous()) if heads else (out_k, out_v)


def _dequantised(codes, scale, blocks):
    """Rows of the blocks [..., n] in fp32: [..., Hkv, 64 n, D]."""
    x = codes.view(torch.uint8)[blocks].view(codes.dtype).float() * scale[blocks][..., None, None]
    return x.transpose(-4, -3).flatten(-3, -2)


def _plain_decode(st):
    case, (k, v, k_scale, v_scale) = st["case"], st["cache"]
    B, Hq, Hkv, D = case["B"], case["Hq"], case["Hkv"], case["D"]
    q = st["q"].float().view(B, Hkv, Hq // Hkv, D)
    table = st["table"].long().clamp(min=0)
    lens = (st["cu"][1:] - st["cu"][:-1])[:, None, None, None]
    s = torch.matmul(q, _dequantised(k, k_scale, table).transpose(-1, -2)) / math.sqrt(D)
    s = torch.where(torch.arange(s.shape[-1], device="cuda") < lens, s, -math.inf)
    n = 0                                                           # columns of the shared segments
    if st["shared"]:
        common = torch.cat([b for b, _ in st["shared"]]).long()
        there = torch.cat([torch.arange(BLOCK * b.numel(), device="cuda") < p for b, p in st["shared"]])
        z = torch.matmul(q.transpose(0, 1).flatten(1, 2), _dequantised(k, k_scale, common).transpose(-1, -2)) / math.sqrt(D)
        z = torch.where(there, z, -math.inf).view(Hkv, B, Hq // Hkv, -1).transpose(0, 1)
        s, n = torch.cat([z, s], -1), z.shape[-1]
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p[..., n:], _dequantised(v, v_scale, table))
    if st["shared"]:
        z = torch.matmul(p[..., :n].transpose(0, 1).flatten(1, 2), _dequantised(v, v_scale, common))
        o = o + z.view(Hkv, B, Hq // Hkv, D).transpose(0, 1)
    lse = top + torch.log(total)
    return (o / total).view(B, Hq, D).to(torch.bfloat16), lse.view(B, Hq)


# ---- the definition in 64 bits ------------------------------------------------------------------
def _meaning(fmt):
    """What each of the 256 codes stands for."""
    c = torch.arange(256)
    if fmt == "i8":
        return torch.where(c < 128, c, c - 256).double().cuda()
    sign, e, m = 1 - 2 * (c >> 7).double(), (c >> 3 & 15).double(), (c & 7).double()
    x = torch.where(e > 0, (1 + m / 8) * torch.exp2(e - 7), m * 2.0 ** -9)
    return (sign * torch.where((c & 127) == 127, math.nan, x)).cuda()


def _nearest(x, fmt):
    """The representable value next to each of x, in 64 bits; of two the even one."""
    if fmt == "i8":
        return torch.round(x)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    st = prepare(case, seed)
    k, v, k_scale, v_scale = st["cache"]
    code = [t.view(torch.uint8) for t in (k, v)]
    scale = [t.double() for t in (k_scale, v_scale)]
    means = _meaning(case["fmt"])
    cu, table = st["cu"].tolist(), st["table"].tolist()

    def history(which, blocks, lo, hi):
        """Rows lo .. hi of the sequence that the blocks hold: [hi - lo, Hkv, D]."""
        some = torch.tensor(blocks[lo // BLOCK:-(-hi // BLOCK)], device="cuda", dtype=torch.int64)
        x = means[code[which][some].int()] * scale[which][some][:, :, None, None]
        lo, hi = lo - lo // BLOCK * BLOCK, hi - lo // BLOCK * BLOCK
        return x.permute(0, 2, 1, 3).reshape(-1, x.shape[1], x.shape[3])[lo:hi]

    if case["kind"] == "decode":
        B, Hq, Hkv, D = case["B"], case["Hq"], case["Hkv"], case["D"]
        common = [[history(w, b.tolist(), 0, p) for b, p in st["shared"]] for w in (0, 1)]
        o, lse = torch.empty(B, Hq, D, dtype=torch.float64, device="cuda"), torch.empty(B, Hq, dtype=torch.float64, device="cuda")
        for b in range(B):
            n = cu[b + 1] - cu[b]
            K, V = (torch.cat(common[w] + [history(w, table[b], 0, n)]).permute(1, 0, 2) for w in (0, 1))
            q = st["q"][b].double().view(Hkv, Hq // Hkv, D)
            s = (q @ K.transpose(1, 2).contiguous()) * D ** -0.5
            lse[b] = torch.logsumexp(s, -1).view(Hq)
            o[b] = (torch.softmax(s, -1) @ V.contiguous()).view(Hq, D)
        return o, lse
    first = st["first"].tolist()
    if case["kind"] == "read":
        out = [torch.cat([history(w, table[b], first[b], first[b] + cu[b + 1] - cu[b]) for b in range(case["B"])]) for w in (0, 1)]
        return tuple(x.transpose(0, 1).contiguous() if case["layout"] == "heads" else x for x in out)
    largest = math.ldexp(*LARGEST[case["fmt"]])
    held = [means[c.int()] for c in code]
    for w, x in enumerate((st["k"], st["v"])):
        x = (x.transpose(0, 1) if case["layout"] == "heads" else x).double()
        for b in range(case["B"]):
            rows, lo = x[cu[b]:cu[b + 1]], first[b]
            n = rows.shape[0]
            some = torch.tensor(table[b][lo // BLOCK:-(-(lo + n) // BLOCK)], device="cuda", dtype=torch.int64)
            kept, count = lo % BLOCK, some.numel()
            fresh = torch.zeros(count * BLOCK, x.shape[1], x.shape[2], dtype=torch.float64, device="cuda")
            fresh[kept:kept + n] = rows
            fresh = fresh.view(count, BLOCK, x.shape[1], x.shape[2]).transpose(1, 2)
            amax = fresh.abs().amax((2, 3))
            f, e = torch.frexp(amax / largest)
            s = torch.where(amax > 0, torch.exp2((e - (f == 0.5).to(e.dtype)).double()), 0.0).clamp(min=MIN_SCALE)
            was = scale[w][some]
            if kept:
                s[0] = torch.maximum(s[0], was[0])
            there = torch.zeros(count * BLOCK, dtype=torch.bool, device="cuda")
            there[kept:kept + n] = True
            there = there.view(count, 1, BLOCK, 1)
            old = held[w][some]
            if kept:
                old[0, :, :kept] = _nearest(old[0, :, :kept] * (was[0] / s[0])[:, None, None], case["fmt"])
            held[w][some] = torch.where(there, _nearest(fresh / s[:, :, None, None], case["fmt"]), old)
            scale[w][some] = s
    return held[0], held[1], scale[0], scale[1]


# ---- what a pass cannot do without --------------------------------------------------------------
def work(case):
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    T = int(_lengths(case).sum())
    if case["kind"] == "decode":
        T += B * case["base"]
        scales = 2 * Hkv * 4 * -(-(T + case["P"]) // BLOCK)
        # codes of every row once, q, o (bf16), lse
        return {"bytes": 2 * (T + case["P"]) * Hkv * D + scales + 4 * B * case["Hq"] * D + 4 * B * case["Hq"],
                "flops": 4 * D * case["Hq"] * (T + B * case["P"])}
    scales = 2 * Hkv * 4 * max(B, T // BLOCK)
    return {"bytes": 2 * T * Hkv * D * (1 + TORCH[case["dtype"]].itemsize) + scales, "flops": 3 * 2 * T * Hkv * D}
