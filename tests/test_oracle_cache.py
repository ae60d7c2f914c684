"""The 8-bit cache's oracle against hand-worked values, PyTorch's conversion and the 16-bit decode oracle (CPU)."""
import numpy as np
import pytest
import torch

from oracle import cartridge_oracle as orc

FMT = ["e4m3", "i8"]


def test_codes_mean_what_the_formats_say():
    e, i = orc.cache_meaning("e4m3"), orc.cache_meaning("i8")
    assert [e[c] for c in (0, 1, 7, 8, 0x38, 0x7E, 0xB8)] == [0, 2.0 ** -9, 7 * 2.0 ** -9, 2.0 ** -6, 1, 448, -1] and np.isnan(e[0x7F])
    assert [i[c] for c in (0, 1, 127, 129, 255)] == [0, 1, 127, -127, -1]
    bits = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(bits, e, equal_nan=True)


@pytest.mark.parametrize("fmt", FMT)
def test_nearest_is_nearest_and_even(fmt):
    g = torch.Generator().manual_seed(1)
    means = orc.cache_meaning(fmt)
    values = np.unique(means[np.abs(means) <= orc.CACHE_QMAX[fmt]])
    x = np.concatenate([(torch.randn(4000, generator=g) * 2.0 ** torch.randint(-12, 7, (4000,), generator=g)).clamp(-127, 127).double().numpy(),
                        (values[1:] + values[:-1]) / 2, values])
    y = means[orc.cache_nearest(x, fmt)]
    assert np.array_equal(np.abs(x - y), np.abs(x[:, None] - values[None]).min(1))
    t = torch.from_numpy(x)
    same = t.round() if fmt == "i8" else t.float().to(torch.float8_e4m3fn).double()        # (every x here is an fp32 number)
    assert np.array_equal(y, same.numpy())


@pytest.mark.parametrize("fmt", FMT)
def test_scale_is_the_smallest_power_of_two(fmt):
    q = orc.CACHE_QMAX[fmt]
    assert orc.cache_scale(q, fmt) == 1 and orc.cache_scale(np.nextafter(q, 1e9), fmt) == 2 and orc.cache_scale(q / 2, fmt) == 0.5
    assert orc.cache_scale(0.0, fmt) == 2.0 ** -64 and orc.cache_scale(1e-300, fmt) == 2.0 ** -64
    assert np.isnan(orc.cache_scale(2.0 ** 127, fmt)) and np.isfinite(orc.cache_scale(np.nextafter(2.0 ** 127, 0), fmt))


@pytest.mark.parametrize("fmt", FMT)
def test_rows_one_at_a_time_stay_within_the_bound(fmt):
    g = torch.Generator().manual_seed(2)
    n, Hkv, d = 150, 2, 16
    x = (torch.randn(n, Hkv, d, generator=g) * 2.0 ** torch.linspace(-6, 3, n)[:, None, None]).double().numpy()
    codes, scale = np.full((4, Hkv, 64, d), 0x7F, np.uint8), np.full((4, Hkv), np.nan)
    table = np.array([[2, 0, 3]])
    for t in range(n):
        orc.cache_write(codes, scale, x[t:t + 1], table, [t], [0, 1], fmt)
    y = orc.cache_read(codes, scale, table, [0], [0, n], fmt)
    s = scale[table[0][np.arange(n) // 64]][:, :, None]
    # all roundings of a value add up to less than one scale (int8); half a step of e4m3, 2^-4 relative, and of its smallest values
    # 2^-10 of a scale at each growth
    bound = s if fmt == "i8" else 2.0 ** -4 * np.abs(x) + 2.0 ** -9 * s
    assert (np.abs(x - y) <= bound).all()
    at_once, one = np.zeros_like(codes), np.zeros_like(scale)
    orc.cache_write(at_once, one, x, table, [0], [0, n], fmt)
    assert np.array_equal(scale[table[0]], one[table[0]])
    assert (scale[1] != scale[1]).all()         # nobody's block


@pytest.mark.parametrize("fmt", FMT)
def test_decode_is_the_16_bit_oracles_on_what_the_codes_stand_for(fmt):
    g = torch.Generator().manual_seed(3)
    Hq, Hkv, d = 6, 2, 16
    lens, p = [70, 1, 0, 130], 90
    cu = np.concatenate([[0], np.cumsum(lens)])
    x = torch.randn(int(cu[-1]) + p, 2, Hkv, d, generator=g).double().numpy()
    table = np.array([[1, 9, -1], [4, -1, -1], [-1, -1, -1], [3, 7, 0]])
    seg = np.array([[8, 2]])
    cache = [(np.full((10, Hkv, 64, d), 0x7F, np.uint8), np.full((10, Hkv), np.nan)) for _ in range(2)]
    for w in (0, 1):
        orc.cache_write(*cache[w], x[:cu[-1], w], table, [0] * 4, cu, fmt)
        orc.cache_write(*cache[w], x[cu[-1]:, w], seg, [0], [0, p], fmt)
    q = torch.randn(4, Hq, d, generator=g).double().numpy()
    o, lse, size, reach = orc.cache_decode(q, *cache[0], *cache[1], [(seg[0], p)], table, cu, fmt)
    own = [orc.cache_read(*cache[w], table, [0] * 4, cu, fmt) for w in (0, 1)]
    z = [orc.cache_read(*cache[w], seg, [0], [0, p], fmt).transpose(1, 0, 2) for w in (0, 1)]
    o2, lse2 = orc.decode(q, z[0], z[1], own[0], own[1], cu)
    assert np.allclose(o, o2, rtol=0, atol=1e-14) and np.allclose(lse, lse2, rtol=0, atol=1e-13)
    assert (size >= np.abs(o) - 1e-14).all() and (reach > 0).all()
    # no key at all
    o, lse, _, _ = orc.cache_decode(q, *cache[0], *cache[1], [], table, cu, fmt)
    assert (o[2] == 0).all() and (lse[2] == -np.inf).all() and np.isfinite(lse[[0, 1, 3]]).all()
