"""Codes and scales of rotated keys next to the borders between two codes, and of two scales, in a 4-bit
cache: reached by a rotation, so that the elements are no numbers of 32 bits.

A pair (b, z) that is turned by a small angle t becomes b cos t - z sin t, within t^2 of b - z t: with b
a border and t some parts of a step of b's 32-bit numbers, the element lies that far from the border, on
the side that t's sign or z's says.  Codes and scales are compared for equality with those of the formula
in 64 bits, whose rotation is right to 2^-51 of the elements; each case says first that none of its
elements lies nearer to its border than 2^-32 of it, and that all are within one step of it.

The rotation's angle pos * rate may have 55 bits, two more than 64-bit numbers hold.  The cases of far
positions look for pairs that the rounded product puts on the wrong side of a border, at least 2^-38
from it; the angle's sine and cosine come from the product and what it lost, taken exactly.
"""
import math
from fractions import Fraction

import numpy as np
import pytest

from test_gpu_cache4 import dtype_of, f64, plain_encode

pytestmark = pytest.mark.gpu

BORDERS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0)  # the last one between two scales
PARTS = (0.1, 0.3, 0.45, 0.55, 0.7, 0.9, 0.99)           # of a step
# dim, rotated elements, neighbours: pieces whose partners are pieces, neighbours, and other halves.
LAYOUTS = {"halves": (64, 64, False), "pairs": (64, 64, True), "odd_half": (64, 60, False)}


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    return torch, tod


def places(layout, pair):
    """The elements of a pair."""
    _, r, neighbours = LAYOUTS[layout]
    return (2 * pair, 2 * pair + 1) if neighbours else (pair, pair + r // 2)


def appended(torch, tod, x, pos, rates, layout, name):
    """(codes, scales) in a cache of the keys x [tokens, dim]."""
    t, dim = x.shape
    cache = tod.Cache4.zeros(t, 1, 1, dim)
    k = torch.from_numpy(x).to(dtype_of(torch, name)).cuda()[:, None]
    assert np.array_equal(f64(k)[:, 0], x)  # numbers of the type
    tod.tod_page_append4(k, k, k, torch.from_numpy(pos.astype(np.int32)).cuda(),
                         torch.arange(t, device="cuda"), torch.from_numpy(rates).cuda(), cache,
                         interleaved=LAYOUTS[layout][2])
    return cache.k_codes.cpu().numpy()[:, 0, 0], cache.k_scales.cpu().numpy()[:, 0, 0]


def compare(got, y, name, lo, hi):
    codes, scales = plain_encode(y, name)
    for i in range(len(y)):
        assert np.array_equal(got[1][i], scales[i]), (i, y[i, lo], got[1][i], scales[i])
        assert np.array_equal(got[0][i] & 0x77, codes[i] & 0x77), (i, y[i, lo], y[i, hi])


# shift: of all magnitudes, as a power of two.
@pytest.mark.parametrize("name,shift", [("fp16", 0), ("fp16", -9), ("bf16", 0), ("bf16", 40),
                                        ("bf16", -60)])
@pytest.mark.parametrize("layout", sorted(LAYOUTS))
def test_rotated_next_to_borders(env, layout, name, shift):
    torch, tod = env
    dim, r, _ = LAYOUTS[layout]
    pair, rate = 9, np.float32(1.37 * 2.0 ** -36)
    rates = np.zeros(r // 2, np.float32)
    rates[pair] = rate
    lo, hi = places(layout, pair)
    x, pos, near = [], [], []
    for b in BORDERS:
        for which in (lo, hi):        # the pair's first or second element is next to the border
            for sign in (1, -1):      # of the border
                for side in (1, -1):  # away from 0 or towards it
                    for part in PARTS:
                        # (Towards 0 from a power of two steps are half as long.)
                        step = float(np.spacing(np.float32(b)) if side > 0
                                     else np.float32(b) - np.nextafter(np.float32(b), np.float32(0)))
                        row = np.zeros(dim)
                        row[places(layout, 0)[0]] = 6.0  # not turned: the block's scale is 1
                        row[places(layout, 0)[1]] = 6.0
                        z = -1.0 if which == lo else 1.0
                        row[which] = sign * b
                        row[lo if which == hi else hi] = sign * z * side
                        x.append(row)
                        pos.append(round(part * step / float(rate)))
                        near.append((which, sign * b, step))
    x, pos = np.array(x) * 2.0 ** shift, np.array(pos)
    t = pos * float(rate)
    y = x.copy()
    y[:, lo] = x[:, lo] * np.cos(t) - x[:, hi] * np.sin(t)
    y[:, hi] = x[:, lo] * np.sin(t) + x[:, hi] * np.cos(t)
    for i, (which, b, step) in enumerate(near):
        off = abs(y[i, which] * 2.0 ** -shift - b)
        assert 2.0 ** -32 * abs(b) < off < step
    compare(appended(torch, tod, x, pos, rates, layout, name), y, name, lo, hi)


def turned(pos, rate):
    """Cosine and sine of pos * rate with the product's rounding and without it."""
    exact = Fraction(int(pos)) * Fraction(float(rate))
    a = float(exact)
    rest = float(exact - Fraction(a))
    c, s = math.cos(a), math.sin(a)
    return (c, s), (c * math.cos(rest) - s * math.sin(rest), s * math.cos(rest) + c * math.sin(rest))


@pytest.mark.parametrize("name", ["fp16", "bf16"])
@pytest.mark.parametrize("layout", sorted(LAYOUTS))
@pytest.mark.parametrize("least,most", [(0.3, 1.0), (1.0, 7.0)])  # 2^31 radians are passed
def test_far_positions(env, layout, name, least, most):
    torch, tod = env
    dim, r, _ = LAYOUTS[layout]
    rng = np.random.default_rng(29)
    bits = 11 if name == "fp16" else 8
    grid = np.concatenate([2.0 ** e * (1 + np.arange(2 ** (bits - 1)) / 2 ** (bits - 1))
                           for e in range(-6, 3)])
    rates = np.zeros(r // 2, np.float32)
    x, pos, y = [], [], []
    for pair in range(1, 15):
        lo, hi = places(layout, pair)
        rates[pair] = rng.uniform(least, most)
        for _ in range(16):
            p = int(rng.integers(2 ** 31 - 2 ** 28, 2 ** 31))
            (c0, s0), (c, s) = turned(p, rates[pair])
            for b in BORDERS[:-1]:
                # For each first element of a pair the second one that comes next to the border.
                z = (grid * c - b) / s
                at = np.searchsorted(grid, np.abs(z)).clip(1, len(grid) - 1)
                at -= np.abs(z) - grid[at - 1] < grid[at] - np.abs(z)
                z = np.copysign(grid[at], z)
                off, wrong = grid * c - z * s - b, grid * c0 - z * s0 - b
                for i in np.nonzero(((off > 0) != (wrong > 0)) & (np.abs(off) > 2.0 ** -38))[0][:4]:
                    row = np.zeros(dim)
                    row[places(layout, 0)[0]] = row[places(layout, 0)[1]] = 6.0
                    row[lo], row[hi] = grid[i], z[i]
                    x.append(row)
                    pos.append(p)
                    y.append(row.copy())
                    y[-1][lo] = row[lo] * c - row[hi] * s
                    y[-1][hi] = row[lo] * s + row[hi] * c
    assert len(x) >= 8
    got = appended(torch, tod, np.array(x), np.array(pos), rates, layout, name)
    compare(got, np.array(y), name, 0, 0)


@pytest.mark.parametrize("name", ["fp16", "bf16"])
@pytest.mark.parametrize("kind", ["keys", "values"])
def test_least_scale(env, name, kind):
    """Blocks whose scale is the least one: the borders of their codes, below the type's normal numbers
    or next to them, and the type's least numbers, unturned."""
    torch, tod = env
    unit = 2.0 ** (-23 if name == "fp16" else -125)
    least = 2.0 ** (-24 if name == "fp16" else -133)
    marks = [0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7]
    rows = []
    for top in (7.0, 3.5, 1.0):
        for by in (-2, -1, 0, 1, 2):
            row = np.zeros(32)
            row[0] = top * unit
            for i, m in enumerate(marks):
                row[i + 1] = (-1) ** i * min(m, top) * unit + by * least
            rows.append(np.round(row / least) * least)
    x = np.array(rows)
    x = f64(torch.from_numpy(x).to(dtype_of(torch, name)))  # numbers of the type
    k = torch.from_numpy(x).to(dtype_of(torch, name)).cuda()[:, None]
    n = len(x)
    cache = tod.Cache4.zeros(n, 1, 1, 32)
    tod.tod_page_append4(k, k, k, torch.zeros(n, dtype=torch.int32, device="cuda"),
                         torch.arange(n, device="cuda"), torch.ones(16, device="cuda"), cache)
    codes, scales = plain_encode(x, name)
    c, s = ((cache.k_codes, cache.k_scales) if kind == "keys"
            else (cache.v_codes, cache.v_scales))
    assert np.array_equal(s.cpu().numpy()[:, 0, 0], scales)
    assert np.array_equal(c.cpu().numpy()[:, 0, 0] & 0x77, codes & 0x77)
