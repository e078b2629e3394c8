"""Rotated keys at the ends of the floats' range: stored like the quantiser's
answer on the rotation in 64 bits."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from cache_model import quantise  # noqa: E402
from paper_2410_18234_gb300 import cache  # noqa: E402
from test_gpu_cache_rotary import DEV, DT, ints, turned, wide  # noqa: E402

LARGEST = float(np.finfo(np.float32).max)


def stored(k, r, interleaved=False):
    """What the cache holds of keys [n][H][D] from position 0 on, and what it should."""
    n, H, D = k.shape
    c = cache.Cache(1, -(-n // 128) + 1, H, D, 1, -(-n // 128) + 1, page_tokens=128,
                    dtype="f32" if k.dtype == torch.float32 else "bf16")
    c.reserve(ints([0]), n)
    c.append_rotated(0, ints([0]), k[None], torch.zeros_like(k[None]), r)
    got = wide(c.read(0, ints([0]), None, n)[0][0])
    new = turned(wide(k), np.arange(n), r.freqs, r.struct.dim, interleaved, r.struct.magnitude)[0]
    want = np.concatenate([np.stack([quantise(new[t:t + 16, h]) for h in range(H)], 1) for t in range(0, n, 16)])
    return got, want, c.status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("magnitude", [2.0 ** -9, 2.0 ** -10, 2.0 ** -12, 2.0 ** -20])
def test_pairs_of_the_largest_numbers_beside_large_ones(magnitude, interleaved, dtype):
    """|a| + |b| passes the largest float, and the block's step is decided by a
    number that does not turn: every stored number is finite and right."""
    rng = np.random.default_rng(4)
    k = rng.standard_normal((16, 2, 128)) * 2.0 ** 100
    k[:, :, :64] = rng.choice([-1.0, 1.0], (16, 2, 64)) * rng.uniform(0.8, 0.99, (16, 2, 64)) * 2.0 ** 128
    k[3, :, 100] = 2.75e38
    k = torch.tensor(k, device=DEV).to(DT[dtype])
    assert torch.isfinite(k).all()
    got, want, status = stored(k, cache.Rotary(64, magnitude=magnitude, interleaved=interleaved), interleaved)
    assert status == (0, "ok") and np.isfinite(got).all()
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("magnitude", [2.0 ** -9, 2.0 ** -10, 2.0 ** -11])
def test_borders_beside_large_numbers(magnitude):
    """Rotated numbers within 2^-23 of themselves of a border of the rounding,
    on either side, closer than 32-bit rotations tell: the exact ones decide."""
    rng = np.random.default_rng(5)
    n, H, top = 512, 2, 2.0 ** 119                       # the block's step: 1 is 2^119
    r = cache.Rotary(64, magnitude=magnitude)
    c, s = (turned(np.broadcast_to(x, (n, 1, 128)), np.arange(n), r.freqs, 64, False, magnitude)[0][:, 0, :32]
            for x in ((np.arange(128) < 32) * 1.0, (np.arange(128) // 32 == 1) * -1.0))
    k = np.zeros((n, H, 128))
    # of pair (a, b) the first becomes a c - b s: halfway between two numbers of four bits
    border = rng.choice([-1, 1], (n, H, 32)) * (rng.integers(8, 16, (n, H, 32)) + 0.5) / 8 * 2.0 ** rng.integers(-6, -4, (n, H, 32)) * top
    b = rng.standard_normal((n, H, 32)) * 0.004 * top / magnitude
    b = b.astype(np.float32).astype(float)
    a = (border + b * s[:, None]) / np.where(np.abs(c) > 0.4 * magnitude, c, 1e9)[:, None]
    k[..., :32], k[..., 32:64] = a, b
    k[::16, :, 127] = 2.9e38
    k = torch.tensor(k, device=DEV).float()
    assert torch.isfinite(k).all()
    got, want, status = stored(k, r)
    assert status == (0, "ok")
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pairs_of_zeros_among_the_least_numbers(dtype):
    """The largest step's inverse, 2^117, times a magnitude of 2^20 passes the
    largest float; pairs of zeros stay zeros."""
    rng = np.random.default_rng(7)
    k = rng.choice([0.0, 2.0 ** -133, -(2.0 ** -132)], (32, 2, 64))
    k[:, :, 8:16] = k[:, :, 24:32] = 0.0
    got, want, status = stored(torch.tensor(k, device=DEV).to(DT[dtype]), cache.Rotary(32, magnitude=1.9 * 2.0 ** 19))
    assert status == (0, "ok")
    np.testing.assert_array_equal(got, want if dtype == "f32" else wide(torch.tensor(want).bfloat16()))


def test_products_beyond_the_largest_float_whose_sums_are_not():
    """magnitude * a * cos is 1.05 of the largest float, the two rotated
    numbers are 7/8 of it, where the step's size is decided."""
    turn, to = math.radians(25), math.radians(20)
    r = cache.Rotary(16, freqs=[turn] * 8, magnitude=2.0)
    k = torch.zeros(2, 1, 64, device=DEV)
    size = math.sqrt(2) * 448 * 2.0 ** 119 / 2
    k[1, 0, 0], k[1, 0, 8], k[0, 0, 30] = size * math.cos(to), size * math.sin(to), 1e37
    assert 2 * float(k[1, 0, 0]) * math.cos(turn) > LARGEST
    got, want, status = stored(k, r)
    assert status == (0, "ok")
    np.testing.assert_array_equal(got, want)
    assert got[1, 0, 0] == got[1, 0, 8] == 448 * 2.0 ** 119


def test_rests_of_products_below_the_smallest_float():
    """(1 + 2^-30) * 2^-127 lies above the border between 0 and the least
    stored number, by less than a float this small can say."""
    r = cache.Rotary(16, magnitude=1 + 2.0 ** -30)
    k = torch.zeros(1, 1, 64, device=DEV)
    k[0, 0, 3], k[0, 0, 12], k[0, 0, 40] = 2.0 ** -127, -(2.0 ** -127), 2.0 ** -125
    got, want, status = stored(k, r)
    assert status == (0, "ok") and want[0, 0, 3] == 2.0 ** -126
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("magnitude", [2.0 ** -20, 1.1875, 1.9 * 2.0 ** 19])
def test_blocks_of_every_size(magnitude, dtype):
    """From the least floats to rotations of the largest."""
    rng = np.random.default_rng(6)
    n = 16 * 140
    most = min(126.0, 125 - math.log2(magnitude))
    size = np.repeat(np.linspace(-149, most - 4, n // 16), 16)[:, None, None]
    k = np.clip(rng.standard_normal((n, 2, 64)), -8, 8) * 2.0 ** size * 2.0 ** rng.uniform(-6, 0, (n, 2, 1))
    got, want, status = stored(torch.tensor(k, device=DEV).to(DT[dtype]), cache.Rotary(48, magnitude=magnitude))
    assert status == (0, "ok")
    np.testing.assert_array_equal(got, want if dtype == "f32" else wide(torch.tensor(want).bfloat16()))
