"""Sine and cosine of rotary positions on the GPU, against angles reduced in whole numbers."""
import math
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")
kmip = pytest.importorskip("paper_2604_03815_amd")

pytestmark = pytest.mark.gpu
BITS = 256


def inverse_two_pi():
    """2^BITS / (2 pi), to about the last bit, by Machin's formula."""
    one = 1 << (2 * BITS)

    def arctan_of(inverse):
        term = total = one // inverse
        n, sign = 1, 1
        while term:
            term //= inverse * inverse
            n, sign = n + 2, -sign
            total += sign * (term // n)
        return total

    return (one << BITS) // (8 * (4 * arctan_of(5) - arctan_of(239)))


INVERSE = inverse_two_pi()


def reduced(position, frequency):
    """position * frequency radians modulo a turn, in [-pi, pi]: off by 2^-52 of itself."""
    top, bottom = float(frequency).as_integer_ratio()
    turns = position * top * INVERSE // bottom               # times 2^BITS
    part = turns & ((1 << BITS) - 1)
    part -= (1 << BITS) if part >> (BITS - 1) else 0
    return 2 * math.pi * (part / (1 << BITS))


@pytest.mark.parametrize("seed,fast", [(1, 1.0), (2, 1.0), (3, 3000.0), (4, 1e-6), (5, 1e9)])
def test_sine_and_cosine(seed, fast):
    """Rows of (1, 0) pairs come out as (cos, sin) in float32: within 2^-22, and what the angle loses: 2^-28 radians, 2^-62 of it."""
    rng = random.Random(seed)
    positions = [0, 1, -1, 2 ** 31 - 1, -2 ** 31] + [rng.randint(-2 ** 31, 2 ** 31 - 1) for _ in range(300)] + \
        [rng.randint(0, 1 << rng.randint(1, 30)) for _ in range(300)]
    freqs = np.array([fast * 10000.0 ** (-i / 64) * rng.uniform(0.9, 1.1) for i in range(64)])
    x = torch.zeros(len(positions), 1, 128, device="cuda")
    x[..., :64] = 1.0
    got = kmip.rotary(x, None, torch.tensor(positions, dtype=torch.int32, device="cuda"), freqs)[:, 0].double().cpu().numpy()
    angle = np.array([[reduced(p, f) for f in freqs] for p in positions])
    far = np.abs(np.outer(positions, freqs)) * 2.0 ** -62
    bound = 2.0 ** -22 + 2.0 ** -28 + far
    assert (np.abs(got[:, :64] - np.cos(angle)) <= bound).all() and (np.abs(got[:, 64:] - np.sin(angle)) <= bound).all()


@pytest.mark.parametrize("rot", [128, 126])   # (runs of 16 bytes, and pair by pair)
def test_rows_past_32_bits(rot):
    """Rows behind the first 4 GB, turned in place, are what the same rows give by themselves; the others are zeros and stay zeros."""
    n, last, d = (1 << 24) + 3000, 300, 128
    freqs, _ = kmip.rotary_frequencies(rot)
    rows = torch.randn(last, 1, d, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    x = torch.zeros(n, 1, d, dtype=torch.bfloat16, device="cuda")
    x[-last:] = rows
    kmip.rotary(x, freqs=freqs, q_out=x)
    positions = torch.arange(n - last, n, dtype=torch.int32, device="cuda")
    assert torch.equal(x[-last:], kmip.rotary(rows, None, positions, freqs)) and not x[:-last].any()
