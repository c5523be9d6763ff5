"""Full attention at the ends of its ranges, on the GPU."""
import math

import pytest

torch = pytest.importorskip("torch")
kmip = pytest.importorskip("paper_2604_03815_amd")

pytestmark = pytest.mark.gpu
BF, HF, SF = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("m,nk", [(1, 2 ** 31 - 5000), (40, 2 ** 31 - 4097)])
def test_most_keys(m, nk):
    """As many keys as a call takes, all the same row (a stride of 0): every one of them is counted."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = torch.zeros(m, 1, 16, dtype=BF, device="cuda")
    k, v = (torch.randn(1, 1, 16, generator=gen, device="cuda").to(BF) for _ in range(2))
    out, lse = kmip.full_fwd(q, k.expand(nk, 1, 16), v.expand(nk, 1, 16), 0.25)
    # every weight is 1: a lane's sum is a whole number below 2^24; at most 1024 runs are added, 2^-24 each; the log's own step.
    # (A run left out is 2^-10 of the keys.)
    assert (lse.double() - math.log(nk)).abs().max() <= 2.0 ** -14 + 2.0 ** -18
    # a run's sums are of at most 2^16 equal parts, off by 2^-24 of what is there at each: 2^-9 in all; and the result's half step
    assert ((out.double() - v.double()).abs() <= (2.0 ** -8 + 2.0 ** -9) * v.double().abs()).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("scale", [2.0 ** -149, 1e-40, 2.0 ** -126, 1e-30])
@pytest.mark.parametrize("m,n", [(5, 70), (3, 2000), (700, 260)])
def test_smallest_scales(m, n, scale, dtype):
    """Scales down to the smallest float32: every key that a row sees has the same weight, and rows that see none stay empty."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(rows, 2, 32, generator=gen, device="cuda").to(dtype) for rows in (m, n, n))
    out, lse = kmip.full_fwd(q, k, v, scale, causal=True)
    sees = (torch.arange(m, device="cuda") + 1 + n - m).clamp(min=0)
    none = sees == 0
    assert (out[none] == 0).all() and (lse[none] == -math.inf).all()
    # the log of a whole number in 32 bits, from a sum that is exact
    assert (lse[~none].double() - sees[~none].double().log()[:, None]).abs().max() <= 2.0 ** -20
    total = v.double().cumsum(0)[sees[~none] - 1] / sees[~none][:, None, None]
    size = v.double().abs().cumsum(0)[sees[~none] - 1] / sees[~none][:, None, None]
    u = torch.finfo(dtype).eps / 2
    assert ((out[~none].double() - total).abs() <= u * total.abs() + n * 2.0 ** -23 * size + (2.0 ** -25 if dtype == HF else 0)).all()
