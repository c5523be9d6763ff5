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
