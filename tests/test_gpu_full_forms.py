"""Every form of full attention's kernels at every pair of widths, in both types, on the GPU against 64 bits."""
import pytest

torch = pytest.importorskip("torch")
kmip = pytest.importorskip("paper_2604_03815_amd")

from full_forms import FORMS, PAIRS, case  # noqa: E402
from full_reference import check, full64, sequences  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.mark.parametrize("d,dv", PAIRS)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("name", list(FORMS))
def test_form(name, dtype, d, dv):
    H, Hk, qo, ko = case(name)
    gen = torch.Generator(device="cuda").manual_seed(17 * d + dv)
    q, k, v, g = (torch.randn(*s, generator=gen, device="cuda").to(TYPES[dtype])
                  for s in ((qo[-1], H, d), (ko[-1], Hk, d), (ko[-1], Hk, dv), (qo[-1], H, dv)))
    where, scale = dict(graph_offsets=qo, key_offsets=ko), d ** -0.5
    out, lse = kmip.full_fwd(q, k, v, scale, causal=True, **where)
    grads = kmip.full_bwd(q, k, v, g, out, lse, scale, causal=True, **where)
    want = full64(q, k, v, scale, sequences(len(q), len(k), **where), True, g)
    for got, key in zip((out, lse, *grads), ("out", "lse", "dq", "dk", "dv")):
        check(key, got, want[key])
