"""Full attention at the ends of its ranges, on the GPU."""
import math

import pytest

torch = pytest.importorskip("torch")
kmip = pytest.importorskip("paper_2604_03815_amd")

from full_reference import check, full64, sequences  # noqa: E402

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


@pytest.mark.parametrize("m,n", [(1, 50_001), (40, 50_001), (1, 300_003), (2048, 30_011)])
def test_many_alike_keys_backward_float16(m, n):
    """Weights of 1 / n, among or below float16's subnormal numbers: their products with dout keep their bits."""
    q, k = (torch.zeros(rows, 1, 16, dtype=HF, device="cuda") for rows in (m, n))
    gen = torch.Generator(device="cuda").manual_seed(1)
    v, g = (torch.randn(rows, 1, 16, generator=gen, device="cuda").to(HF) for rows in (n, m))
    g = (g.abs() + 1.0) * 64.0
    out, lse = kmip.full_fwd(q, k, v, 0.25)
    dv = kmip.full_bwd(q, k, v, g, out, lse, 0.25)[2]
    want = g.double().sum(0) / n
    # a weight off by half a step (2^-11), its exponent by lse's and its own roundings (2^-22 of 17.4 at most), m sums in 32 bits,
    # the result's half step (2^-25 among subnormal numbers)
    bound = want * (2.0 ** -11 + 2.0 ** -17 + m * 2.0 ** -24 + 2.0 ** -11) + 2.0 ** -25
    assert ((dv.double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("size", [2.0 ** 8, 2.0 ** 12, 2.0 ** 16, 2.0 ** 20])
@pytest.mark.parametrize("m,n", [(3, 90), (700, 700)])
def test_gradients_of_large_scores(m, n, size, dtype):
    """Scores of about `size`, of either sign, that differ by a few: weights come back from one float32 lse, off by |lse| 2^-22
    in their exponent, which the reference's bound holds (2 (|scale s| 2^-22 and the product's own))."""
    H, d = 2, 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, g = (torch.randn(rows, H, d, generator=gen, device="cuda") for rows in (m, n, n, m))
    # one dimension makes the size, the others the differences
    k = k * (0.5 if size <= 2.0 ** 12 else 8.0)
    q[..., 0] = size ** 0.5
    q[:, 1, 0] *= -1.0
    k[..., 0] = size ** 0.5
    q, k, v, g = (t.to(dtype) for t in (q, k, v, g))
    out, lse = kmip.full_fwd(q, k, v, 1.0, causal=True)
    dq, dk, dv = kmip.full_bwd(q, k, v, g, out, lse, 1.0, causal=True)
    want = full64(q, k, v, 1.0, sequences(m, n), True, g)
    # The reference's bound is relative, and scores 2^8 apart give weights below the smallest normal float32, 2^-126, for which 0
    # may come out.  Up to 700 of them meet |dp - D| <= 2 * 16 * 5 * 5 < 2^10 and |q|, |k| <= 2^10: 2^9.5 * 2^20 * 2^-126 < 2^-96.
    for name, x in dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv).items():
        value, bound = want[name]
        check(name, x, (value, bound + 2.0 ** -96))


@pytest.mark.parametrize("slope", [0.02, -0.02])
def test_gradients_of_scores_far_apart(slope):
    """Scores that rise and fall by hundreds from tile to tile: every gradient."""
    n, d = 700, 64
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, k, v, g = (torch.randn(n, 2, d, generator=gen, device="cuda").to(HF) for _ in range(4))
    steep = (k.float() * 0.1 + slope * torch.arange(n, device="cuda")[:, None, None] * torch.sign(q[:1].float())).to(HF)
    same = q[:1].expand(n, 2, d).contiguous()
    out, lse = kmip.full_fwd(same, steep, v, 1.0)
    dq, dk, dv = kmip.full_bwd(same, steep, v, g, out, lse, 1.0)
    want = full64(same, steep, v, 1.0, sequences(n, n), False, g)
    for name, x in dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv).items():
        check(name, x, want[name])


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("d,dv", [(16, 16), (64, 64), (128, 128)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("m", [50, 4096])
def test_gradients_that_are_not_finite(m, bad, d, dv, dtype):
    """An infinity or a NaN in dout comes out in the gradients it enters, and in no other sequence's."""
    H, offsets = 2, [0, m, m + 70]
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, g = (torch.randn(m + 70, H, w, generator=gen, device="cuda").to(dtype) for w in (d, d, dv, dv))
    row, head, column = m // 2, 1, 5
    clean = []
    for value in (1.0, bad):
        g[row, head, column] = value
        out, lse = kmip.full_fwd(q, k, v, d ** -0.5, graph_offsets=offsets, causal=True)
        clean.append(kmip.full_bwd(q, k, v, g, out, lse, d ** -0.5, graph_offsets=offsets, causal=True))
    (dq0, dk0, dv0), (dq, dk, dvv) = clean
    assert not torch.isfinite(dq[row, head]).any()
    assert not torch.isfinite(dk[:row + 1, head]).any() and not torch.isfinite(dvv[:row + 1, head, column]).any()
    for x, y in ((dq, dq0), (dk, dk0), (dvv, dv0)):
        assert torch.equal(x[m:], y[m:]) and torch.equal(x[:m, 0], y[:m, 0])


def test_overflow_of_float16_gradients():
    """dout so large that p (dp - D) passes 65504: not finite, so that a scaled loss is seen to be scaled too far."""
    q, k = (torch.zeros(n, 1, 16, dtype=HF, device="cuda") for n in (3, 2))
    k[:] = 1.0   # (alike keys: both weights are 1/2)
    v = torch.zeros(2, 1, 16, dtype=HF, device="cuda")
    v[0], v[1] = 30.0, -30.0
    g = torch.full((3, 1, 16), 1.0, dtype=HF, device="cuda")
    g[1] = 1000.0   # dp = +-480,000, D = 0
    out, lse = kmip.full_fwd(q, k, v, 1.0)
    dq, dk, dv = kmip.full_bwd(q, k, v, g, out, lse, 1.0)
    assert torch.isfinite(dq[[0, 2]]).all() and not torch.isfinite(dq[1]).any()
    assert not torch.isfinite(dk).any()
    assert torch.equal(dv, torch.full_like(dv, 501.0))


def test_queries_past_32_bits():
    """Queries, gradients and results behind the first 4 GB of their tensors; the rows before them see no key."""
    far, m, n, H, d = (1 << 23) + 1000, 77, 130, 2, 128
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(n, 1, d, generator=gen, device="cuda").to(BF) for _ in range(2))
    q, g = (torch.zeros(far + m, H, d, dtype=BF, device="cuda") for _ in range(2))
    q[far:], g[far:] = (torch.randn(m, H, d, generator=gen, device="cuda").to(BF) for _ in range(2))
    where = dict(graph_offsets=[0, far, far + m], key_offsets=[0, 0, n])
    out, lse = kmip.full_fwd(q, k, v, 0.1, causal=True, **where)
    dq, dk, dv = kmip.full_bwd(q, k, v, g, out, lse, 0.1, causal=True, **where)
    assert not out[:far].any() and (lse[:far] == -math.inf).all() and not dq[:far].any()
    want = full64(q[far:], k, v, 0.1, sequences(m, n), True, g[far:])
    for name, x in dict(out=out[far:], lse=lse[far:], dq=dq[far:], dk=dk, dv=dv).items():
        check(name, x, want[name])


@pytest.mark.parametrize("d,dv", [(16, 16), (128, 128), (32, 64)])
@pytest.mark.parametrize("m", [150, 20])
def test_rows_far_apart(m, d, dv):
    """Rows as far apart as a call takes them (2^23 - 8 values): views give what their copies give."""
    n, stride = 150, 2 ** 23 - 8
    H, Hk = (256, 256) if m == 150 else (4, 2)   # (tiles of 128 rows, of 32)
    gen = torch.Generator(device="cuda").manual_seed(1)
    whole = torch.zeros(n * stride, dtype=BF, device="cuda")
    at, views = 0, []
    for rows, heads, width in ((m, H, d), (n, Hk, d), (n, Hk, dv), (m, H, dv)):
        view = torch.as_strided(whole, (rows, heads, width), (stride, width, 1), at)
        view.copy_(torch.randn(rows, heads, width, generator=gen, device="cuda").to(BF))
        views.append(view)
        at += heads * width
    results = []
    for q, k, v, g in (views, [t.contiguous() for t in views]):
        out, lse = kmip.full_fwd(q, k, v, 0.1)
        results.append((out, lse, *kmip.full_bwd(q, k, v, g, out, lse, 0.1)))
    for x, y in zip(*results):
        assert torch.equal(x, y)
