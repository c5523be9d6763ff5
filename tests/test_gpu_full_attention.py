"""Full softmax attention on the GPU against 64 bits: out and lse within derived bounds, element by element."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
kmip = pytest.importorskip("paper_2604_03815_amd")

from full_reference import check, full64, sequences  # noqa: E402

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def make(seed, nq, nk, H, Hk, d, dv, dtype):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

    return normal(nq, H, d), normal(nk, Hk, d), normal(nk, Hk, dv), normal(nq, H, dv)


def sums(x):
    return np.concatenate([[0], np.cumsum(x)]).tolist()


# (queries, keys) of each sequence; None: one sequence of these
CASES = [
    # one token, one key; one query and one key more or less than a block and a tile
    (BF, 1, 1, 16, 16, [(1, 1)], False), (HF, 1, 1, 128, 128, [(1, 1)], True),
    (BF, 2, 2, 32, 32, [(31, 31), (32, 32), (33, 33), (63, 65), (64, 64), (65, 63)], False),
    (BF, 4, 2, 64, 64, [(1, 33), (33, 1), (127, 129), (128, 128), (129, 127)], True),
    (HF, 8, 1, 128, 128, [(3, 300), (5, 5), (17, 40)], True),
    # empty on either side, queries that see nothing
    (BF, 3, 3, 32, 32, [(0, 0), (5, 0), (0, 7), (9, 4), (4, 9)], True),
    (BF, 3, 1, 16, 16, [(0, 3), (40, 0), (50, 13)], False),
    # widths of their own
    (BF, 2, 1, 16, 128, [(45, 70)], False), (HF, 2, 2, 128, 16, [(70, 45)], True), (BF, 4, 2, 32, 64, [(100, 100)], True),
    (HF, 1, 1, 64, 32, [(37, 200)], False),
    # single tokens over long caches, few and many heads on a key head
    (BF, 8, 1, 64, 64, [(1, 5001)], True), (BF, 32, 8, 128, 128, [(1, 1), (1, 2000), (1, 3), (2, 777)], True),
    (HF, 40, 1, 32, 32, [(1, 3333), (3, 64)], True), (BF, 1, 1, 16, 16, [(2, 20000)], False),
    # enough rows for tiles of 128
    (BF, 8, 8, 64, 64, [(4097, 4097)], True), (HF, 16, 4, 128, 128, [(700, 1300), (1500, 1500), (1, 9)], True),
    (BF, 16, 16, 32, 32, [(2100, 2100), (33, 129)], False), (BF, 33, 11, 16, 16, [(1000, 1000), (1, 64), (129, 1)], True),
    (HF, 12, 4, 64, 128, [(3000, 2900)], True),
    # every pair of widths, in both forms
    *[(BF if i % 2 else HF, 2, 1, d, dv, [(33 + i, 70), (5, 129)], i % 3 == 0)
      for i, (d, dv) in enumerate((a, b) for a in (16, 32, 64, 128) for b in (16, 32, 64, 128) if a != b)],
    *[(HF if i % 2 else BF, 16, 8, d, dv, [(1100, 2100), (997, 1200)], i % 3 != 0)
      for i, (d, dv) in enumerate((a, b) for a in (16, 32, 64, 128) for b in (16, 32, 64, 128))],
    # tiles of 128 rows or keys whose streams are cut into runs
    (BF, 8, 2, 128, 128, [(2048, 4096), (7, 100)], True), (BF, 4, 4, 128, 32, [(3001, 2999)], True),
    (HF, 2, 1, 16, 128, [(5000, 6001)], False), (BF, 6, 2, 32, 32, [(900, 7000), (1, 5), (700, 1100)], True),
    (BF, 1, 1, 16, 16, [(9001, 9001)], False), (HF, 8, 1, 64, 64, [(1500, 1500), (0, 300), (40, 0)], True), (BF, 3, 3, 32, 32, [(n, n) for n in range(100, 451, 3)] , False),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_forward(i):
    dtype, H, Hk, d, dv, lens, causal = CASES[i]
    ql, kl = zip(*lens)
    q, k, v, _ = make(i, sum(ql), sum(kl), H, Hk, d, dv, dtype)
    scale = 1.0 / math.sqrt(d)
    where = dict(graph_offsets=sums(ql), key_offsets=sums(kl))
    out, lse = kmip.full_fwd(q, k, v, scale, causal=causal, **where)
    want = full64(q, k, v, scale, sequences(len(q), len(k), **where), causal)
    assert out.dtype == dtype and lse.dtype == torch.float32
    check("out", out, want["out"])
    check("lse", lse, want["lse"])
    again = kmip.full_fwd(q, k, v, scale, causal=causal, **where)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("i", range(len(CASES)))
def test_backward(i):
    dtype, H, Hk, d, dv, lens, causal = CASES[i]
    ql, kl = zip(*lens)
    q, k, v, dout = make(100 + i, sum(ql), sum(kl), H, Hk, d, dv, dtype)
    scale = 1.0 / math.sqrt(d)
    where = dict(graph_offsets=sums(ql), key_offsets=sums(kl))
    out, lse = kmip.full_fwd(q, k, v, scale, causal=causal, **where)
    got = kmip.full_bwd(q, k, v, dout, out, lse, scale, causal=causal, **where)
    want = full64(q, k, v, scale, sequences(len(q), len(k), **where), causal, dout)
    for name, x in zip(("dq", "dk", "dv"), got):
        assert x.dtype == dtype
        check(name, x, want[name])
    again = kmip.full_bwd(q, k, v, dout, out, lse, scale, causal=causal, **where)
    for x, y in zip(got, again):
        assert torch.equal(x, y)
