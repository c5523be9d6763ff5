"""Full attention and rotary positions without a GPU: refusals of the Python front end and of the C ABI (every call
fails before anything is launched), workspace sizes, frequencies, and the 64-bit reference against differences and autograd."""
import ctypes
import math
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")
kmip = pytest.importorskip("paper_2604_03815_amd")
from paper_2604_03815_amd import _lib  # noqa: E402

from full_reference import full64, sequences  # noqa: E402

BF, HF, SF = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2604_03815_amd import build
        build.build()
    return _lib.load()


def z(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype)


def good(**kw):
    a = dict(q=z(40, 4, 32), k_=z(50, 2, 32), v=z(50, 2, 16), scale=0.25)
    a.update(kw)
    return a


REFUSED = [
    (dict(q=z(40, 4, 32, dtype=SF)), TypeError, "float16"), (dict(k_=z(50, 2, 32, dtype=HF)), TypeError, "K must be"),
    (dict(v=z(50, 2, 16, dtype=SF)), TypeError, "V must be"), (dict(k_=z(50, 2, 64)), ValueError, "K must have"),
    (dict(k_=z(49, 2, 32)), ValueError, "K must have"), (dict(v=z(50, 1, 16)), ValueError, "K must have"),
    (dict(q=z(40, 128)), ValueError, "Q must be"), (dict(q=[1, 2]), ValueError, "Q must be"),
    (dict(q=z(40, 4, 64)[:, :, ::2]), ValueError, "last dimension"),
    (dict(out=z(40, 4, 32)), ValueError, "out must have"), (dict(out=z(40, 4, 16, dtype=SF)), TypeError, "out must be"),
    (dict(out=z(16, 4, 40).permute(2, 1, 0)), ValueError, "out"), (dict(lse=z(40, 4)), TypeError, "lse must be"),
    (dict(lse=z(40, 4, 1, dtype=SF)), ValueError, "lse must have"),
    (dict(graph_offsets=[0]), ValueError, "graph_offsets"), (dict(graph_offsets=[0, 2 ** 31]), ValueError, "graph_offsets"),
    (dict(graph_offsets=[0.0, 40.0]), ValueError, "graph_offsets"), (dict(graph_offsets=np.zeros((2, 2), int)), ValueError, "graph_offsets"),
    (dict(key_offsets=[0, 50]), ValueError, "key_offsets needs"), (dict(graph_offsets=[0, 40], key_offsets=[0, 1, 50]), ValueError, "key_offsets"),
    (dict(graph_offsets=[0, 40], key_offsets=[0, 50], key_lengths=[1, 2]), ValueError, "key_lengths"),
    (dict(), TypeError, "CUDA"),   # everything else in order: host tensors
]


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_forward_refuses(i):
    bad, kind, text = REFUSED[i]
    with pytest.raises(kind, match=text):
        kmip.full_fwd(**good(**bad))


@pytest.mark.parametrize("bad,kind,text", [
    (dict(dout=z(40, 4, 32)), ValueError, "dOut must have"), (dict(dout=z(40, 4, 16, dtype=SF)), TypeError, "dOut must be"),
    (dict(out=z(40, 4, 16, dtype=HF)), TypeError, "out must be"), (dict(lse=z(40, 3, dtype=SF)), ValueError, "lse must have"),
    (dict(dq=z(40, 4, 16)), ValueError, "dQ must have"), (dict(dk=z(50, 4, 32)), ValueError, "dK must have"),
    (dict(dv=z(50, 2, 32)), ValueError, "dV must have"), (dict(dv=z(50, 2, 16, dtype=SF)), TypeError, "dV must be"),
    (dict(), TypeError, "CUDA"),
])
def test_backward_refuses(bad, kind, text):
    a = good(dout=z(40, 4, 16), out=z(40, 4, 16), lse=z(40, 4, dtype=SF))
    a.update(bad)
    with pytest.raises(kind, match=text):
        kmip.full_bwd(**a)


F4 = np.ones(4)


@pytest.mark.parametrize("kw,kind,text", [
    (dict(q=z(5, 2, 16), freqs=None), ValueError, "freqs"), (dict(q=z(5, 32), freqs=F4), ValueError, "q must be"),
    (dict(q=torch.zeros(5, 2, 16, dtype=torch.float64), freqs=F4), TypeError, "q must be"),
    (dict(q=z(5, 2, 16), k_=z(4, 2, 16), freqs=F4), ValueError, "k must have"),
    (dict(q=z(5, 2, 16), k_=z(5, 2, 16, dtype=SF), freqs=F4), TypeError, "k must be"),
    (dict(q=z(5, 2, 16), freqs=np.ones((2, 2))), ValueError, "freqs"), (dict(q=z(5, 2, 16), freqs=F4, dtype=torch.int32), TypeError, "dtype"),
    (dict(q=z(5, 2, 16), freqs=F4, positions=torch.zeros(5)), TypeError, "positions"),
    (dict(q=z(5, 2, 16), freqs=F4, positions=torch.zeros(4, dtype=torch.int32)), ValueError, "positions"),
    (dict(q=z(5, 2, 16), freqs=F4, q_out=z(5, 2, 8)), ValueError, "q_out"),
    (dict(q=z(5, 2, 16), freqs=F4, q_out=z(5, 1, 16).expand(5, 2, 16)), ValueError, "overlaps"),
    (dict(q=z(5, 2, 16), freqs=F4, q_out=z(1, 2, 16).expand(5, 2, 16)), ValueError, "overlaps"),
    (dict(q=z(5, 2, 16), freqs=F4, k_out=z(5, 2, 16)), ValueError, "k_out"),
    (dict(q=z(5, 2, 16).requires_grad_(), freqs=F4, q_out=z(5, 2, 16)), ValueError, "differentiable"),
    (dict(q=z(5, 2, 16), freqs=F4), TypeError, "CUDA"),
])
def test_rotary_refuses(kw, kind, text):
    with pytest.raises(kind, match=text):
        kmip.rotary(**kw)


P = ctypes.c_void_p
FAKE = P(256)   # never dereferenced: every call below fails its checks


def _i32(x):
    return None if x is None else np.ascontiguousarray(x, np.int32).ctypes.data_as(P)


def _fwd(lib, q=FAKE, dtype=0, strides=None, qo=None, ko=None, kl=None, G=1, Nq=64, Nk=64, H=2, Hk=1, d=32, dv=32, scale=0.5,
         out=FAKE, ws=None, ws_bytes=0):
    keep = [None if x is None else np.ascontiguousarray(x, np.int32) for x in (qo, ko, kl)]
    st = None if strides is None else np.ascontiguousarray(strides, np.int64)
    return lib.kmip_full_fwd(q, FAKE, FAKE, dtype, None if st is None else st.ctypes.data_as(P),
                             *(None if x is None else x.ctypes.data_as(P) for x in keep), G, Nq, Nk, H, Hk, d, dv, scale, 0, out, FAKE,
                             ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(d=24), 2), (dict(dv=256), 2), (dict(dtype=2), 2), (dict(dtype=-1), 2), (dict(H=3, Hk=2), 1), (dict(H=0), 1), (dict(Hk=0), 1),
    (dict(Nq=-1), 1), (dict(Nk=1 << 31), 1), (dict(Nq=1 << 30, H=4), 1), (dict(scale=0.0), 1), (dict(scale=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(q=None), 1), (dict(q=P(264)), 1), (dict(out=P(264)), 1), (dict(out=None), 1),
    (dict(strides=[64, 32, 32, 32, 32, 36]), 1), (dict(strides=[64, -8, 32, 32, 32, 32]), 1), (dict(strides=[1 << 23, 32, 32, 32, 32, 32]), 2),
    (dict(qo=[0, 63]), 1), (dict(qo=[1, 64]), 1), (dict(qo=[0, 40, 30, 64], G=3), 1), (dict(qo=[0, 64], G=0), 1),
    (dict(ko=[0, 64]), 1), (dict(qo=[0, 64], ko=[0, 60]), 1), (dict(qo=[0, 64], kl=[65]), 1), (dict(kl=[65]), 1), (dict(kl=[-1]), 1),
    (dict(Nk=200000, Nq=1), 3), (dict(Nk=200000, Nq=1, ws=P(8), ws_bytes=1 << 40), 3), (dict(Nk=200000, Nq=1, ws=FAKE, ws_bytes=64), 3),
])
def test_abi_refuses(lib, kw, status):
    assert _fwd(lib, **kw) == status
    assert lib.kmip_last_error()


def test_abi_backward_refuses(lib):
    def bwd(**kw):
        a = dict(dout=FAKE, dq=FAKE, ws=FAKE, nbytes=1 << 40, d=32)
        a.update(kw)
        return lib.kmip_full_bwd(FAKE, FAKE, FAKE, a["dout"], FAKE, FAKE, 0, None, None, None, None, 1, 64, 64, 2, 1, a["d"], 32, 0.5, 0,
                                 a["dq"], FAKE, FAKE, a["ws"], a["nbytes"], None)

    assert bwd(dout=None) == 1 and bwd(dq=None) == 1 and bwd(dq=P(264)) == 1 and bwd(dout=P(264)) == 1 and bwd(d=8) == 2
    assert bwd(ws=None) == 3 and bwd(nbytes=8) == 3 and bwd(ws=P(264)) == 3


def test_abi_rotary_refuses(lib):
    f = np.ones(64)

    def rot(x=FAKE, y=FAKE, H=2, x2=None, y2=None, H2=0, ti=0, to=0, strides=None, freqs=f, N=10, d=32, rot=32, m=1.0):
        st = None if strides is None else np.ascontiguousarray(strides, np.int64)
        return lib.kmip_rotary(x, y, H, x2, y2, H2, ti, to, None if st is None else st.ctypes.data_as(P), None,
                               None if freqs is None else freqs.ctypes.data_as(P), N, d, rot, 0, m, 0, None)

    assert rot(d=31) == 2 and rot(d=258) == 2 and rot(ti=3) == 2 and rot(to=-1) == 2
    for bad in (dict(rot=34), dict(rot=31), dict(rot=0), dict(H=0), dict(H2=-1), dict(N=-1), dict(N=1 << 31), dict(freqs=None),
                dict(freqs=np.full(64, np.inf)), dict(freqs=np.full(64, np.nan)), dict(m=float("inf")), dict(x=None), dict(H2=1),
                dict(x=P(257)), dict(to=2), dict(strides=[64, 32, 96, 32, 0, 0, 0, 0]), dict(strides=[64, -32, 64, -32, 0, 0, 0, 0])):
        assert rot(**bad) == 1, bad
    assert rot(N=0) == 0


def test_workspace_sizes(lib):
    # none where no sequence has 1024 keys
    assert kmip.full_fwd_workspace_size(1, 1023, 8, 1, 64, 64) == 0
    assert kmip.full_fwd_workspace_size(100 * 1023, 100 * 1023, 8, 1, 64, 64, graph_offsets=[1023 * i for i in range(101)]) == 0
    # one token over a long cache: runs of its keys, each with its rows' sums (64 floats) and two figures
    n = kmip.full_fwd_workspace_size(1, 65537, 8, 1, 64, 64)
    assert n > 0 and n % 256 == 0 and n <= 256 * 32 * (64 + 2) * 4
    assert kmip.full_fwd_workspace_size(1, 65537, 8, 1, 24, 64) == 0   # refused sizes
    assert kmip.full_bwd_workspace_size(100, 100, 4, 2, 32, 32) == 2 * ((100 * 4 * 4 + 255) // 256 * 256)


def test_rotary_frequencies():
    f, m = kmip.rotary_frequencies(8, base=100.0)
    assert m == 1.0 and np.allclose(f, [100.0 ** (-2 * i / 8) for i in range(4)])
    g, m = kmip.rotary_frequencies(8, base=100.0, scaling="linear", factor=4.0)
    assert m == 1.0 and np.allclose(g, f / 4)
    g, m = kmip.rotary_frequencies(8, base=100.0, scaling="base", factor=4.0)
    assert m == 1.0 and math.isclose(g[0], 1.0) and math.isclose(g[-1], f[-1] / 4) and (np.diff(g) < 0).all()
    g, m = kmip.rotary_frequencies(64, scaling="blend", factor=4.0, original_length=4096)
    f, _ = kmip.rotary_frequencies(64)
    turns = 4096 * f / (2 * math.pi)
    assert math.isclose(m, 0.1 * math.log(4) + 1)
    assert np.allclose(g[turns >= 32], f[turns >= 32]) and np.allclose(g[turns <= 1], f[turns <= 1] / 4)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and (g[mid] < f[mid]).all() and (g[mid] > f[mid] / 4).all()
    for bad in (dict(rot=7), dict(rot=8, base=0.0), dict(rot=8, factor=-1.0), dict(rot=8, scaling="x"), dict(rot=8, scaling="blend")):
        with pytest.raises(ValueError):
            kmip.rotary_frequencies(**bad)


def test_layer_refuses():
    with pytest.raises(ValueError):
        kmip.FullAttention(64, 4, 16, kv_heads=3)
    with pytest.raises(ValueError):
        kmip.FullAttention(64, 4, 16, rotary=kmip.Rotary(32))
    with pytest.raises(ValueError):
        kmip.KMIPAttention(64, 4, 16, rotary=kmip.Rotary(32))
    layer = kmip.FullAttention(64, 4, 16, rotary=kmip.Rotary(16))
    with pytest.raises(ValueError, match="positions"):
        layer(torch.zeros(10, 64), graph_offsets=[0, 4, 10])
    with pytest.raises(ValueError, match="rotary"):
        kmip.FullAttention(64, 4, 16)(torch.zeros(10, 64), positions=torch.zeros(10, dtype=torch.int32))
    with pytest.raises(ValueError, match="x must be"):
        layer(torch.zeros(10, 32))


CASES = [(3, 5, 2, 1, False), (5, 3, 2, 2, True), (4, 6, 4, 2, True), (1, 1, 1, 1, True)]


@pytest.mark.parametrize("m,n,H,Hk,causal", CASES)
def test_reference(m, n, H, Hk, causal):
    """The 64-bit gradients against autograd of the plain formula, and against central differences of the reference's own forward."""
    gen = torch.Generator().manual_seed(m * 100 + n)
    q, k, v, g = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((m, H, 4), (n, Hk, 4), (n, Hk, 3), (m, H, 3)))
    q, k, v, g = (t.to(SF) for t in (q, k, v, g))
    seqs = sequences(m, n)
    want = full64(q, k, v, 0.7, seqs, causal, g)
    Q, K, V = (t.double().requires_grad_() for t in (q, k, v))
    s = 0.7 * torch.einsum("mhd,nhd->hmn", Q, K.repeat_interleave(H // Hk, 1))
    hide = torch.ones(m, n, dtype=torch.bool).triu(n - m + 1) if causal else torch.zeros(m, n, dtype=torch.bool)
    p = torch.softmax(s.masked_fill(hide, -math.inf), -1).nan_to_num(0.0)
    out = torch.einsum("hmn,nhd->mhd", p, V.repeat_interleave(H // Hk, 1))
    assert torch.allclose(out, want["out"][0], atol=1e-12)
    if not (hide.all(1)).any():
        for x, name in zip(torch.autograd.grad(out, (Q, K, V), g.double()), ("dq", "dk", "dv")):
            assert torch.allclose(x, want[name][0], atol=1e-12)
    h = 2.0 ** -10
    for t, name in ((q, "dq"), (k, "dk"), (v, "dv")):
        for at in np.ndindex(*t.shape):
            values = []
            for step in (h, -h):
                t2 = t.double().clone()
                t2[at] += step
                args = [t2 if t is x else x.double() for x in (q, k, v)]
                values.append((full64(*(_as32(a) for a in args), 0.7, seqs, causal)["out"][0] * g.double()).sum().item())
            assert abs((values[0] - values[1]) / (2 * h) - want[name][0][at].item()) < 1e-5


class _as32:
    """A float64 tensor that says it is float32, for the reference's table of steps."""

    def __init__(self, t):
        self.t = t
        self.dtype, self.shape, self.device = SF, t.shape, t.device

    def __len__(self):
        return len(self.t)

    def __getitem__(self, at):
        return self.t[at]
