"""Full attention and rotary positions as they are called: views, caches with room, long offsets, many sequences, other
streams, captured graphs, autograd, the layers, and the two together."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
kmip = pytest.importorskip("paper_2604_03815_amd")

from full_reference import check, full64, sequences  # noqa: E402
from test_gpu_rotary import check as check_turned, turned64  # noqa: E402

pytestmark = pytest.mark.gpu
BF, HF, SF = torch.bfloat16, torch.float16, torch.float32


def normal(seed, *shape, dtype=BF):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=gen, device="cuda").to(dtype)


def sums(x):
    return np.concatenate([[0], np.cumsum(x)]).tolist()


def both(q, k, v, g, scale, causal=False, **where):
    out, lse = kmip.full_fwd(q, k, v, scale, causal=causal, **where)
    return dict(zip(("out", "lse", "dq", "dk", "dv"),
                    (out, lse, *kmip.full_bwd(q, k, v, g, out, lse, scale, causal=causal, **where))))


def against64(got, q, k, v, g, scale, causal=False, **where):
    want = full64(q, k, v, scale, sequences(len(q), len(k), **where), causal, g)
    for name, x in got.items():
        check(name, x, want[name])


@pytest.mark.parametrize("n,heads,d", [(77, 4, 32), (700, 8, 128)])
def test_views(n, heads, d):
    """Slices of a fused projection, heads-first tensors and shared heads by stride 0 give what their copies give."""
    fused = normal(1, n, 3 * heads, d)
    views = [
        (fused[:, :heads], fused[:, heads:2 * heads], fused[:, 2 * heads:]),
        tuple(normal(s, heads, n, d).transpose(0, 1) for s in (2, 3, 4)),
        (normal(5, n, heads, d), normal(6, n, 1, d).expand(n, heads, d), normal(7, n, heads, 2 * d)[:, :, :d]),
        (normal(8, 2 * n, heads, d)[::2], normal(9, 1, heads, d).expand(n, heads, d), normal(10, n, heads, d)),
    ]
    for q, k, v in views:
        for g in (normal(11, heads, n, d).transpose(0, 1), normal(12, n, heads, d)):
            got = both(q, k, v, g, d ** -0.5, causal=True)
            want = both(q.contiguous(), k.contiguous(), v.contiguous(), g.contiguous(), d ** -0.5, causal=True)
            for name in got:
                assert got[name].is_contiguous() and torch.equal(got[name], want[name]), name
    q, k, v = views[0]
    with pytest.raises(kmip.KmipError):   # rows that start off a 16-byte step
        kmip.full_fwd(normal(13, n, heads, d + 4)[:, :, :d], k, v, 1.0)


def test_strides_of_single_rows_and_far_gradients():
    """Strides of dimensions of one do not matter; rows of dout too far apart for the kernels are copied."""
    q, k, v, g = normal(1, 1, 2, 32), normal(2, 90, 2, 64)[:, :, :32], normal(3, 90, 2, 32), normal(4, 1, 2, 32)
    q = torch.as_strided(q, (1, 2, 32), (7, 32, 1))
    got, want = both(q, k, v, g, 0.2), both(q.contiguous(), k.contiguous(), v, g, 0.2)
    for name in got:
        assert torch.equal(got[name], want[name]), name
    q, k, v = (normal(s, 3, 2, 32).requires_grad_() for s in (5, 6, 7))
    far = torch.zeros(3, 1 << 23, dtype=BF, device="cuda")
    far[:, :64] = normal(8, 3, 64)
    g = far[:, :64].view(3, 2, 32)
    out = kmip.full_attention(q, k, v, 0.2)
    for x, y in zip(torch.autograd.grad(out, (q, k, v), g, retain_graph=True), torch.autograd.grad(out, (q, k, v), g.contiguous())):
        assert torch.equal(x, y)


@pytest.mark.parametrize("m", [1, 300])
def test_small_float16_weights(m):
    """One key outweighs each other one by e^12.2 and has value 0: the result is the sum of 4,000 like, small weights."""
    n, d = 4001, 16
    q, k, v = (torch.zeros(*s, 1, d, dtype=HF, device="cuda") for s in ((m,), (n,), (n,)))
    q[..., 0] = 1.0
    k[..., 0] = 0.3
    k[0, 0, 0] = 12.5
    v[1:] = 4096.0
    out, lse = kmip.full_fwd(q, k, v, 1.0)
    s = k[:, 0, 0].double()
    want = torch.softmax(s, 0)[1:].sum() * 4096.0
    # every weight off by half a step of its own (2^-11), the result by another; n additions in 32 bits, for the sum and
    # its normaliser, by at most 2^-24 each; scores and exponentials by 2^-20.  (A weight of e^-12.2 among float16's
    # subnormal numbers, 2^-24 apart, would be off by 0.5 %.)
    bound = want * (2.0 ** -10 + 2 * n * 2.0 ** -24 + 2.0 ** -20)
    assert ((out.double() - want).abs() <= bound).all()
    assert (lse.double() - torch.logsumexp(s, 0)).abs().max() <= 2.0 ** -18


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("m,n", [(1, 700), (1, 5000), (600, 600)])
def test_large_scores(m, n, dtype):
    """Scores of nearly 2^24, all alike, of either sign: every key has the same weight."""
    d = 16
    for sign in (1.0, -1.0):
        q = torch.full((m, 1, d), 1000.0 * sign, dtype=dtype, device="cuda")
        k = torch.full((n, 1, d), 1000.0, dtype=dtype, device="cuda")
        v = normal(1, n, 1, d, dtype=dtype)
        out, lse = kmip.full_fwd(q, k, v, 1.0)
        want = v.double().mean(0)
        # weights and the result, half a step each, and n additions in 32 bits each of the sum and its normaliser
        u = torch.finfo(dtype).eps / 2
        assert ((out.double() - want).abs() <= (u + 2 * n * 2.0 ** -24) * v.double().abs().mean(0) + u * want.abs()).all()
        score = d * 1000.0 * 1000.0 * sign
        assert (lse.double() - score - math.log(n)).abs().max() <= 2.0 ** -22 * abs(score)


@pytest.mark.parametrize("heads,kv,d,dv,causal", [(8, 2, 64, 64, True), (3, 3, 16, 32, False), (4, 1, 128, 128, True)])
def test_cache_with_room(heads, kv, d, dv, causal):
    """Rows behind a slot's keys in use are not read (NaN there) and get gradient 0; nothing beside the outputs is written."""
    ql, kl, room = [3, 0, 40, 1, 200], [70, 9, 40, 1500, 130], [0, 7, 100, 33, 1]
    where = dict(graph_offsets=sums(ql), key_offsets=sums([a + b for a, b in zip(kl, room)]), key_lengths=kl)
    nq, nk = where["graph_offsets"][-1], where["key_offsets"][-1]
    q, k, v, g = normal(1, nq, heads, d), normal(2, nk, kv, d), normal(3, nk, kv, dv), normal(4, nq, heads, dv)
    used = torch.zeros(nk, dtype=torch.bool, device="cuda")
    for lo, n in zip(where["key_offsets"], kl):
        used[lo:lo + n] = True
    k[~used] = math.nan
    v[~used] = math.nan

    def guarded(rows, *shape, dtype=BF):
        whole = torch.full((rows + 32, *shape), 7.0, dtype=dtype, device="cuda")
        return whole, whole[16:16 + rows]

    made = [guarded(nq, heads, dv), guarded(nq, heads, dtype=SF), guarded(nq, heads, d), guarded(nk, kv, d), guarded(nk, kv, dv)]
    out, lse, dq, dk, dvv = (x[1] for x in made)
    kmip.full_fwd(q, k, v, 0.3, causal=causal, out=out, lse=lse, **where)
    kmip.full_bwd(q, k, v, g, out, lse, 0.3, causal=causal, dq=dq, dk=dk, dv=dvv, **where)
    for whole, _ in made:
        assert (whole[:16] == 7.0).all() and (whole[-16:] == 7.0).all()
    assert (dk[~used] == 0).all() and (dvv[~used] == 0).all()
    k[~used], v[~used] = 0.0, 0.0
    against64(dict(out=out, lse=lse, dq=dq, dk=dk, dv=dvv), q, k, v, g, 0.3, causal, **where)


def test_other_sequences_do_not_matter():
    ql = [50, 64, 33, 300, 1]
    o = sums(ql)
    q, k, v, g = (normal(s, o[-1], 4, 32) for s in range(4))
    clean = both(q, k, v, g, 0.2, graph_offsets=o)
    for t in (q, k, v, g):
        t[o[2]:o[3]] = math.nan
    dirty = both(q, k, v, g, 0.2, graph_offsets=o)
    keep = torch.ones(o[-1], dtype=torch.bool, device="cuda")
    keep[o[2]:o[3]] = False
    for name in clean:
        assert torch.equal(clean[name][keep], dirty[name][keep]), name


def test_scores_far_apart():
    """Scores whose maximum rises by hundreds from tile to tile, and falls: the running reference follows."""
    n, d = 700, 64
    q, k, v, g = (normal(s, n, 2, d, dtype=HF) for s in range(4))
    for slope in (0.02, -0.02):
        steep = (k.float() * 0.1 + slope * torch.arange(n, device="cuda")[:, None, None] * torch.sign(q[:1].float())).to(HF)
        same = q[:1].expand(n, 2, d).contiguous()
        got = both(same, steep, v, g, 1.0)
        against64({x: got[x] for x in ("out", "lse", "dv")}, same, steep, v, g, 1.0)


def test_rows_that_see_nothing_everywhere():
    q, k, v, g = normal(1, 300, 2, 32), normal(2, 40, 2, 32), normal(3, 40, 2, 32), normal(4, 300, 2, 32)
    got = both(q, k, v, g, 0.2, causal=True)
    assert (got["out"][:260] == 0).all() and (got["lse"][:260] == -math.inf).all() and (got["dq"][:260] == 0).all()
    against64(got, q, k, v, g, 0.2, True)
    empty = both(q, k[:0], v[:0], g, 0.2)
    assert (empty["out"] == 0).all() and (empty["lse"] == -math.inf).all() and (empty["dq"] == 0).all()
    none = both(q[:0], k, v, g[:0], 0.2)
    assert (none["dk"] == 0).all() and (none["dv"] == 0).all()


def test_many_sequences():
    """More sequences than one launch takes, with empty ones among them."""
    rng = np.random.default_rng(3)
    ql, kl = rng.integers(0, 40, 401).tolist(), rng.integers(0, 70, 401).tolist()
    kl[17], ql[17] = 3000, 5       # and one that is cut into runs
    where = dict(graph_offsets=sums(ql), key_offsets=sums(kl))
    q, k = normal(1, sum(ql), 2, 16), normal(2, sum(kl), 1, 16)
    v, g = normal(3, sum(kl), 1, 16), normal(4, sum(ql), 2, 16)
    against64(both(q, k, v, g, 0.25, True, **where), q, k, v, g, 0.25, True, **where)


@pytest.mark.parametrize("n,causal", [(256, False), (257, True), (600, False)])
def test_many_graphs(n, causal):
    """As many graphs as one launch takes where queries and keys lie alike, one more, and many; empty ones among them."""
    ql = np.random.default_rng(n).integers(0, 30, n).tolist()
    ql[5], ql[n - 1] = 0, 150
    where = dict(graph_offsets=sums(ql))
    q, k, v, g = (normal(s, sum(ql), h, 16) for s, h in ((1, 2), (2, 1), (3, 1), (4, 2)))
    got = both(q, k, v, g, 0.25, causal, **where)
    against64(got, q, k, v, g, 0.25, causal, **where)
    if not causal:   # the same with the offsets of the keys given
        again = both(q, k, v, g, 0.25, causal, key_offsets=list(where["graph_offsets"]), **where)
        for name in got:
            assert torch.equal(got[name], again[name]), name


def test_offsets_past_32_bits():
    """A sequence at the end of a cache of more than 4 GB, and its gradients."""
    nk, n, m, d = (1 << 24) + 5000, 333, 40, 128
    k, v = (torch.zeros(nk, 1, d, dtype=BF, device="cuda") for _ in range(2))
    k[-n:], v[-n:] = normal(1, n, 1, d), normal(2, n, 1, d)
    q, g = normal(3, m, 2, d), normal(4, m, 2, d)
    where = dict(graph_offsets=[0, 0, m], key_offsets=[0, nk - n, nk])
    out, lse = kmip.full_fwd(q, k, v, 0.1, causal=True, **where)
    dq, dk, dv = kmip.full_bwd(q, k, v, g, out, lse, 0.1, causal=True, **where)
    assert not dk[:-n].any() and not dv[:-n].any()
    got = dict(out=out, lse=lse, dq=dq, dk=dk[-n:], dv=dv[-n:])
    against64(got, q, k[-n:].contiguous(), v[-n:].contiguous(), g, 0.1, True)


def test_two_streams():
    """Two calls at once on streams of their own, one of them cut into runs."""
    a = [normal(s, 3000, 2, 64) for s in range(4)]
    b = [normal(s + 9, n, h, 64) for s, (n, h) in enumerate([(2, 8), (9000, 1), (9000, 1), (2, 8)])]
    want = both(*a, 0.1), both(*b, 0.1, True)
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(one):
            x = both(*a, 0.1)
        with torch.cuda.stream(two):
            y = both(*b, 0.1, True)
        torch.cuda.synchronize()
        for got, ref in zip((x, y), want):
            for name in got:
                assert torch.equal(got[name], ref[name]), name


def test_workspace_is_reused():
    ws = kmip.Workspace("cuda")
    q, k, v, g = normal(1, 4, 8, 64), normal(2, 20000, 1, 64), normal(3, 20000, 1, 64), normal(4, 4, 8, 64)
    want = both(q, k, v, g, 0.1)
    for _ in range(2):
        out, lse = kmip.full_fwd(q, k, v, 0.1, workspace=ws)
        grads = kmip.full_bwd(q, k, v, g, out, lse, 0.1, workspace=ws)
        for x, name in zip((out, lse, *grads), ("out", "lse", "dq", "dk", "dv")):
            assert torch.equal(x, want[name])


def test_captured():
    """Rotary, forward and backward in one graph, next to another graph: every replay gives what the eager calls give."""
    H, Hk, d, ql, kl = 4, 2, 64, [1, 60, 300], [3000, 60, 900]
    where = dict(graph_offsets=sums(ql), key_offsets=sums(kl))
    nq, nk = sum(ql), sum(kl)
    freqs, m = kmip.rotary_frequencies(d)
    pos = torch.arange(nq, dtype=torch.int32, device="cuda")
    static = [normal(s, n, h, d) for s, (n, h) in enumerate([(nq, H), (nk, Hk), (nk, Hk), (nq, H)])]
    ws = kmip.Workspace("cuda")

    def step(q, k, v, g):
        q = kmip.rotary(q, None, pos, freqs, magnitude=m)
        out, lse = kmip.full_fwd(q, k, v, 0.125, causal=True, workspace=ws, **where)
        return (out, lse, *kmip.full_bwd(q, k, v, g, out, lse, 0.125, causal=True, workspace=ws, **where))

    step(*static)   # (the workspace has its size before the captures)
    torch.cuda.synchronize()
    graphs, results = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results.append(step(*static))
        graphs.append(graph)
    for round_ in range(4):
        fresh = [normal(20 * round_ + s, *t.shape) for s, t in enumerate(static)]
        want = step(*fresh)
        for t, f in zip(static, fresh):
            t.copy_(f)
        for r in results:
            for x in r:
                x.zero_()
        torch.cuda.synchronize()
        graphs[round_ % 2].replay()
        graphs[1 - round_ % 2].replay()
        torch.cuda.synchronize()
        for r in results:
            for x, y in zip(r, want):
                assert torch.equal(x, y)


def test_captured_training():
    """Autograd through rotary and attention in a graph, eager results of the same leaves dropped before: every replay gives the
    eager gradients, with eager calls in between."""
    H, Hk, d, o = 4, 2, 32, [0, 70, 71, 300]
    rotary = kmip.Rotary(d)
    pos = torch.cat([torch.arange(b - a) for a, b in zip(o, o[1:])]).to(torch.int32).cuda()
    leaves = [normal(s, o[-1], h, d).requires_grad_() for s, h in ((1, H), (2, Hk), (3, Hk))]
    g = normal(4, o[-1], H, d)

    def step():
        q, k = rotary(leaves[0], leaves[1], pos)
        out = kmip.full_attention(q, k, leaves[2], 0.2, graph_offsets=o, causal=True)
        return (out.detach(), *torch.autograd.grad(out, leaves, g))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for round_ in range(3):
        with torch.no_grad():
            for i, t in enumerate(leaves):
                t.copy_(normal(10 * round_ + i, *t.shape))
        want = [x.clone() for x in step()]
        for x in got:
            x.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y)


def test_autograd():
    ql, kl = [40, 7, 120], [40, 30, 90]
    where = dict(graph_offsets=sums(ql), key_offsets=sums(kl))
    q, k, v, g = normal(1, 167, 4, 32), normal(2, 160, 2, 32), normal(3, 160, 2, 64), normal(4, 167, 4, 64)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    offsets = list(where["graph_offsets"])
    out = kmip.full_attention(*leaves, 0.2, graph_offsets=offsets, key_offsets=where["key_offsets"], causal=True)
    offsets[1] = 0   # the caller's own list
    grads = torch.autograd.grad(out, leaves, g)
    want = both(q, k, v, g, 0.2, True, **where)
    assert torch.equal(out, want["out"])
    for x, name in zip(grads, ("dq", "dk", "dv")):
        assert torch.equal(x, want[name])
    # a gradient that is one number expanded, and one whose rows lie apart
    out = kmip.full_attention(*leaves, 0.2, causal=False, **where)
    grads = torch.autograd.grad(out.sum(), leaves)
    ones = both(q, k, v, torch.ones_like(g), 0.2, **where)
    for x, name in zip(grads, ("dq", "dk", "dv")):
        assert torch.equal(x, ones[name])


@pytest.mark.parametrize("inter", [False, True])
def test_rotary_views_and_places(inter):
    n, H, Hk, d, rot = 333, 6, 2, 64, 32
    freqs, m = kmip.rotary_frequencies(rot, scaling="blend", factor=3.0, original_length=2048)
    pos = torch.randint(0, 1 << 20, (n,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(1))
    fused = normal(1, n, H + 2 * Hk, d)
    kw = dict(interleaved=inter, magnitude=m)
    want_q, want_k = kmip.rotary(fused[:, :H].contiguous(), fused[:, H:H + Hk].contiguous(), pos, freqs, **kw)
    check_turned(want_q, fused[:, :H], pos, freqs, inter, m)
    assert torch.equal(kmip.rotary(fused[:, :H], None, pos, freqs, **kw), want_q)
    heads_first = torch.empty(Hk, n, d, dtype=BF, device="cuda").transpose(0, 1)
    q, k = kmip.rotary(fused[:, :H], fused[:, H:H + Hk], pos, freqs, k_out=heads_first, **kw)
    assert torch.equal(q, want_q) and k is heads_first and torch.equal(k, want_k)
    # odd places: rows that allow no vector loads
    odd = torch.empty(n, H, d + 1, dtype=BF, device="cuda")[:, :, 1:]
    odd.copy_(fused[:, :H])
    assert torch.equal(kmip.rotary(odd, None, pos, freqs, **kw), want_q)
    rest = fused[:, H + Hk:].clone()
    kmip.rotary(fused[:, :H], fused[:, H:H + Hk], pos, freqs, q_out=fused[:, :H], k_out=fused[:, H:H + Hk], **kw)   # in place
    assert torch.equal(fused[:, :H], want_q) and torch.equal(fused[:, H:H + Hk], want_k) and torch.equal(fused[:, H + Hk:], rest)
    # no positions: row i at i
    x = normal(3, n, H, d)
    rows = torch.arange(n, dtype=torch.int32, device="cuda")
    assert torch.equal(kmip.rotary(x, freqs=freqs), kmip.rotary(x, None, rows, freqs))


def test_rotary_gradient():
    n, H, Hk, d = 129, 3, 1, 32
    rotary = kmip.Rotary(16, interleaved=True, scaling="blend", factor=2.0, original_length=500)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 1001
    q, k = (normal(s, n, h, d, dtype=SF).requires_grad_() for s, h in ((1, H), (2, Hk)))
    a, b = rotary(q, k, pos, dtype=BF)
    ga, gb = normal(3, n, H, d), normal(4, n, Hk, d)
    dq, dk = torch.autograd.grad((a, b), (q, k), (ga, gb))
    assert dq.dtype == SF and dk.dtype == SF
    for x, g in ((dq, ga), (dk, gb)):
        check_turned(x, g, pos, rotary.freqs, True, rotary.magnitude, inverse=True)
    # against differences: the turn is linear, <g, f(q + u) - f(q)> = <dq, u>
    u = normal(5, n, H, d, dtype=SF)
    left = (ga.double() * (turned64(q + u, pos, rotary.freqs, True, rotary.magnitude)[0]
                           - turned64(q, pos, rotary.freqs, True, rotary.magnitude)[0])).sum()
    right = (dq.double() * u.double()).sum()
    size = (ga.double().abs() * u.double().abs()).sum()
    assert abs(left - right) <= 2.0 ** -18 * size
    only = kmip.rotary(q, None, pos, rotary.freqs)
    assert torch.autograd.grad(only.sum(), q)[0].shape == q.shape


@pytest.mark.parametrize("far", [0, 1 << 30])
def test_positions_and_attention(far):
    """Rotary, then attention, as a model calls them; and scores depend on differences of positions alone."""
    ql, kl, H, Hk, d = [1, 30], [500, 70], 8, 2, 64
    where = dict(graph_offsets=sums(ql), key_offsets=sums(kl))
    freqs, m = kmip.rotary_frequencies(d)
    q, k, v, g = normal(1, 31, H, d), normal(2, 570, Hk, d), normal(3, 570, Hk, d), normal(4, 31, H, d)
    kp = torch.cat([torch.arange(n) for n in kl]).to(torch.int32).cuda() + far
    qp = torch.cat([torch.arange(n - a, n) for a, n in zip(ql, kl)]).to(torch.int32).cuda() + far
    tq, tk = kmip.rotary(q, None, qp, freqs), kmip.rotary(k, None, kp, freqs)
    check_turned(tq, q, qp, freqs, False, m)
    against64(both(tq, tk, v, g, 0.125, True, **where), tq, tk, v, g, 0.125, True, **where)
    base, _ = kmip.full_fwd(kmip.rotary(q, None, qp - far, freqs), kmip.rotary(k, None, kp - far, freqs), v, 0.125, causal=True, **where)
    out, _ = kmip.full_fwd(tq, tk, v, 0.125, causal=True, **where)
    # rounding of turned q and k (half a step each) moves a score by at most 2^-7 |q| |k| scale
    assert (out.float() - base.float()).abs().max() < 0.25


def layer_reference(layer, x, positions, offsets, grad):
    """The layer's output and parameter gradients in float64 from its own bf16 projections."""
    with torch.no_grad():
        q, k, v = layer.project(x, positions, offsets)
    w = [p.detach().double() for p in (layer.w_q, layer.w_k, layer.w_v, layer.w_o)]
    N = len(x)
    dout = (grad.double() @ w[3].t()).to(BF).view(N, layer.heads, layer.d_v)
    want = full64(q, k, v, layer.scale, sequences(N, N, offsets), layer.causal, dout)
    out, dq, dk, dv = (want[n][0] for n in ("out", "dq", "dk", "dv"))
    if layer.rotary is not None:
        pos = torch.arange(N, device=x.device, dtype=torch.int32) if positions is None else positions
        r = layer.rotary
        dq, dk = (turned64(t, pos, r.freqs, r.interleaved, r.magnitude, inverse=True)[0] for t in (dq, dk))
    flat = [t.reshape(N, -1) for t in (dq, dk, dv)]
    X = x.double()
    return (out.reshape(N, -1) @ w[3], sum(f @ wi.t() for f, wi in zip(flat, w)), *(X.t() @ f for f in flat),
            out.reshape(N, -1).t() @ grad.double())


@pytest.mark.parametrize("heads,kv,d_k,d_v,causal,rot", [(4, 2, 32, 32, True, 32), (3, 3, 16, 64, False, 0), (8, 1, 64, 64, True, 16)])
def test_full_layer(heads, kv, d_k, d_v, causal, rot):
    gen = torch.Generator(device="cuda").manual_seed(heads)
    rotary = kmip.Rotary(rot, interleaved=heads == 8) if rot else None
    layer = kmip.FullAttention(64, heads, d_k, d_v, kv_heads=kv, causal=causal, device="cuda", generator=gen, rotary=rotary)
    offsets = [0, 90, 91, 91, 300]
    pos = torch.cat([torch.arange(b - a) for a, b in zip(offsets, offsets[1:])]).to(torch.int32).cuda() if rot else None
    x = normal(1, 300, 64, dtype=SF).requires_grad_()
    grad = normal(2, 300, 64, dtype=SF)
    out = layer(x, offsets, positions=pos)
    got = (out, *torch.autograd.grad(out, (x, layer.w_q, layer.w_k, layer.w_v, layer.w_o), grad))
    want = layer_reference(layer, x.detach(), pos, offsets, grad)
    for name, a, b in zip(("out", "dx", "dw_q", "dw_k", "dw_v", "dw_o"), got, want):
        # 16-bit results and gradients between the products, each within a step (2^-7) in the sum of squares
        assert torch.linalg.norm(a.double() - b) <= 2.0 ** -6 * torch.linalg.norm(b), name


def test_kmip_layer_with_rotary():
    gen = torch.Generator(device="cuda").manual_seed(5)
    rotary = kmip.Rotary(32)
    layer = kmip.KMIPAttention(64, 2, 32, k=8, device="cuda", generator=gen, rotary=rotary)
    x = normal(1, 200, 64, dtype=SF).requires_grad_()
    pos = torch.arange(200, dtype=torch.int32, device="cuda")
    offsets = [0, 80, 200]
    out = layer(x, offsets, positions=pos)
    q, k = rotary((x @ layer.w_q).view(200, 2, 32), (x @ layer.w_k).view(200, 2, 32), pos, dtype=BF)
    o = kmip.attention(q, k, (x @ layer.w_v).to(BF).view(200, 2, 32), 8, layer.scale, graph_offsets=offsets)
    assert torch.equal(out, o.reshape(200, 64) @ layer.w_o)
    assert torch.isfinite(torch.autograd.grad(out.sum(), layer.w_q)[0]).all()
    # no rotary: as it was
    plain = kmip.KMIPAttention(64, 2, 32, k=8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    q, k, v = plain.project(x)
    assert torch.equal(q, (x @ plain.w_q).to(BF).view(200, 2, 32)) and torch.equal(k, (x @ plain.w_k).to(BF).view(200, 2, 32))
