"""Full softmax attention and its gradients in 64 bits, from the definition, with bounds on what 16-bit operands and
32-bit sums may be off.  Everything is a loop over sequences and heads of plain products on float64 tensors."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
# The smallest half step of float16 (subnormals are 2^-24 apart): weights and results below 2^-14 lose relative precision.
FLOOR = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}


def sequences(nq, nk, graph_offsets=None, key_offsets=None, key_lengths=None):
    """(query begin, end, key begin, end in use) of each sequence."""
    if graph_offsets is None:
        return [(0, nq, 0, nk if key_lengths is None else int(key_lengths[0]))]
    ko = graph_offsets if key_offsets is None else key_offsets
    return [(int(a), int(b), int(c), int(c + key_lengths[g]) if key_lengths is not None else int(ko[g + 1]))
            for g, (a, b, c) in enumerate(zip(graph_offsets, graph_offsets[1:], ko))]


def hidden(m, n, causal, device):
    """True where query t of m does not see key j of n."""
    t, j = torch.arange(m, device=device)[:, None], torch.arange(n, device=device)[None, :]
    return j > t + n - m if causal else torch.zeros(m, n, dtype=torch.bool, device=device)


def full64(q, k, v, scale, seqs, causal, dout=None):
    """Results and bounds: {"out", "lse", "dq", "dk", "dv"} -> (value, bound), all float64.

    u: half a step of the inputs' type; sums of n products in 32 bits are off by at most n 2^-23 of the sum of magnitudes
    (a chain of n additions and roundings of products, doubled for the order).
      s (times scale): e = d 2^-23 scale sum |q||k| + 2^-22 |scale s|
      weights: relative 2e (their own and the normaliser's), plus 2^-20 for exp2 and the running factors
      out: (u + 2e + 2^-20 + n 2^-23) sum p |v| + u |out|
      gradients: weights are recomputed from lse (relative e_p = 2e + 2^-20), rounded (u); D from the rounded out:
      u sum |dout||out| + its bound's part; dp: dv 2^-23 sum |dout||v|; g rounded (u); the final product n 2^-23; the result u."""
    H, Hk = q.shape[1], k.shape[1]
    rep, u, fl = H // Hk, HALF_STEP[q.dtype], FLOOR[q.dtype]
    d, dv = q.shape[2], v.shape[2]
    dev = q.device

    def zeros(*shape):
        return torch.zeros(*shape, dtype=torch.float64, device=dev)

    got = {n: [zeros(*s), zeros(*s)] for n, s in (("out", (len(q), H, dv)), ("lse", (len(q), H)), ("dq", q.shape),
                                                  ("dk", k.shape), ("dv", v.shape))}
    for a, b, c, e in seqs:
        m, n = b - a, e - c
        if m == 0 or n == 0:
            if m:
                got["lse"][0][a:b] = -math.inf
            continue
        hide = hidden(m, n, causal, dev)
        none = hide.all(1)
        for h in range(H):
            Q, K, V = q[a:b, h].double(), k[c:e, h // rep].double(), v[c:e, h // rep].double()
            s = (Q @ K.t().contiguous()) * scale
            s[hide] = -math.inf
            err = (Q.abs() @ K.abs().t().contiguous()) * (scale * d * 2.0 ** -23)
            err = torch.where(hide, torch.zeros_like(s), err + s.abs() * 2.0 ** -22).amax(1, keepdim=True)   # of the row
            lse = torch.logsumexp(s, 1, keepdim=True)
            p = torch.where(none[:, None], torch.zeros_like(s), torch.exp(s - torch.where(none[:, None], torch.zeros_like(lse), lse)))
            ep = 2 * err + 2.0 ** -20
            O, Oa = p @ V, p @ V.abs()
            Ob = (u + ep + n * 2.0 ** -23) * Oa + u * O.abs() + fl * (1 + V.abs().sum(0))
            got["out"][0][a:b, h], got["out"][1][a:b, h] = O, Ob
            got["lse"][0][a:b, h] = lse[:, 0]
            got["lse"][1][a:b, h] = (err + 2.0 ** -20 + 2.0 ** -22 * torch.where(none[:, None], torch.zeros_like(lse), lse).abs())[:, 0]
            if dout is None:
                continue
            G = dout[a:b, h].double()
            dp, dpa = G @ V.t().contiguous(), G.abs() @ V.abs().t().contiguous()
            D, Db = (G * O).sum(1, keepdim=True), (G.abs() * (Ob + dv * 2.0 ** -23 * O.abs())).sum(1, keepdim=True)
            g = p * (dp - D)
            gb = p * ((dp - D).abs() * (ep + u) + Db + dv * 2.0 ** -23 * dpa) + fl
            n2, m2 = n * 2.0 ** -23, m * rep * 2.0 ** -23
            x = scale * (g @ K)
            got["dq"][0][a:b, h] = x
            got["dq"][1][a:b, h] = scale * ((gb + n2 * g.abs()) @ K.abs()) + u * x.abs() + fl
            got["dk"][0][c:e, h // rep] += scale * (g.t().contiguous() @ Q)
            got["dk"][1][c:e, h // rep] += scale * ((gb + m2 * g.abs()).t().contiguous() @ Q.abs())
            got["dv"][0][c:e, h // rep] += p.t().contiguous() @ G
            got["dv"][1][c:e, h // rep] += (p * (ep + u + m2) + fl).t().contiguous() @ G.abs()
    for name in ("dk", "dv"):
        got[name][1] += u * got[name][0].abs() + fl
    return {n: tuple(x) for n, x in got.items()}


def check(name, x, want, rows=slice(None)):
    """x within the bound of the 64-bit value, elementwise; infinities must agree."""
    value, bound = (t[rows] for t in want)
    x = x[rows].double()
    assert x.shape == value.shape
    inf = torch.isinf(value)
    assert torch.equal(inf, torch.isinf(x)) and torch.equal(x[inf], value[inf]), f"{name}: infinities differ"
    assert not torch.isnan(x).any(), f"{name}: NaN"
    over = ((x - value).abs() - bound)[~inf]
    assert over.numel() == 0 or over.max() <= 0, f"{name}: {over.max():.3g} over a bound of {bound[~inf].flatten()[over.argmax()]:.3g}"
