"""Full softmax attention and rotary positions: the calls whose speed and results are tracked.

Full softmax attention over packed sequences (or graphs) is the dense counterpart of k-MIP attention:

  out_i = sum_j p_ij v_j,  p_ij = exp(scale q_i.k_j - lse_i),  lse_i = log sum_j exp(scale q_i.k_j),

j over the keys of i's own sequence; causal: query t of a sequence with m queries and n keys sees keys 0 .. t + n - m
(the queries are the last m of the n positions), which may be none (out 0, lse -inf).  H query heads share H / kv_heads to
one key head.  Its gradients, with D_i = dout_i.out_i and g_ij = p_ij (dout_i.v_j - D_i):

  dv_j = sum_i p_ij dout_i,  dq_i = scale sum_j g_ij k_j,  dk_j = scale sum_i g_ij q_i.

Rotary positions turn each pair (a, b) of a row's first `rot` dimensions by the angle t = position * frequency:
(a cos t - b sin t, b cos t + a sin t), times a magnitude; a pair is two neighbours (interleaved) or dimensions i and
i + rot / 2; the rest of the row is passed on.  The gradient is turned back by the same angle, times the magnitude.

A case is a dict:
  kind      attend (forward), train (forward and backward), rotary, rotary_train (forward and backward);
  dtype     of the inputs (rotary cases: `to` of the outputs);
  seqs      number of sequences; their queries are uniform in [q_lo, q_hi], and as many keys stand before these as
            [c_lo, c_hi] says (tokens of an earlier call, in the log of their number); the same for every seed;
  room      keys lie in slots this much longer than the longest sequence (a cache with room), 0: packed;
  fused     q, k and v are views of one projection's rows;
  heads, kv_heads, d (query and key width), dv (value width), causal;
  rot, interleaved, scaling ("none", "linear", "base", "blend"), factor, far (positions up to it).
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _attend(name, kind, dtype, seqs, q, c, heads, kv_heads, d, dv, causal, room=0, fused=False):
    case = dict(kind=kind, dtype=dtype, seqs=seqs, q_lo=q[0], q_hi=q[1], c_lo=c[0], c_hi=c[1], heads=heads,
                kv_heads=kv_heads, d=d, dv=dv, causal=causal, room=room, fused=fused)
    return dict(case, name=name) if name else case


def _rotary(name, kind, dtype, to, tokens, heads, kv_heads, d, rot, interleaved, scaling, factor, far):
    case = dict(kind=kind, dtype=dtype, to=to, tokens=tokens, heads=heads, kv_heads=kv_heads, d=d, rot=rot,
                interleaved=interleaved, scaling=scaling, factor=factor, far=far)
    return dict(case, name=name) if name else case


def listed():
    return [
        # One superpixel-sized graph at inference, all pairs: latency and launches count.
        _attend("attend_graph_311", "attend", "bf16", 1, (311, 311), (0, 0), 3, 3, 32, 32, False),
        # A training batch of superpixel graphs (the second benchmark configuration), attended in full.
        _attend("train_128_graphs", "train", "bf16", 128, (100, 450), (0, 0), 3, 3, 32, 32, False),
        # The efficiency study's dense side, at an odd size near 10^4: one head, d = 16, training.
        _attend("train_dense_10007", "train", "bf16", 1, (10007, 10007), (0, 0), 1, 1, 16, 16, False),
        # Prompts of different lengths in one call, grouped heads, read from a fused projection.
        _attend("prompts_17_ragged", "attend", "fp16", 17, (37, 4001), (0, 0), 16, 4, 64, 64, True, fused=True),
        # One long prompt.
        _attend("prompt_16384", "attend", "bf16", 1, (16384, 16384), (0, 0), 8, 2, 128, 128, True),
        # A training step over one long sequence.
        _attend("train_8192", "train", "bf16", 1, (8192, 8192), (0, 0), 8, 2, 128, 128, True),
        # A training batch of short texts with wider values, one head group each.
        _attend("train_24_texts", "train", "fp16", 24, (1, 1500), (0, 0), 6, 6, 64, 128, True),
        # Serving: one new token for each of 64 sequences, caches from a few tokens to a long context.
        _attend("serve_64_tokens", "attend", "bf16", 64, (1, 1), (7, 32767), 32, 8, 128, 128, True, room=128),
        # Serving: one token of one sequence over a long cache, one key head.
        _attend("serve_1_of_65537", "attend", "bf16", 1, (1, 1), (65536, 65536), 8, 1, 64, 64, True),
        # Serving: the new tokens of 32 sequences get their positions, far into a stretched context.
        _rotary("rotary_32_tokens", "rotary", "bf16", "bf16", 32, 32, 8, 128, 128, False, "blend", 8.0, 131072),
        # A long prompt, half of each head turned, neighbours paired.
        _rotary("rotary_prompt_16383", "rotary", "fp16", "fp16", 16383, 32, 8, 128, 64, True, "base", 4.0, 16384),
        # The layer's projections of a 100k-node graph, float32 to bf16 and back again.
        _rotary("rotary_train_100k", "rotary_train", "fp32", "bf16", 100000, 4, 4, 32, 32, False, "none", 1.0, 100000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng, most):
    kv = rng.choice((1, 2, 3, 4, 8))
    rep = rng.choice((1, 1, 2, 4, 8))
    return min(kv * rep, most // kv * kv), kv


def draw(rng):
    kind = rng.randrange(8)
    dtype = rng.choice(("bf16", "bf16", "fp16"))
    if kind == 0:   # batches of graphs
        lo = _log_int(rng, 1, 150)
        d = rng.choice((16, 32, 64))
        heads = rng.randint(1, 8)
        return _attend("", rng.choice(("attend", "train")), dtype, _log_int(rng, 1, 128), (lo, lo + rng.randint(10, 330)),
                       (0, 0), heads, heads, d, d, False)
    if kind == 1:   # packed prompts
        hi = _log_int(rng, 64, 4000)
        heads, kv = _heads(rng, 16)
        return _attend("", "attend", dtype, max(1, min(_log_int(rng, 1, 24), (1 << 32) // (heads * hi * hi))),
                       (rng.randint(1, hi // 2), hi), (0, 0), heads, kv, *(rng.choice((32, 64, 128)),) * 2, True,
                       fused=rng.random() < 0.5)
    if kind == 2:   # one long prompt
        n = _log_int(rng, 500, 16000)
        d = rng.choice((64, 128))
        kv = rng.choice((1, 2, 4))
        return _attend("", "attend", dtype, 1, (n, n), (0, 0), 2 * kv if n > 8000 and kv == 4 else kv * rng.choice((1, 2)),
                       kv, d, d, rng.random() < 0.6 or n > 8000)
    if kind == 3:   # new tokens over caches
        q = rng.choice((1, 1, 1, 2, 4))
        heads, kv = _heads(rng, 32)
        return _attend("", "attend", dtype, _log_int(rng, 1, 32), (1, q), (rng.randint(0, 100), _log_int(rng, 200, 16000)),
                       heads, kv, *(rng.choice((32, 64, 128)),) * 2, True, room=rng.choice((0, 1, 77, 512)))
    if kind == 4:   # a chunk of a prompt behind its cache
        q = _log_int(rng, 9, 1024)
        heads, kv = _heads(rng, 16)
        return _attend("", "attend", dtype, rng.randint(1, 4), (q, q + rng.randint(0, 50)), (0, _log_int(rng, 100, 8000)),
                       heads, kv, *(rng.choice((64, 128)),) * 2, True, room=rng.choice((0, 64)))
    if kind == 5:   # training
        n = _log_int(rng, 200, 6000)
        heads, kv = _heads(rng, 8)
        return _attend("", "train", dtype, 1 if n > 2000 else rng.randint(1, 8), (n // 2 + 1, n), (0, 0), heads, kv,
                       rng.choice((16, 32, 64, 128)), rng.choice((16, 32, 64, 128)), rng.random() < 0.7,
                       fused=False)
    far, d = _log_int(rng, 1000, 1000000), rng.choice((16, 32, 64, 128))
    scaling = rng.choice(("none", "linear", "base", "blend"))
    factor = 1.0 if scaling == "none" else float(rng.randint(2, 16))
    rot = rng.choice((d, d, d // 2))
    if kind == 6:   # positions at inference
        heads, kv = _heads(rng, 32)
        return _rotary("", "rotary", dtype, dtype, _log_int(rng, 1, 16000), heads, kv, d, rot, rng.random() < 0.5, scaling,
                       factor, far)
    heads = rng.randint(1, 8)
    return _rotary("", "rotary_train", "fp32", rng.choice(("bf16", "fp16", "fp32")), _log_int(rng, 100, 50000), heads, heads,
                   d, rot, rng.random() < 0.5, scaling, factor, far)


# ---- inputs ----


def _lengths(case):
    """Queries and keys of each sequence: the case's own, the same for every seed."""
    rng = random.Random("%(seqs)d of %(q_lo)d to %(q_hi)d behind %(c_lo)d to %(c_hi)d" % case)
    q = [rng.randint(case["q_lo"], case["q_hi"]) for _ in range(case["seqs"])]
    c = [_log_int(rng, case["c_lo"] + 1, case["c_hi"] + 1) - 1 for _ in range(case["seqs"])]
    return q, [a + b for a, b in zip(q, c)]


def _sums(sizes):
    o = [0]
    for s in sizes:
        o.append(o[-1] + s)
    return o


def _frequencies(case):
    """Radians a position of each pair, and the magnitude.  linear: positions divided by the factor.  base: the base raised so
    that the slowest pair turns factor times slower.  blend: pairs that turn less than once in the original length (`far` / factor)
    as in linear, those that turn more than 32 times as they were, in between a blend; magnitude 0.1 log(factor) + 1."""
    r, s = case["rot"], case["factor"]
    base = 10000.0
    if case["scaling"] == "base":
        base *= s ** (r / (r - 2)) if r > 2 else 1.0
    f = base ** (-2.0 * np.arange(r // 2, dtype=np.float64) / r)
    if case["scaling"] == "linear":
        return f / s, 1.0
    if case["scaling"] == "blend":
        keep = np.clip((case["far"] / s * f / (2 * math.pi) - 1.0) / 31.0, 0.0, 1.0)
        return f * keep + f / s * (1.0 - keep), 0.1 * math.log(s) + 1.0
    return f, 1.0


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    t = TYPES[case["dtype"]]
    H, Hk, d = case["heads"], case["kv_heads"], case["d"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE)

    s = {"case": case}
    if case["kind"].startswith("rotary"):
        n = case["tokens"]
        s["q"], s["k"] = normal(n, H, d).to(t), normal(n, Hk, d).to(t)
        s["positions"] = torch.randint(case["far"], (n,), generator=gen, device=DEVICE, dtype=torch.int32)
        s["freqs"], s["magnitude"] = _frequencies(case)
        if case["kind"] == "rotary_train":
            s["dq"], s["dk"] = (normal(n, h, d).to(TYPES[case["to"]]) for h in (H, Hk))
        return s
    dv = case["dv"]
    ql, kl = _lengths(case)
    slots = [max(kl) + case["room"]] * len(kl) if case["room"] else kl
    s["offsets"], s["key_offsets"], s["key_lengths"] = _sums(ql), _sums(slots), kl
    nq, nk = s["offsets"][-1], s["key_offsets"][-1]
    if case["fused"]:
        row = normal(nq, H + 2 * Hk, d).to(t)
        s["q"], s["k"], s["v"] = row[:, :H], row[:, H:H + Hk], row[:, H + Hk:]
    else:
        s["q"], s["k"], s["v"] = normal(nq, H, d).to(t), normal(nk, Hk, d).to(t), normal(nk, Hk, dv).to(t)
    s["scale"] = 1.0 / math.sqrt(d)
    if case["kind"] == "train":
        s["dout"] = normal(nq, H, dv).to(t)
    return s


# ---- the plain forms ----


def _turn(x, cos, sin, rot, interleaved, to):
    x = x.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((y, x[..., rot:]), -1).to(to)


def _plain_rotary(s):
    case = s["case"]
    to, args = TYPES[case["to"]], (case["rot"], case["interleaved"])
    # angles of far positions in 64 bits
    angle = s["positions"].double()[:, None, None] * torch.from_numpy(s["freqs"]).to(DEVICE)
    cos, sin = (angle.cos() * s["magnitude"]).float(), (angle.sin() * s["magnitude"]).float()
    got = {"q": _turn(s["q"], cos, sin, *args, to), "k": _turn(s["k"], cos, sin, *args, to)}
    if case["kind"] == "rotary_train":
        got["dq"] = _turn(s["dq"], cos, -sin, *args, s["q"].dtype)
        got["dk"] = _turn(s["dk"], cos, -sin, *args, s["k"].dtype)
    return got


def _padded(offsets, lengths):
    """Row of each padded place [G, L] (the first row where there is none), and the padded place of each row."""
    o, n = np.asarray(offsets, np.int64)[:-1], np.asarray(lengths, np.int64)
    at = np.arange(n.max())
    there = at < n[:, None]
    row = np.where(there, o[:, None] + at, 0)
    return torch.from_numpy(row).to(DEVICE), torch.from_numpy(np.flatnonzero(there)).to(DEVICE)


def _plain_attend(s):
    case = s["case"]
    H, Hk, G = case["heads"], case["kv_heads"], case["seqs"]
    rep, t = H // Hk, s["q"].dtype
    ql = np.diff(s["offsets"])
    qrow, qplace = _padded(s["offsets"], ql)
    krow, kplace = _padded(s["key_offsets"], s["key_lengths"])
    Lq, Lk = qrow.shape[1], krow.shape[1]
    m = torch.from_numpy(ql).to(DEVICE)[:, None, None]
    n = torch.tensor(s["key_lengths"], device=DEVICE)[:, None, None]

    def rows(x, at):    # queries [G, kv_heads, rep, Lq, width]
        return x.float()[at].view(G, Lq, Hk, rep, -1).permute(0, 2, 3, 1, 4)

    q = rows(s["q"], qrow).reshape(G, Hk, rep * Lq, -1)
    k, v = (x.float()[krow].transpose(1, 2).contiguous() for x in (s["k"], s["v"]))   # [G, kv_heads, Lk, width]
    z = (q @ k.transpose(2, 3)).mul_(s["scale"]).view(G, Hk, rep, Lq, Lk)
    i, j = torch.arange(Lq, device=DEVICE)[None, :, None], torch.arange(Lk, device=DEVICE)[None, None, :]
    seen = j < n
    if case["causal"]:
        seen = seen & (j <= i + n - m)
    z.masked_fill_(~seen[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = top + total.log()
    p.div_(torch.where(total == 0, torch.ones_like(total), total))
    out = p.view(G, Hk, rep * Lq, Lk) @ v

    def packed(x, width):    # [G, kv_heads, rep, Lq, width] to rows [Nq, H, width]
        return x.view(G, Hk, rep, Lq, width).permute(0, 3, 1, 2, 4).reshape(G * Lq, H, width)[qplace]

    got = {"out": packed(out, case["dv"]).to(t), "lse": packed(lse, 1).squeeze(-1)}
    if case["kind"] == "train":
        do = rows(s["dout"], qrow).reshape(G, Hk, rep * Lq, -1)
        # places behind a sequence's end have no gradient
        live = (i < m)[:, None, None].expand(G, Hk, rep, Lq, 1).reshape(G, Hk, rep * Lq, 1)
        do = do * live
        p = p.view(G, Hk, rep * Lq, Lk)
        g = (do @ v.transpose(2, 3)).sub_((do * out).sum(-1, keepdim=True)).mul_(p)
        got["dq"] = packed((g @ k).mul_(s["scale"]), case["d"]).to(t)
        for name, x in (("dk", (g.transpose(2, 3) @ q).mul_(s["scale"])), ("dv", p.transpose(2, 3) @ do)):
            got[name] = x.transpose(1, 2).reshape(G * Lk, Hk, -1)[kplace].to(t)
    return got


def run(state):
    case, s = state["case"], state
    if not own:
        return _plain_rotary(s) if case["kind"].startswith("rotary") else _plain_attend(s)
    import paper_2604_03815_amd as kmip

    if case["kind"].startswith("rotary"):
        to = TYPES[case["to"]]
        q, k = kmip.rotary(s["q"], s["k"], s["positions"], s["freqs"], interleaved=case["interleaved"],
                           magnitude=s["magnitude"], dtype=to)
        got = {"q": q, "k": k}
        if case["kind"] == "rotary_train":
            got["dq"], got["dk"] = kmip.rotary(s["dq"], s["dk"], s["positions"], s["freqs"], interleaved=case["interleaved"],
                                               magnitude=s["magnitude"], inverse=True, dtype=s["q"].dtype)
        return got
    where = dict(graph_offsets=s["offsets"], key_offsets=s["key_offsets"], key_lengths=s["key_lengths"],
                 causal=case["causal"])
    out, lse = kmip.full_fwd(s["q"], s["k"], s["v"], s["scale"], **where)
    got = {"out": out, "lse": lse}
    if case["kind"] == "train":
        got["dq"], got["dk"], got["dv"] = kmip.full_bwd(s["q"], s["k"], s["v"], s["dout"], out, lse, s["scale"], **where)
    return got


# ---- what a pass cannot do without ----


def work(case):
    """Inputs read once (keys of a cache: the used ones), outputs written once; the products over the seen pairs: two in the
    forward, five in the backward."""
    H, Hk, d = case["heads"], case["kv_heads"], case["d"]
    size = {"bf16": 2, "fp16": 2, "fp32": 4}
    if case["kind"].startswith("rotary"):
        values, pairs = case["tokens"] * (H + Hk) * d, case["tokens"] * (H + Hk) * (case["rot"] // 2)
        passes = 2 if case["kind"] == "rotary_train" else 1
        return {"bytes": passes * (values * (size[case["dtype"]] + size[case["to"]]) + 4 * case["tokens"]),
                "flops": passes * 6 * pairs}
    ql, kl = _lengths(case)
    dv, b = case["dv"], size[case["dtype"]]
    pairs = 0
    for m, n in zip(ql, kl):
        pairs += m * n - m * (m - 1) // 2 if case["causal"] else m * n     # (n >= m here)
    nq, nk = sum(ql), sum(kl)
    nbytes = b * (nq * H * (d + dv) + nk * Hk * (d + dv)) + 4 * nq * H
    flops = 2 * H * pairs * (d + dv)
    if case["kind"] == "train":
        nbytes += b * (nq * H * (d + dv) + nk * Hk * (d + dv))
        flops += 2 * H * pairs * (3 * d + 2 * dv)
    return {"bytes": nbytes, "flops": flops}


# ---- the same in 64 bits ----


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("rotary"):
        rot, half = case["rot"], case["rot"] // 2
        first = torch.arange(half, device=DEVICE) * 2 if case["interleaved"] else torch.arange(half, device=DEVICE)
        second = first + 1 if case["interleaved"] else first + half
        t = torch.outer(s["positions"].double(), torch.as_tensor(s["freqs"], device=DEVICE))
        unit = torch.polar(torch.full_like(t, s["magnitude"]), t)[:, None, :]

        def turned(x, factor):
            y = x.double().clone()
            z = torch.complex(y[..., first], y[..., second]) * factor
            y[..., first], y[..., second] = z.real, z.imag
            return y

        got = {"q": turned(s["q"], unit), "k": turned(s["k"], unit)}
        if case["kind"] == "rotary_train":
            got["dq"], got["dk"] = turned(s["dq"], unit.conj()), turned(s["dk"], unit.conj())
        return got
    H, rep, scale = case["heads"], case["heads"] // case["kv_heads"], s["scale"]
    nq, nk = s["offsets"][-1], sum(s["key_lengths"])

    def zeros(*shape):
        return torch.zeros(*shape, dtype=torch.float64, device=DEVICE)

    got = {"out": zeros(nq, H, case["dv"]), "lse": zeros(nq, H)}
    train = case["kind"] == "train"
    if train:
        got.update(dq=zeros(nq, H, case["d"]), dk=zeros(nk, case["kv_heads"], case["d"]),
                   dv=zeros(nk, case["kv_heads"], case["dv"]))
    behind = 0   # keys of the sequences before this one
    for g in range(case["seqs"]):
        a, b = s["offsets"][g], s["offsets"][g + 1]
        lo, n = s["key_offsets"][g], s["key_lengths"][g]
        hidden = None
        if case["causal"]:
            hidden = torch.ones(b - a, n, dtype=torch.bool, device=DEVICE).triu(n - (b - a) + 1)
        for h in range(H):
            q, k, v = s["q"][a:b, h].double(), s["k"][lo:lo + n, h // rep].double(), s["v"][lo:lo + n, h // rep].double()
            z = torch.mm(q, k.t().contiguous()) * scale
            if hidden is not None:
                z[hidden] = -math.inf
            got["lse"][a:b, h] = torch.logsumexp(z, 1)
            p = torch.softmax(z, 1)
            del z
            o = torch.mm(p, v)
            got["out"][a:b, h] = o
            if train:
                do = s["dout"][a:b, h].double()
                dp = torch.mm(do, v.t().contiguous())
                g_ = p * (dp - (p * dp).sum(1, keepdim=True)) * scale
                got["dq"][a:b, h] = torch.mm(g_, k)
                got["dk"][behind:behind + n, h // rep] += torch.mm(g_.t().contiguous(), q)
                got["dv"][behind:behind + n, h // rep] += torch.mm(p.t().contiguous(), do)
        behind += n
    return got
