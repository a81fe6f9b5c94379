"""Cases of the operators that a mesh network's blocks are trained and run with, beside the convolutions and the pooling:
layer norm over rows of features, attention among the vertices of every mesh of a mini-batch (packed one behind the other,
as ``picasso_decimate_batch`` leaves them), and the norm and clipping of all gradients of a network.

Sizes: the resolutions of the encoder's ladder (16 rooms of 60 thousand vertices, each level 40 % of the one before: 24,000,
9,600, 3,840, 1,536), widths of 6 to 2,048 channels, heads of 16 to 128 of them, sequences of up to 60 thousand, networks of
a few thousand to 100 million weights.  A case is a dict of plain values; see ``listed`` for what each stands for.
"""
import functools
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def _norm(rows, channels, dtype, train):
    return dict(op="norm", rows=rows, channels=channels, dtype=dtype, train=train)


def _attention(meshes, queries, keys, heads, groups, width, dtype, causal, train):
    """queries, keys: vertices per mesh on average; keys = 0: the queries' own.  groups: heads of keys and values."""
    return dict(op="attention", meshes=meshes, queries=queries, keys=keys, heads=heads, groups=groups, width=width, dtype=dtype,
                causal=causal, train=train)


def _clip(tensors, values, dtype, scale):
    return dict(op="clip", tensors=tensors, values=values, dtype=dtype, scale=scale)


def listed():
    return [
        # inference on one small object's coarsest level: launches count, not bytes; an odd width
        dict(_norm(512, 100, "f32", False), name="norm-forward-512-c100"),
        # a training step's mini-batch at the first level, at an inner layer's width
        dict(_norm(960000, 64, "f32", True), name="norm-train-16x60k-c64"),
        # blocks over long sequences of facets, 16-bit features
        dict(_norm(24000, 1024, "bf16", True), name="norm-train-24k-c1024"),
        # two small objects at a coarse level, all vertices with all others of their mesh: latency
        dict(_attention(2, 120, 0, 4, 4, 32, "f32", False, False), name="attention-2x120"),
        # the bottleneck of an encoder in training: 16 rooms at the ladder's last level, 32-bit features as the convolutions'
        dict(_attention(16, 1536, 0, 4, 4, 32, "f32", False, True), name="attention-train-16x1536"),
        # across levels: every vertex of a level looks at the next coarser one's, grouped heads, inference
        dict(_attention(16, 3840, 1536, 8, 2, 64, "f16", False, False), name="attention-levels-16x3840"),
        # readout: one token for each of 16 rooms over all its vertices (the form for single tokens)
        dict(_attention(16, 1, 60000, 4, 1, 64, "bf16", False, False), name="attention-readout-16x60k"),
        # facets as sequences, each looking at those in front of it: training with grouped heads, packed, of different lengths
        dict(_attention(3, 8000, 0, 8, 2, 128, "bf16", True, True), name="attention-causal-3x8k"),
        # the filters, norms and dense halves of a small convolution network
        dict(_clip(64, 60000, "f32", 4.0), name="clip-64-tensors-60k"),
        # a wide network: 200 tensors, 100 million weights
        dict(_clip(200, 100000000, "f32", 4.0), name="clip-200-tensors-100m"),
        # 16-bit gradients that are within the bound already
        dict(_clip(120, 20000000, "bf16", 0.5), name="clip-120-tensors-20m-bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over the logarithm of the ranges above, odd ones as often as not."""
    kind = rng.choice(("norm", "norm", "attention", "attention", "attention", "readout", "clip", "clip"))
    dtype = rng.choice(("f32", "f32", "bf16", "f16"))
    if kind == "norm":
        channels = _log(rng, 6, 2048)
        channels = max(8, channels // 8 * 8) if rng.random() < 0.6 else channels
        return _norm(_log(rng, 200, min(960000, 60000000 // channels)), channels, dtype, rng.random() < 0.6)
    if kind == "clip":
        tensors = rng.randint(1, 300)
        return _clip(tensors, max(tensors, _log(rng, 2000, 60000000)), dtype, rng.choice((0.5, 2.0, 10.0)))
    groups = rng.choice((1, 2, 4))
    heads = groups * rng.choice((1, 1, 2, 4))
    width = rng.choice((16, 32, 40, 64, 64, 96, 128))
    if kind == "readout":
        meshes = rng.randint(1, 16)
        return _attention(meshes, rng.randint(1, 4), _log(rng, 100, min(960000, 45000000 // (groups * width)) // meshes), heads, groups, width, dtype, False, rng.random() < 0.3)
    meshes = rng.choice((1, 2, rng.randint(3, 16)))
    most = min(12000 // meshes, int(math.sqrt(4.5e10 / (heads * width * meshes))))
    queries = _log(rng, 30, most)
    keys = rng.choice((0, 0, 0, _log(rng, 30, most)))
    return _attention(meshes, queries, keys, heads, groups, width, dtype, rng.random() < 0.4, rng.random() < 0.6)


# ---- inputs -----------------------------------------------------------------------------------


def _lengths(meshes, average, salt):
    """Lengths of a batch's meshes: half to one and a half times the average, the sum fixed; with five meshes or more one is empty."""
    rng = random.Random(meshes * 1000003 + average * 101 + salt)
    if average <= 4 or meshes == 1:
        return [average] * meshes
    share = [rng.uniform(0.5, 1.5) for _ in range(meshes)]
    if meshes >= 5:
        share[rng.randrange(meshes)] = 0.0
    n = [int(average * meshes * s / sum(share)) for s in share]
    n[share.index(max(share))] += average * meshes - sum(n)
    return n


def _sequences(case):
    lq = _lengths(case["meshes"], case["queries"], 1)
    return lq, (_lengths(case["meshes"], case["keys"], 2) if case["keys"] else lq)


def _sizes(case):
    """Sizes of a network's tensors: from a filter's few values to dense ones that hold most of them."""
    rng = random.Random(case["tensors"] * 7919 + case["values"])
    share = [math.exp(rng.uniform(0.0, 7.0)) for _ in range(case["tensors"])]
    n = [max(1, int((case["values"] - case["tensors"]) * s / sum(share))) for s in share]
    n[share.index(max(share))] += max(0, case["values"] - sum(n))
    return n


def _host_inputs(case, seed):
    """The inputs of a case, in the type that it names."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    t = TYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)

    if case["op"] == "norm":
        n, c = case["rows"], case["channels"]
        # features behind a convolution: channels of different means and scales
        s = dict(x=(randn(n, c) * (0.5 + torch.rand((c,), generator=gen, device=DEV)) + 0.3 * randn(c)).to(t),
                 gamma=1.0 + 0.2 * randn(c), beta=0.1 * randn(c))
        if case["train"]:
            s["gy"] = randn(n, c).to(t)
        return s
    if case["op"] == "clip":
        sizes = _sizes(case)
        flat = randn(sum(sizes))
        # tensors' gradients differ in scale by orders of magnitude; the whole's norm is about `scale` times the bound
        grads = [(g * 10.0 ** (-(k % 4))).to(t) for k, g in enumerate(flat.split(sizes))]
        total = math.sqrt(sum(m * 100.0 ** (-(k % 4)) for k, m in enumerate(sizes)))
        return dict(grads=grads, max_norm=total / case["scale"])
    lq, lk = _sequences(case)
    h, g, d = case["heads"], case["groups"], case["width"]
    s = dict(q=randn(sum(lq), h, d).to(t), k=randn(sum(lk), g, d).to(t), v=randn(sum(lk), g, d).to(t))
    if case["train"]:
        s["gout"] = randn(sum(lq), h, d).to(t)
    return s


def prepare(case, seed):
    torch.cuda.set_device(0)
    s = _host_inputs(case, seed)
    s["case"] = case
    if case["op"] == "attention":
        lq, lk = _sequences(case)
        s["lq"], s["lk"] = lq, lk
        s["q_offsets"] = torch.tensor([0] + list(np.cumsum(lq)), dtype=torch.int32, device=DEV)
        s["k_offsets"] = torch.tensor([0] + list(np.cumsum(lk)), dtype=torch.int32, device=DEV) if case["keys"] else s["q_offsets"]
    if case["op"] == "clip":
        # what the optimiser takes: one array of all tensors, one behind the other
        sizes = [g.numel() for g in s["grads"]]
        s["flat"] = torch.empty((sum(sizes),), dtype=s["grads"][0].dtype, device=DEV)
        s["clipped"] = list(s["flat"].split(sizes))
    return s


# ---- one pass -----------------------------------------------------------------------------------


def run(s):
    return _run_own(s) if own else _run_plain(s)


@functools.lru_cache(maxsize=1)
def _handle():
    """The program's context."""
    import paper_2103_15076_amd as pk
    return pk.Context(1024, 2048, 1, device=0)


def _run_own(s):
    case, ctx = s["case"], _handle()
    if case["op"] == "norm":
        y, mean, rstd = ctx.picasso_layer_norm_forward(s["x"], s["gamma"], s["beta"], EPS)
        if not case["train"]:
            return y, mean, rstd
        return (y, mean, rstd) + ctx.picasso_layer_norm_backward(s["gy"], s["x"], s["gamma"], mean, rstd)
    if case["op"] == "clip":
        return ctx.picasso_clip_gradients(s["grads"], s["max_norm"], out=s["clipped"]), s["flat"]
    at = (s["q_offsets"], s["k_offsets"], case["causal"])
    out, lse = ctx.picasso_attention_forward(s["q"], s["k"], s["v"], *at)
    if not case["train"]:
        return out, lse
    return (out, lse) + ctx.picasso_attention_backward(s["gout"], s["q"], s["k"], s["v"], out, lse, *at)


def _run_plain(s):
    case = s["case"]
    if case["op"] == "norm":
        return _plain_norm(s, case)
    if case["op"] == "clip":
        return _plain_clip(s)
    return _plain_attention(s, case)


def _plain_norm(s, case):
    t, x, gamma = s["x"].dtype, s["x"].float(), s["gamma"]
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((x - mean) * (x - mean)).mean(1, keepdim=True) + EPS)
    xh = (x - mean) * rstd
    y = (xh * gamma + s["beta"]).to(t)
    if not case["train"]:
        return y, mean[:, 0], rstd[:, 0]
    gy = s["gy"].float()
    h = gy * gamma
    gx = rstd * (h - h.mean(1, keepdim=True) - xh * (h * xh).mean(1, keepdim=True))
    # (sums over up to a million rows: in 64 bits)
    return y, mean[:, 0], rstd[:, 0], gx.to(t), (gy * xh).sum(0, dtype=torch.float64).float(), gy.sum(0, dtype=torch.float64).float()


def _plain_clip(s):
    norm = torch.stack([(g.double() * g.double()).sum() for g in s["grads"]]).sum().sqrt()
    c = torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0).float()
    return norm.float().reshape(1), torch.cat([(g.float() * c).to(g.dtype) for g in s["grads"]])


def _padded(x, offsets, longest):
    """[meshes, heads, longest, width] of the packed rows, zero behind a mesh's last; and which places those are."""
    at = offsets[:-1, None] + torch.arange(longest, device=DEV)
    used = at < offsets[1:, None]
    rows = x.float()[at.clamp(max=x.shape[0] - 1).long()] * used[:, :, None, None]
    return rows.permute(0, 2, 1, 3).contiguous(), used


def _plain_attention(s, case):
    t, h, g, d = s["q"].dtype, case["heads"], case["groups"], case["width"]
    nq, nk, b = max(max(s["lq"]), 1), max(max(s["lk"]), 1), case["meshes"]
    scale = 1.0 / math.sqrt(d)
    q, q_used = _padded(s["q"], s["q_offsets"], nq)
    k, k_used = _padded(s["k"], s["k_offsets"], nk)
    v, _ = _padded(s["v"], s["k_offsets"], nk)
    # the heads of a group one behind the other, over its keys: [meshes * groups, heads per group * queries, width]
    q, k, v = q.reshape(b * g, h // g * nq, d), k.reshape(b * g, nk, d), v.reshape(b * g, nk, d)
    allowed = q_used[:, :, None] & k_used[:, None, :]
    if case["causal"]:
        i, j = torch.arange(nq, device=DEV)[:, None], torch.arange(nk, device=DEV)[None, :]
        behind = (s["k_offsets"].diff() - s["q_offsets"].diff())[:, None, None]
        allowed = allowed & (j <= i + behind)
    allowed = allowed[:, None, None].expand(b, g, h // g, nq, nk).reshape(b * g, h // g * nq, nk)
    p = torch.where(allowed, torch.bmm(q, k.transpose(1, 2).contiguous()) * scale, -math.inf)
    most = p.amax(2, keepdim=True)
    p = torch.exp(p - torch.where(most == -math.inf, 0.0, most))
    total = p.sum(2, keepdim=True)
    lse = (most + torch.log(total))[:, :, 0]
    p = p / torch.where(total == 0, 1.0, total)
    out = torch.bmm(p, v)

    def packed(x, used, heads, n):
        return x.reshape(b, heads, n, -1).permute(0, 2, 1, 3)[used]

    answer = (packed(out, q_used, h, nq).to(t), packed(lse[:, :, None], q_used, h, nq)[:, :, 0].t().contiguous())
    if not case["train"]:
        return answer
    gout = _padded(s["gout"], s["q_offsets"], nq)[0].reshape(b * g, h // g * nq, d)
    gv = torch.bmm(p.transpose(1, 2).contiguous(), gout)
    ds = p * (torch.bmm(gout, v.transpose(1, 2).contiguous()) - (gout * out).sum(2, keepdim=True)) * scale
    gq, gk = torch.bmm(ds, k), torch.bmm(ds.transpose(1, 2).contiguous(), q)
    return answer + (packed(gq, q_used, h, nq).to(t), packed(gk, k_used, g, nk).to(t), packed(gv, k_used, g, nk).to(t))


# ---- the same from the definitions, in 64 bits ----------------------------------------------------


def exact(case, seed):
    torch.cuda.set_device(0)
    s = _host_inputs(case, seed)
    if case["op"] == "norm":
        return _exact_norm(case, s)
    if case["op"] == "clip":
        whole = torch.cat([g.double() for g in s["grads"]])
        norm = torch.linalg.vector_norm(whole)
        return norm.reshape(1), min(1.0, s["max_norm"] / (float(norm) + 1e-6)) * whole
    # every mesh and head by itself
    lq, lk = _sequences(case)
    h, per, scale = case["heads"], case["heads"] // case["groups"], 1.0 / math.sqrt(case["width"])
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    out, gq, gk, gv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    lse = torch.full((h, q.shape[0]), -math.inf, dtype=torch.float64, device=DEV)
    a0 = b0 = 0
    for n, m in zip(lq, lk):
        a, b = slice(a0, a0 + n), slice(b0, b0 + m)
        a0, b0 = a0 + n, b0 + m
        if not n or not m:
            continue
        hidden = torch.ones((n, m), dtype=torch.bool, device=DEV).triu(m - n + 1) if case["causal"] else None
        for head in range(h):
            x, y, z = q[a, head], k[b, head // per], v[b, head // per]
            score = (x @ y.t()).mul_(scale)
            if case["causal"]:
                score.masked_fill_(hidden, -math.inf)
            lse[head, a] = torch.logsumexp(score, 1)
            p = torch.softmax(score, 1)
            if case["causal"]:
                p[hidden.all(1)] = 0.0  # queries that no key is in front of
            out[a, head] = p @ z
            if case["train"]:
                go = s["gout"][a, head].double()
                gv[b, head // per] += p.t() @ go
                dp = go @ z.t()
                ds = p * (dp - (p * dp).sum(1, keepdim=True))
                gq[a, head] = scale * (ds @ y)
                gk[b, head // per] += scale * (ds.t() @ x)
    return (out, lse, gq, gk, gv) if case["train"] else (out, lse)


def _exact_norm(case, s):
    x = s["x"].double()
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    rstd = (var + EPS).rsqrt()
    gamma = s["gamma"].double()
    answer = (((x - mean) * rstd) * gamma + s["beta"].double(), mean.flatten(), rstd.flatten())
    if not case["train"]:
        return answer
    # d y_i / d x_j = gamma_i rstd (delta_ij - 1 / C - xh_i xh_j / C), applied to gy
    gy, xh = s["gy"].double(), (x - mean) * rstd
    h = gy * gamma
    gx = rstd * (h - (h.sum(1, keepdim=True) + xh * (h * xh).sum(1, keepdim=True)) / case["channels"])
    ones = torch.ones((1, case["rows"]), dtype=torch.float64, device=DEV)
    return answer + (gx, (ones @ (gy * xh))[0], (ones @ gy)[0])


# ---- what a pass cannot do without --------------------------------------------------------------


def work(case):
    """Inputs read once, outputs written once; the arithmetic of the definitions."""
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        values = case["rows"] * case["channels"]
        # x -> y; and in training gy, x -> gx
        return dict(bytes=values * size * (5 if case["train"] else 2) + 8 * case["rows"] + 8 * case["channels"],
                    flops=values * (24 if case["train"] else 8))
    if case["op"] == "clip":
        return dict(bytes=2 * size * sum(_sizes(case)), flops=3 * sum(_sizes(case)))
    lq, lk = _sequences(case)
    h, g, d = case["heads"], case["groups"], case["width"]
    pairs = sum(_pairs(n, m, case["causal"]) for n, m in zip(lq, lk))
    rows, cols = sum(lq) * h * d, sum(lk) * g * d
    nbytes = size * (2 * rows + 2 * cols) + 4 * h * sum(lq)
    if case["train"]:  # q, k, v, out and gout read, three gradients written
        nbytes += size * (4 * rows + 4 * cols) + 4 * h * sum(lq)
    return dict(bytes=nbytes, flops=(14 if case["train"] else 4) * h * d * pairs)


def _pairs(n, m, causal):
    """Pairs of a query and a key that it looks at, of n queries and m keys (causal: query i sees the keys up to i + m - n)."""
    if not causal:
        return n * m
    short = max(0, n - m)  # queries that see nothing
    n -= short
    return n * (m - n) + n * (n + 1) // 2
