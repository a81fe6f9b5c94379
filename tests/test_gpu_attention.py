"""Attention among packed sequences, forward and backward, against a plain implementation in 64 bits.

Bars, from the inputs of each test (u = 2^-24, h = half a step of the features' type, 0 beside u for float32):
a score of D products, summed in binary32 in some order and scaled, is off by at most d_ij = (D + 4) u scale sum |q| |k|,
its exponential, relative, by d_ij + 8 u (1 + |s|); with e the largest of these over a row's keys the normalised
weights are off by 2 e + (n + 8) u relative (n keys: the sum of the weights), and each weight is rounded once more (h) as
an operand.  So |out - exact| <= (2 e + 2 (n + 8) u + h) sum p |v| + h |out|, |lse - exact| <= e + (n + 8) u + 2 u |lse|.
Backward: p from the scores and lse is off by 2 e + (n + 8) u + 4 u |lse| =: f relative; ds = p (dp - delta) by
p (f |dp - delta| + (D + 2) u (sum |gout| |v| + sum |gout| |out|) + sum |gout| |error of out|), and rounded (h); the sums over
n or m terms add (n + 8) u of the sum of absolute values, the result's rounding h of itself.
float16: below 2^-14 a value is off by half of 2^-24 instead.  The weights, carried times 2^15, so by 2^-40 (absolute, of weights
that add up to 1); ds, carried times a power of two that puts the largest of it between 2^13 and 2^15, by 2^-38 of that largest.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    import paper_2103_15076_amd as pk
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    with pk.Context(64, 64, 1, device=0) as c:
        yield c


def offsets(lengths, first=0):
    o = [first]
    for n in lengths:
        o.append(o[-1] + n)
    return torch.tensor(o, dtype=torch.int32, device="cuda")


def make(lq, lk, hq, hkv, d, dtype, seed, scale_up=1.0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: (torch.randn(*s, generator=g) * scale_up).to(DTYPES[dtype]).cuda()  # noqa: E731
    return r(sum(lq), hq, d), r(sum(lk), hkv, d), r(sum(lk), hkv, d), (torch.randn(sum(lq), hq, d, generator=g)).to(DTYPES[dtype]).cuda()


def reference(q, k, v, gout, lq, lk, causal, scale, h, small=False):
    """Every output in 64 bits and its bar: {name: (value, bar)}; small: float16's bars for what is below its normal range."""
    w0, d0 = (2.0 ** -40, 2.0 ** -38) if small else (0.0, 0.0)
    q, k, v, go = (t.double().cpu() for t in (q, k, v, gout))
    hq, hkv, d = q.shape[1], k.shape[1], q.shape[2]
    G = hq // hkv
    z = lambda t: torch.zeros_like(t)  # noqa: E731
    out, b_out, gq, b_gq = z(q), z(q), z(q), z(q)
    gk, b_gk, gv, b_gv, a_gk, a_gv = z(k), z(k), z(k), z(k), z(k), z(k)
    lse = torch.full((hq, q.shape[0]), -math.inf, dtype=torch.float64)
    b_lse = torch.zeros_like(lse)
    a = b = 0
    for n, m in zip(lq, lk):
        i, j = slice(a, a + n), slice(b, b + m)
        a, b = a + n, b + m
        if n == 0 or m == 0:
            continue
        ok = torch.ones(n, m, dtype=torch.bool)
        if causal:
            ok = torch.arange(m)[None, :] <= torch.arange(n)[:, None] + (m - n)
        for x in range(hq):
            Q, K, V, O = q[i, x], k[j, x // G], v[j, x // G], go[i, x]
            s = torch.where(ok, scale * Q @ K.T, -math.inf)
            sa = scale * (Q.abs() @ K.abs().T)
            e = torch.where(ok, (d + 4) * U * sa + 8 * U * (1 + sa), torch.zeros(())).amax(1, keepdim=True)
            l = torch.logsumexp(s, 1, keepdim=True)
            l0 = torch.where(l == -math.inf, 0.0, l)
            p = torch.where(ok, torch.exp(s - l0), 0.0)
            out[i, x] = p @ V
            lse[x, i] = l[:, 0]
            b_out[i, x] = (2 * e + 2 * (m + 8) * U + h) * (p @ V.abs()) + w0 * V.abs().sum(0) + (h + U) * out[i, x].abs()
            b_lse[x, i] = (e + (m + 8) * U + 2 * U * l0.abs())[:, 0]
            f = 2 * e + (m + 8) * U + 4 * U * l0.abs()
            dp = O @ V.T
            delta = (O * out[i, x]).sum(1, keepdim=True)
            ds = p * (dp - delta)
            off = (d + 2) * U * (O.abs() @ V.abs().T + (O.abs() * out[i, x].abs()).sum(1, keepdim=True)) + (O.abs() * b_out[i, x]).sum(1, keepdim=True)
            b_ds = p * (f * (dp - delta).abs() + off) + h * ds.abs() + d0 * ds.abs().max()
            gq[i, x] = scale * ds @ K
            b_gq[i, x] = scale * (b_ds @ K.abs() + (m + 8) * U * (ds.abs() @ K.abs())) + (h + 2 * U) * gq[i, x].abs()
            gk[j, x // G] += scale * ds.T @ Q
            b_gk[j, x // G] += scale * (b_ds.T @ Q.abs())
            a_gk[j, x // G] += scale * (ds.abs().T @ Q.abs())
            gv[j, x // G] += p.T @ O
            b_gv[j, x // G] += ((f + h) * p + w0).T @ O.abs()
            a_gv[j, x // G] += p.T @ O.abs()
    terms = (max(lq) * G + 8) * U
    b_gk += terms * a_gk + (h + 2 * U) * gk.abs()
    b_gv += terms * a_gv + (h + 2 * U) * gv.abs()
    return dict(out=(out, b_out), lse=(lse, b_lse), gq=(gq, b_gq), gk=(gk, b_gk), gv=(gv, b_gv))


def held(got, want, what):
    value, bar = want
    got = got.double().cpu()
    same = got == value  # (infinities)
    bad = ~(same | ((got - value).abs() <= bar + 1e-30))
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), float((got - value).abs()[bad].max()), float(bar[bad].min()))


def check(ctx, lq, lk, hq, hkv, d, dtype, causal, seed=1, scale=None, scale_up=1.0):
    print(f"attention lq={lq} lk={lk} {hq}/{hkv} d={d} {dtype} causal={causal}", flush=True)
    q, k, v, go = make(lq, lk, hq, hkv, d, dtype, seed, scale_up)
    qo, ko = offsets(lq), offsets(lk)
    same = lq == lk
    out, lse = ctx.picasso_attention_forward(q, k, v, qo, None if same else ko, causal=causal, scale=scale)
    g = ctx.picasso_attention_backward(go, q, k, v, out, lse, qo, None if same else ko, causal=causal, scale=scale)
    h = 0.0 if dtype == "f32" else torch.finfo(DTYPES[dtype]).eps / 2
    want = reference(q, k, v, go, lq, lk, causal, scale or 1 / math.sqrt(d), h, small=dtype == "f16")
    if dtype == "f16":  # (results below the type's normal range are off by half its smallest step)
        want = {n: (x, b + (2.0 ** -25 if n != "lse" else 0.0)) for n, (x, b) in want.items()}
    for name, got in zip(("out", "lse", "gq", "gk", "gv"), (out, lse) + g):
        held(got, want[name], name)
    again = ctx.picasso_attention_forward(q, k, v, qo, ko, causal=causal, scale=scale)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])  # the same to the bit


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", [8, 32, 40, 64, 96, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_widths_and_types(ctx, dtype, d, causal):
    check(ctx, [77, 1, 0, 130], [77, 1, 0, 130], 4, 2, d, dtype, causal, seed=d)


@pytest.mark.parametrize("lq,lk", [([1], [1]), ([1], [1000]), ([1, 3, 0, 2], [700, 0, 5, 333]), ([300], [1]), ([31, 32, 33], [63, 64, 65]),
                                   ([129], [128]), ([127, 128], [200, 100]), ([5, 0, 0], [0, 0, 9]), ([600], [40])])
@pytest.mark.parametrize("heads", [(1, 1), (6, 2), (5, 1)])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths_and_groups(ctx, lq, lk, heads, causal):
    # (causal with fewer keys than queries: the first queries see none)
    check(ctx, lq, lk, *heads, 32, "f32", causal, seed=len(lq) + heads[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_wide_tiles_and_every_row_shape(ctx, dtype):
    # enough rows that workgroups of 128 of them are taken, for every width
    for d in (32, 64, 128):
        lens = [520, 260, 3, 700, 0, 513] if d < 128 else [400, 300, 513]
        check(ctx, lens, lens, 16, 8, d, dtype, d == 64, seed=d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_axes_are_split(ctx, dtype):
    check(ctx, [1], [9001], 2, 1, 64, dtype, False)
    check(ctx, [2, 1], [5000, 3], 2, 2, 40, dtype, True)
    check(ctx, [3001], [5], 2, 2, 32, dtype, False)


def test_float16_weights_below_its_normal_range(ctx):
    # one of 40,000 keys has a weight of 2^-15; gradients of 2^-10 and of 2^6 beside each other
    q, k, v, go = make([3], [40000], 1, 1, 32, "f16", 8)
    go[0] *= 2.0 ** -10
    go[2] *= 2.0 ** 6
    o1, o2 = offsets([3]), offsets([40000])
    out, lse = ctx.picasso_attention_forward(q, k, v, o1, o2)
    g = ctx.picasso_attention_backward(go, q, k, v, out, lse, o1, o2)
    h = torch.finfo(torch.float16).eps / 2
    want = reference(q, k, v, go, [3], [40000], False, 1 / math.sqrt(32), h, small=True)
    for name, got in zip(("out", "lse", "gq", "gk", "gv"), (out, lse) + g):
        value, bar = want[name]
        held(got, (value, bar + (2.0 ** -25 if name != "lse" else 0.0)), name)


def test_many_sequences(ctx):
    lens = [(7 * i) % 5 for i in range(300)]
    check(ctx, lens, lens, 2, 1, 16, "f32", True)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_large_scores(ctx, dtype):
    # scores of some hundreds: one key takes nearly everything
    check(ctx, [100], [100], 2, 2, 64, dtype, False, scale_up=4.0)


def test_strided_heads_of_one_projection(ctx):
    T, hq, hkv, d = 150, 4, 2, 32
    for dtype in (torch.float32, torch.bfloat16):
        qkv = torch.randn(T, (hq + 2 * hkv), d, device="cuda").to(dtype)
        q, k, v = qkv.split([hq, hkv, hkv], dim=1)
        o = offsets([90, 60])
        out, lse = ctx.picasso_attention_forward(q, k, v, o, causal=True)
        want = ctx.picasso_attention_forward(q.contiguous(), k.contiguous(), v.contiguous(), o, causal=True)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        go = torch.randn_like(out)
        gqkv = torch.full_like(qkv, 7.0)
        ctx.picasso_attention_backward(go, q, k, v, out, lse, o, causal=True, grads=gqkv.split([hq, hkv, hkv], dim=1))
        plain = ctx.picasso_attention_backward(go, q.contiguous(), k.contiguous(), v.contiguous(), out, lse, o, causal=True)
        assert torch.equal(gqkv, torch.cat(plain, 1))
        # heads outermost, and a query that is one row broadcast to all
        hm = lambda t: t.permute(1, 0, 2).contiguous().permute(1, 0, 2)  # noqa: E731
        assert torch.equal(ctx.picasso_attention_forward(hm(q), hm(k), hm(v), o, causal=True)[0], out)
        one = q[:1].expand(T, hq, d)
        assert torch.equal(ctx.picasso_attention_forward(one, k, v, o)[0], ctx.picasso_attention_forward(one.contiguous(), k, v, o)[0])


@pytest.mark.parametrize("keys", [70, 4000])  # (4000: split)
def test_rows_of_no_sequence(ctx, keys):
    """Rows in front of the first and behind the last sequence: 0 / -inf in what the call allocates, left as they were in the
    caller's tensors; NaN in them, or in another sequence, reaches nothing."""
    q, k, v, go = (torch.randn(n, 2, 32, device="cuda") for n in (60, keys, keys, 60))
    qo, ko = offsets([20, 30], 4), offsets([keys - 25, 20], 2)
    clean = ctx.picasso_attention_forward(q, k, v, qo, ko)
    gclean = ctx.picasso_attention_backward(go, q, k, v, *clean, qo, ko)
    for t, o in ((q, qo), (k, ko), (v, ko), (go, qo)):
        t[: int(o[0])] = math.nan
        t[int(o[-1]):] = math.nan
    out, lse = ctx.picasso_attention_forward(q, k, v, qo, ko)
    assert torch.equal(out[4:54], clean[0][4:54]) and torch.equal(lse[:, 4:54], clean[1][:, 4:54])
    assert (out[:4] == 0).all() and (out[54:] == 0).all() and (lse[:, :4] == -math.inf).all() and (lse[:, 54:] == -math.inf).all()
    g = ctx.picasso_attention_backward(go, q, k, v, out, lse, qo, ko)
    for x, y, (s, e) in zip(g, gclean, ((4, 54), (2, keys - 3), (2, keys - 3))):
        assert torch.equal(x[s:e], y[s:e]) and (x[:s] == 0).all() and (x[e:] == 0).all()
    mine = torch.full_like(q, 5.0)
    back, _ = ctx.picasso_attention_forward(q, k, v, qo, ko, out=mine)
    assert back.data_ptr() == mine.data_ptr() and (mine[:4] == 5).all() and (mine[54:] == 5).all() and torch.equal(mine[4:54], out[4:54])
    grads = tuple(torch.full_like(t, 5.0) for t in (q, k, v))
    ctx.picasso_attention_backward(go, q, k, v, out, lse, qo, ko, grads=grads)
    for x, y, (s, e) in zip(grads, g, ((4, 54), (2, keys - 3), (2, keys - 3))):
        assert torch.equal(x[s:e], y[s:e]) and (x[:s] == 5).all() and (x[e:] == 5).all()
    # NaN in the second sequence leaves the first as it was
    k[keys - 20:keys - 10] = math.nan
    assert torch.equal(ctx.picasso_attention_forward(q, k, v, qo, ko)[0][4:24], clean[0][4:24])


def test_causal_queries_ahead_of_all_keys(ctx):
    q, k, v, go = make([50], [20], 2, 1, 32, "f32", 3)
    out, lse = ctx.picasso_attention_forward(q, k, v, offsets([50]), offsets([20]), causal=True)
    assert (out[:30] == 0).all() and (lse[:, :30] == -math.inf).all() and torch.isfinite(lse[:, 30:]).all()
    gq, gk, gv = ctx.picasso_attention_backward(go, q, k, v, out, lse, offsets([50]), offsets([20]), causal=True)
    assert (gq[:30] == 0).all() and all(torch.isfinite(t).all() for t in (gq, gk, gv))


def test_descending_offsets_stay_within_the_arrays(ctx):
    q, k, v, go = make([64], [64], 2, 1, 32, "f32", 3)
    for o in ([0, 200, 100], [50, 10, 64], [-5, 30, 1 << 30], [64, 0, 0]):
        o = torch.tensor(o, dtype=torch.int32, device="cuda")
        print("offsets", o.tolist(), flush=True)
        out, lse = ctx.picasso_attention_forward(q, k, v, o, causal=True)
        ctx.picasso_attention_backward(go, q, k, v, out, lse, o, causal=True)
    torch.cuda.synchronize()


def test_gradients_against_differences(ctx):
    """Central differences of sum(out * g) in a random direction, in 64 bits of the plain formula, against the kernels' gradients."""
    lq, lk, scale = [9, 4], [11, 6], 0.3
    q, k, v, go = make(lq, lk, 2, 1, 16, "f32", 5)
    qo, ko = offsets(lq), offsets(lk)
    out, lse = ctx.picasso_attention_forward(q, k, v, qo, ko, causal=True, scale=scale)
    grads = ctx.picasso_attention_backward(go, q, k, v, out, lse, qo, ko, causal=True, scale=scale)
    f = lambda *a: float((reference(*a, go, lq, lk, True, scale, 0.0)["out"][0] * go.double().cpu()).sum())  # noqa: E731
    base = [t.double() for t in (q, k, v)]
    for x in range(3):
        way = torch.randn(base[x].shape, dtype=torch.float64, device="cuda")
        plus, minus = list(base), list(base)
        plus[x], minus[x] = base[x] + 1e-5 * way, base[x] - 1e-5 * way
        slope = (f(*plus) - f(*minus)) / 2e-5
        assert abs(slope - float((grads[x].double() * way).sum())) <= 1e-4 * (1 + abs(slope))


def test_empty_calls(ctx):
    z = lambda n: torch.zeros(n, 2, 32, device="cuda")  # noqa: E731
    o1, o2 = offsets([0]), offsets([5])
    out, lse = ctx.picasso_attention_forward(z(0), z(5), z(5), o1, o2)
    assert out.shape == (0, 2, 32) and lse.shape == (2, 0)
    gq, gk, gv = ctx.picasso_attention_backward(z(0), z(0), z(5), z(5), out, lse, o1, o2)
    assert gq.numel() == 0 and (gk == 0).all() and (gv == 0).all()
    out, lse = ctx.picasso_attention_forward(z(5), z(0), z(0), o2, o1)
    assert (out == 0).all() and (lse == -math.inf).all()
    gq, gk, gv = ctx.picasso_attention_backward(z(5), z(5), z(0), z(0), out, lse, o2, o1)
    assert (gq == 0).all() and gk.numel() == 0


def test_refusals(ctx):
    import paper_2103_15076_amd as pk
    q, k, v, go = make([10], [10], 4, 2, 32, "f32", 1)
    o = offsets([10])
    bad = [
        lambda: ctx.picasso_attention_forward(q, k.half(), v, o),
        lambda: ctx.picasso_attention_forward(q.double(), k.double(), v.double(), o),
        lambda: ctx.picasso_attention_forward(q, k, v[:5], o),
        lambda: ctx.picasso_attention_forward(q, k[:5], v[:5], o),              # the keys' offsets are missing
        lambda: ctx.picasso_attention_forward(q, k, v, o.long()),
        lambda: ctx.picasso_attention_forward(q, k, v, o[:1]),
        lambda: ctx.picasso_attention_forward(q, k, v, o, offsets([5, 5])),
        lambda: ctx.picasso_attention_forward(q.transpose(1, 2), k, v, o),
        lambda: ctx.picasso_attention_forward(q.cpu(), k, v, o),
        lambda: ctx.picasso_attention_forward(q, k, v, o, out=torch.empty(10, 4, 16, device="cuda")),
        lambda: ctx.picasso_attention_backward(go, q, k, v, q, torch.zeros(4, 9, device="cuda"), o),
        lambda: ctx.picasso_attention_backward(go, q, k, v, q, torch.zeros(4, 10, device="cuda"), o, grads=(q, None, None)),
    ]
    for n, f in enumerate(bad):
        with pytest.raises(TypeError):
            f()
            print("not refused:", n)
    invalid = [
        lambda: ctx.picasso_attention_forward(q[:, :3], k, v, o),               # 3 heads over 2
        lambda: ctx.picasso_attention_forward(q[..., :20], k[..., :20], v[..., :20], o),
        lambda: ctx.picasso_attention_forward(torch.zeros(10, 4, 136, device="cuda"), torch.zeros(10, 2, 136, device="cuda"),
                                              torch.zeros(10, 2, 136, device="cuda"), o),
        lambda: ctx.picasso_attention_forward(q, k, v, o, scale=0.0),
        lambda: ctx.picasso_attention_forward(q, k, v, o, scale=math.inf),
        lambda: ctx.picasso_attention_forward(q, k, v, o, out=q),
        lambda: ctx.picasso_attention_forward(torch.zeros(10 * 128 + 1, device="cuda")[1:].view(10, 4, 32), k, v, o),  # not 16-byte aligned
    ]
    for n, f in enumerate(invalid):
        with pytest.raises(pk.PicassoError) as e:
            f()
            print("not refused:", n)
        assert e.value.status == pk.PICASSO_ERR_INVALID_ARG


def shifted(lq, lk, hq, hkv, d, seed, by):
    """Inputs whose scores (times 1 / sqrt(d)) all have `by` < 0 added: feature 0 is of one size and opposite signs in q and k."""
    q, k, v, go = make(lq, lk, hq, hkv, d, "f16", seed)
    a = math.sqrt(-by * math.sqrt(d))
    q[..., 0], k[..., 0] = a, -a
    return q, k, v, go


@pytest.mark.parametrize("by", [-5.0, -30.0, -60.0, -95.0])
@pytest.mark.parametrize("lq,lk,heads,d", [([32], [40], (1, 1), 32), ([70, 33], [1, 97], (2, 1), 64), ([45], [130], (2, 2), 128), ([40], [2100], (1, 1), 32)])
def test_float16_keys_behind_the_last_do_not_weigh(ctx, lq, lk, heads, d, by):
    """All scores far below 0 and a number of keys that no tile is a multiple of: what lanes without a key hold (a score of 0) is no
    weight of anything, and the gradients of the keys beside them are held to the bars."""
    print(f"attention f16 lq={lq} lk={lk} {heads} d={d} shifted by {by}", flush=True)
    q, k, v, go = shifted(lq, lk, *heads, d, 5, by)
    qo, ko = offsets(lq), offsets(lk)
    out, lse = ctx.picasso_attention_forward(q, k, v, qo, ko)
    g = ctx.picasso_attention_backward(go, q, k, v, out, lse, qo, ko)
    want = reference(q, k, v, go, lq, lk, False, 1 / math.sqrt(d), torch.finfo(torch.float16).eps / 2, small=True)
    for name, got in zip(("out", "lse", "gq", "gk", "gv"), (out, lse) + g):
        value, bar = want[name]
        held(got, (value, bar + (2.0 ** -25 if name != "lse" else 0.0)), name)


def test_float16_gradients_of_far_sizes_side_by_side(ctx):
    """Every second key has weights near 2^-27 beside keys that share the rest: gradients from 2^13 down to 2^-14, neighbours in one
    tile, each within its own bar: ds, carried by a power of two that puts the largest of a key (of gk; of a query, of gq) between 2^13 and
    2^15, is off by 2^-38 of the largest of that key or query."""
    n, m, d = 40, 44, 32
    scale = 1 / math.sqrt(d)
    q, k, v, go = make([n], [m], 1, 1, d, "f16", 11)
    q, v, go = q * 2.0 ** -2, v * 2.0 ** 7, go * 2.0 ** 7
    q[..., 0] = 2.0 ** -4
    k[..., 0] = 0.0
    k[1::2, :, 0] = -27 * math.log(2) / (scale * 2.0 ** -4)
    o1, o2 = offsets([n]), offsets([m])
    out, lse = ctx.picasso_attention_forward(q, k, v, o1, o2)
    gq, gk, gv = ctx.picasso_attention_backward(go, q, k, v, out, lse, o1, o2)
    want = reference(q, k, v, go, [n], [m], False, scale, torch.finfo(torch.float16).eps / 2)
    Q, K, V, O = (t[:, 0].double().cpu() for t in (q, k, v, go))
    p = torch.softmax(scale * Q @ K.T, 1)
    dp = O @ V.T
    ds = p * (dp - (p * dp).sum(1, keepdim=True))
    value, bar = want["gk"]
    assert value[0::2].abs().max() > 2.0 ** 8 and value[1::2].abs().max() < 2.0 ** -12 and (value[1::2].abs() > 2.0 ** -24).any()
    held(gk, (value, bar + scale * 2.0 ** -38 * (ds.abs().amax(0)[:, None] * Q.abs().sum(0))[:, None] + 2.0 ** -25), "gk")
    value, bar = want["gq"]
    held(gq, (value, bar + scale * 2.0 ** -38 * (ds.abs().amax(1)[:, None] * K.abs().sum(0))[:, None] + 2.0 ** -25), "gq")


def test_outputs_as_parts_of_the_inputs_array(ctx):
    """Every way that parts of one array lie beside each other is taken as an output; what lies over an input is refused and left as it was."""
    import paper_2103_15076_amd as pk
    T, H, D = 150, 2, 32
    o = offsets([90, 60])
    for shape, cut in (((T, 4, H, D), lambda a, i: a[:, i]), ((T, H, 4, D), lambda a, i: a[:, :, i]), ((4, H, T, D), lambda a, i: a[i].transpose(0, 1)),
                       ((H, T, 4, D), lambda a, i: a[:, :, i].transpose(0, 1))):
        a = torch.randn(shape, device="cuda")
        q, k, v, to = (cut(a, i) for i in range(4))
        before = a.clone()
        want, lse = ctx.picasso_attention_forward(q.contiguous(), k.contiguous(), v.contiguous(), o)
        ctx.picasso_attention_forward(q, k, v, o, out=to)
        assert torch.equal(to, want) and all(torch.equal(cut(a, i), cut(before, i)) for i in range(3))
        g = torch.zeros_like(a)
        go = torch.randn(T, H, D, device="cuda")
        ctx.picasso_attention_backward(go, q, k, v, to, lse, o, grads=tuple(cut(g, i) for i in range(3)))
        plain = ctx.picasso_attention_backward(go, q.contiguous(), k.contiguous(), v.contiguous(), want, lse, o)
        assert all(torch.equal(cut(g, i), plain[i]) for i in range(3)) and (cut(g, 3) == 0).all()
        for over in (q, k, v):
            with pytest.raises(pk.PicassoError) as e:
                ctx.picasso_attention_forward(q, k, v, o, out=over)
            assert e.value.status == pk.PICASSO_ERR_INVALID_ARG
            with pytest.raises(pk.PicassoError):
                ctx.picasso_attention_backward(go, q, k, v, to, lse, o, grads=(cut(g, 0), cut(g, 1), over))
        with pytest.raises(pk.PicassoError):
            ctx.picasso_attention_backward(go, q, k, v, to, lse, o, grads=(cut(g, 0), cut(g, 1), cut(g, 1)))
        assert all(torch.equal(cut(a, i), cut(before, i)) for i in range(3))


@pytest.fixture
def much_memory():
    """What a test of many gigabytes took is given back, also to what does not allocate through torch."""
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_more_rows_than_work_items_of_one_launch(ctx, much_memory):
    """2^28 + 160 rows of 8 features: sixteen work items a row would be more than 2^32.  All queries (and all gradients of the outputs) are one
    broadcast row of each head, so every row's results are those of a small call."""
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("less than 30 GB free")
    T, H, D = (1 << 24) + 10, 16, 8
    g = torch.Generator().manual_seed(2)
    q, k, v, go = (torch.randn(n, h, D, generator=g).bfloat16().cuda() for n, h in ((1, H), (3, 1), (3, 1), (1, H)))
    wide = lambda t, n: t.expand(n, H, D)  # noqa: E731
    ko = offsets([3])
    out, lse = ctx.picasso_attention_forward(wide(q, T), k, v, offsets([T]), ko)
    gq, gk, gv = ctx.picasso_attention_backward(wide(go, T), wide(q, T), k, v, out, lse, offsets([T]), ko)
    few = 40
    out0, lse0 = ctx.picasso_attention_forward(wide(q, few), k, v, offsets([few]), ko)
    gq0, _, _ = ctx.picasso_attention_backward(wide(go, few), wide(q, few), k, v, out0, lse0, offsets([few]), ko)
    assert (gq0 != 0).any()
    for name, big, small in (("out", out, out0), ("gq", gq, gq0)):
        for i, c in enumerate(big.split(1 << 20)):
            assert torch.equal(c, small[:1].expand_as(c)), (name, i << 20, (c != small[:1]).any(2).nonzero()[:3].tolist())
    assert all((c == lse0[:, :1]).all() for c in lse.split(1 << 20, dim=1))
    assert torch.isfinite(gk.float()).all() and torch.isfinite(gv.float()).all()


def test_more_heads_and_rows_than_32_bits_count(ctx, much_memory):
    """64 heads of keys, 2^25 + 7 queries: 2^31 rows and more in one launch, of which each axis counts for itself."""
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("less than 120 GB free")
    T, H, D = (1 << 25) + 7, 64, 8
    g = torch.Generator().manual_seed(3)
    q, k, v, go = (torch.randn(n, H, D, generator=g).bfloat16().cuda() for n in (1, 2, 2, 1))
    wide = lambda t, n: t.expand(n, H, D)  # noqa: E731
    ko = offsets([2])
    out, lse = ctx.picasso_attention_forward(wide(q, T), k, v, offsets([T]), ko)
    gq, gk, gv = ctx.picasso_attention_backward(wide(go, T), wide(q, T), k, v, out, lse, offsets([T]), ko)
    few = 40
    out0, lse0 = ctx.picasso_attention_forward(wide(q, few), k, v, offsets([few]), ko)
    gq0, _, _ = ctx.picasso_attention_backward(wide(go, few), wide(q, few), k, v, out0, lse0, offsets([few]), ko)
    for name, big, small in (("out", out, out0), ("gq", gq, gq0)):
        assert all(torch.equal(c, small[:1].expand_as(c)) for c in big.split(1 << 20)), name
    assert all((c == lse0[:, :1]).all() for c in lse.split(1 << 20, dim=1))
    assert torch.isfinite(gk.float()).all() and torch.isfinite(gv.float()).all()


@pytest.mark.parametrize("count", [62, 63, 64, 4000, 70_001, 300_000])
def test_very_many_sequences(ctx, count):
    """Sequences of 0 to 2 queries over 0 to 3 keys each, as many as `count`, against the same by sequences side by side in 64 bits."""
    g = torch.Generator().manual_seed(count)
    lq, lk = torch.randint(0, 3, (count,), generator=g), torch.randint(0, 4, (count,), generator=g)
    cum = lambda n: torch.cat([torch.zeros(1, dtype=torch.long), n.cumsum(0)])  # noqa: E731
    cq, ck = cum(lq), cum(lk)
    q, k, v = (torch.randn(n, 1, 8, generator=g) for n in (int(cq[-1]), int(ck[-1]), int(ck[-1])))
    out, lse = ctx.picasso_attention_forward(q.cuda(), k.cuda(), v.cuda(), cq.int().cuda(), ck.int().cuda(), scale=0.5)
    of = torch.repeat_interleave(torch.arange(count), lq)                     # a query's sequence
    at = (ck[:-1][of][:, None] + torch.arange(3)).clamp(max=len(k) - 1)       # its keys' rows
    seen = torch.arange(3)[None, :] < lk[of][:, None]
    s = torch.where(seen, 0.5 * (q.double() * k[:, 0].double()[at]).sum(2), -math.inf)
    l = torch.logsumexp(s, 1)
    p = torch.where(seen, torch.exp(s - torch.where(l == -math.inf, 0.0, l)[:, None]), 0.0)
    want = (p[:, :, None] * v[:, 0].double()[at]).sum(1)
    # (scores up to 20 of 8 products: (8 + 4) u 20, exponentials 8 u 21; all of it twice, values up to 6)
    assert ((out[:, 0].double().cpu() - want).abs() <= 1000 * U * 6).all()
    got = lse[0].double().cpu()
    assert ((got == l) | ((got - l).abs() <= 1000 * U)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lq,lk,heads", [(50, 20, (2, 1)), (300, 177, (3, 1)), (40, 39, (1, 1)), (2500, 1100, (2, 2))])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_queries_that_see_no_key_reach_nothing(ctx, dtype, lq, lk, heads, bad):
    """Causal, fewer keys than queries: whatever stands in the first rows of q and of the outputs' gradient, every result is the same."""
    print(f"attention {dtype} lq={lq} lk={lk} {heads} {bad} in rows without keys", flush=True)
    q, k, v, go = make([7, lq], [9, lk], *heads, 32, dtype, 4)
    qo, ko = offsets([7, lq]), offsets([9, lk])
    out, lse = ctx.picasso_attention_forward(q, k, v, qo, ko, causal=True)
    want = ctx.picasso_attention_backward(go, q, k, v, out, lse, qo, ko, causal=True)
    assert all(torch.isfinite(t.float()).all() for t in want)
    rows = slice(7, 7 + lq - lk)
    q[rows], go[rows] = bad, bad
    o2, l2 = ctx.picasso_attention_forward(q, k, v, qo, ko, causal=True)
    assert torch.equal(o2, out) and torch.equal(l2, lse)
    for name, a, b in zip(("gq", "gk", "gv"), ctx.picasso_attention_backward(go, q, k, v, out, lse, qo, ko, causal=True), want):
        assert torch.equal(a, b), name


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("causal", [False, True])
def test_non_finite_sequences_stay_by_themselves(ctx, dtype, causal):
    lens = [70, 45, 33]
    for which in range(4):
        a = list(make(lens, lens, 2, 1, 40, dtype, 6))
        o = offsets(lens)
        first = lambda x: [t[s] for t in x for s in (slice(0, 70), slice(115, 148))]  # noqa: E731

        def run(q, k, v, go):
            out, lse = ctx.picasso_attention_forward(q, k, v, o, causal=causal)
            return (out, lse.t()) + ctx.picasso_attention_backward(go, q, k, v, out, lse, o, causal=causal)
        want = first(run(*a))
        a[which][70:115] = math.nan if which % 2 else math.inf
        assert all(torch.equal(x, y) for x, y in zip(first(run(*a)), want))


@pytest.mark.parametrize("dtype,size", [("f32", 3e3), ("f32", 1e6), ("bf16", 1e6), ("f16", 8e3)])
@pytest.mark.parametrize("lq,lk", [(100, 150), (40, 3000), (2, 9000)])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_that_leave_binary32s_whole_numbers(ctx, dtype, size, lq, lk, d):
    """Scores of 2^24 up to 2^41, which binary32 holds to some bits or thousands of bits: the weights still add up to 1 and are finite.  Where the
    largest score is ahead by more than all roundings together (twice the bar of a score, and 40) the row is its key's value exactly."""
    q, k, v, _ = make([lq], [lk], 2, 2, d, dtype, 3)
    q, k = (q.float() * size).to(q.dtype), (k.float() * size).to(k.dtype)
    out, lse = ctx.picasso_attention_forward(q, k, v, offsets([lq]), offsets([lk]))
    scale = 1 / math.sqrt(d)
    assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
    rows = 0
    for x in range(2):
        Q, K, V = (t[:, x].double() for t in (q, k, v))
        s = scale * Q @ K.T
        bar = (d + 4) * U * (scale * Q.abs() @ K.abs().T).amax(1) + 2 * U * s.abs().amax(1)
        top = s.topk(2, dim=1)
        sure = top.values[:, 0] - top.values[:, 1] > 2 * bar + 40
        rows += int(sure.sum())
        assert torch.equal(out[sure][:, x], v[top.indices[sure, 0], x])
        assert ((lse[x].double() - top.values[:, 0]).abs() <= bar + 4 * U * top.values[:, 0].abs() + math.log(lk)).all()
        # every output lies between the smallest and the largest value of its feature
        h = torch.finfo(v.dtype).eps
        assert (out[:, x].double() <= V.amax(0) + h * V.abs().amax(0) + (lk + 8) * U * 8).all()
        assert (out[:, x].double() >= V.amin(0) - h * V.abs().amax(0) - (lk + 8) * U * 8).all()
    assert rows > 0


# 128 rows a workgroup are taken from 256 of them on (rows / 128 and one a sequence, times the heads of keys), and the keys are split
# where there are fewer than 512 and 512 keys or more a sequence.
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lq,lk,split", [([1500, 0, 1303, 1290], [300, 5, 417, 500], False), ([900, 1101], [900, 1101], True)])
def test_128_rows_a_workgroup(ctx, dtype, d, causal, lq, lk, split):
    import paper_2103_15076_amd as pk
    groups = (sum(lq) * 2 // 128 + len(lq)) * 8
    assert groups >= 512 if not split else 256 <= groups < 512
    need = pk.load_library().picasso_attention_workspace_bytes({"f32": 0, "bf16": 1, "f16": 2}[dtype], len(lq), sum(lq), sum(lk), 16, 8, d, 0)
    assert (need > 0) == split
    check(ctx, lq, lk, 16, 8, d, dtype, causal, seed=d)
