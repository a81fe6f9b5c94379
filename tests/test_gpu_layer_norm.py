"""Layer norm, forward and backward, against a plain implementation in 64 bits.

Bars, from the inputs of each test (u = 2^-24, h = half a step of the features' type): sums of C values in some order are off
by (C + 2) u of the sum of absolute values, so dm = (C + 2) u mean|x| for the mean; a difference d = x - mean by dd = dm + u |d|;
the variance, relative to variance + eps, by (C + 4) u + (2 dm mean|d| + dm^2) / (var + eps), rstd by dr = half of that + 4 u;
xh by dx = rstd dd + |xh| (dr + 2 u); y by |gamma| dx + 2 u (|y| + |beta|) + h |y|.  The backward pass's two row sums are off by
(C + 3) u mean|h| and (C + 3) u mean|h xh| + mean(|h| dx); the columns' sums by (N + 64) u of theirs (any order of N terms)
and sum |gy| dx.
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


def held(got, want, bar, what):
    got = got.double().cpu()
    bad = ~((got - want).abs() <= bar + 1e-30)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), float((got - want).abs()[bad].max()), float(bar[bad].min()))


def check(ctx, n, c, dtype, seed=1, affine=True, eps=1e-5, offset=0.3, place=0):
    print(f"layer norm {n} x {c} {dtype} affine={affine}", flush=True)
    g = torch.Generator().manual_seed(seed)
    t = DTYPES[dtype]
    h = 0.0 if dtype == "f32" else torch.finfo(t).eps / 2
    tiny = 2.0 ** -24 if dtype == "f16" else 0.0  # (below the type's normal range)

    def on_gpu(a):  # `place` values behind an aligned address
        room = torch.zeros(a.numel() + place, dtype=a.dtype, device="cuda")
        room[place:] = a.reshape(-1).cuda()
        return room[place:].view(a.shape)

    x = (torch.randn(n, c, generator=g) * (0.5 + torch.rand(c, generator=g)) + offset * torch.randn(c, generator=g)).to(t)
    gy = torch.randn(n, c, generator=g).to(t)
    gamma = 1 + 0.3 * torch.randn(c, generator=g) if affine else None
    beta = 0.2 * torch.randn(c, generator=g) if affine else None
    dx, dgy = on_gpu(x), on_gpu(gy)
    dgam, dbet = (on_gpu(gamma), on_gpu(beta)) if affine else (None, None)
    y, mean, rstd = ctx.picasso_layer_norm_forward(dx, dgam, dbet, eps)
    gx, gg, gb = ctx.picasso_layer_norm_backward(dgy, dx, dgam, mean, rstd)
    x, gy = x.double(), gy.double()
    ga = gamma.double() if affine else torch.ones(c, dtype=torch.float64)
    be = beta.double() if affine else torch.zeros(c, dtype=torch.float64)
    m = x.mean(1, keepdim=True)
    d = x - m
    var = (d * d).mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    xh = d * r
    dm = (c + 2) * U * x.abs().mean(1, keepdim=True)
    dd = dm + U * d.abs()
    dr = 0.5 * ((c + 4) * U + (2 * dm * d.abs().mean(1, keepdim=True) + dm * dm) / (var + eps)) + 4 * U
    dxh = r * dd + xh.abs() * (dr + 2 * U)
    want = xh * ga + be
    held(y, want, ga.abs() * dxh + 2 * U * (want.abs() + be.abs()) + h * (want.abs() + ga.abs() * dxh) + tiny, "y")
    held(mean, m[:, 0], (dm + U * m.abs())[:, 0], "mean")
    held(rstd, r[:, 0], (r * (dr + U))[:, 0], "rstd")
    hh = gy * ga
    s1, s2 = hh.mean(1, keepdim=True), (hh * xh).mean(1, keepdim=True)
    b1 = (c + 3) * U * hh.abs().mean(1, keepdim=True)
    b2 = (c + 3) * U * (hh * xh).abs().mean(1, keepdim=True) + (hh.abs() * dxh).mean(1, keepdim=True)
    want = r * (hh - s1 - xh * s2)
    bar = r * (b1 + xh.abs() * b2 + s2.abs() * dxh + dxh * b2 + 4 * U * (hh.abs() + s1.abs() + (xh * s2).abs())) + want.abs() * (dr + 2 * U)
    held(gx, want, bar * (1 + h) + h * want.abs() + tiny, "gx")
    held(gg, (gy * xh).sum(0), (n + 64) * U * (gy * xh).abs().sum(0) + (gy.abs() * dxh).sum(0), "ggamma")
    held(gb, gy.sum(0), (n + 64) * U * gy.abs().sum(0), "gbeta")
    again = ctx.picasso_layer_norm_backward(dgy, dx, dgam, mean, rstd)
    assert all(torch.equal(a, b) for a, b in zip(again, (gx, gg, gb)))


# every way that a row is shared out, at its ends and with odd tails
WIDTHS = [1, 2, 3, 4, 5, 6, 8, 9, 15, 16, 17, 31, 33, 64, 65, 100, 128, 129, 250, 256, 257, 500, 512, 513, 1000, 1024, 1025, 2000, 2048, 2049, 4096, 4097, 8191,
          8192, 8193, 10007]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("c", WIDTHS)
def test_widths(ctx, c, dtype):
    check(ctx, 37 if c > 600 else 301, c, dtype, seed=c)


@pytest.mark.parametrize("n", [1, 2, 3, 63, 64, 65, 1000, 20011])
def test_row_counts(ctx, n):
    check(ctx, n, 64, "f32", seed=n)
    check(ctx, n, 6, "bf16", seed=n)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_addresses_aligned_to_a_value_only(ctx, dtype):
    for c in (3, 7, 64, 100, 257, 1031):
        check(ctx, 50, c, dtype, place=1, seed=c)


def test_without_parameters_and_with_a_large_mean(ctx):
    check(ctx, 100, 48, "f32", affine=False)
    check(ctx, 100, 48, "f32", offset=300.0)   # the mean is hundreds of deviations: nothing may cancel
    check(ctx, 100, 1200, "f32", offset=300.0)


def test_constant_rows(ctx):
    x = torch.full((5, 40), 2.5, device="cuda")
    y, mean, rstd = ctx.picasso_layer_norm_forward(x, eps=1e-5)
    assert (y == 0).all() and (mean == 2.5).all()
    assert torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=4 * U)


def test_non_finite_rows_stay_by_themselves(ctx):
    x = torch.randn(9, 64, device="cuda")
    y0, m0, r0 = ctx.picasso_layer_norm_forward(x)
    x[4, 3], x[7, 0] = math.nan, math.inf
    y, m, r = ctx.picasso_layer_norm_forward(x)
    rows = [0, 1, 2, 3, 5, 6, 8]
    assert torch.equal(y[rows], y0[rows]) and y[4].isnan().all() and y[7].isnan().any()


def test_no_rows(ctx):
    x = torch.zeros(0, 12, device="cuda")
    y, mean, rstd = ctx.picasso_layer_norm_forward(x)
    assert y.shape == (0, 12) and mean.shape == (0,)
    gx, gg, gb = ctx.picasso_layer_norm_backward(x, x, None, mean, rstd)
    assert gx.shape == (0, 12) and (gg == 0).all() and (gb == 0).all()
    for c in (2000, 9000):
        x = torch.zeros(0, c, device="cuda")
        _, mean, rstd = ctx.picasso_layer_norm_forward(x)
        _, gg, gb = ctx.picasso_layer_norm_backward(x, x, None, mean, rstd)
        assert (gg == 0).all() and (gb == 0).all()


def test_gradient_against_differences(ctx):
    g = torch.Generator().manual_seed(3)
    x, gy, gamma = torch.randn(4, 10, generator=g), torch.randn(4, 10, generator=g), 1 + 0.3 * torch.randn(10, generator=g)
    _, mean, rstd = ctx.picasso_layer_norm_forward(x.cuda(), gamma.cuda())
    gx, gg, _ = ctx.picasso_layer_norm_backward(gy.cuda(), x.cuda(), gamma.cuda(), mean, rstd)

    def f(x, gamma):
        d = x - x.mean(1, keepdim=True)
        return float((d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * gamma * gy.double()).sum())

    x, gamma = x.double(), gamma.double()
    way, turn = torch.randn(4, 10, generator=g).double(), torch.randn(10, generator=g).double()
    slope = (f(x + 1e-5 * way, gamma) - f(x - 1e-5 * way, gamma)) / 2e-5
    assert abs(slope - float((gx.double().cpu() * way).sum())) <= 1e-4 * (1 + abs(slope))
    slope = (f(x, gamma + 1e-5 * turn) - f(x, gamma - 1e-5 * turn)) / 2e-5
    assert abs(slope - float((gg.double().cpu() * turn).sum())) <= 1e-4 * (1 + abs(slope))


def test_refusals(ctx):
    import paper_2103_15076_amd as pk
    x = torch.randn(6, 8, device="cuda")
    v = torch.zeros(8, device="cuda")
    r = torch.zeros(6, device="cuda")
    for f in (lambda: ctx.picasso_layer_norm_forward(x.double()), lambda: ctx.picasso_layer_norm_forward(x.t()), lambda: ctx.picasso_layer_norm_forward(x.cpu()),
              lambda: ctx.picasso_layer_norm_forward(x[0]), lambda: ctx.picasso_layer_norm_forward(x, v[:7]), lambda: ctx.picasso_layer_norm_forward(x, v.half()),
              lambda: ctx.picasso_layer_norm_forward(x, out=x.half()), lambda: ctx.picasso_layer_norm_backward(x.half(), x, v, r, r),
              lambda: ctx.picasso_layer_norm_backward(x, x, v, r[:5], r), lambda: ctx.picasso_layer_norm_backward(x, x, v, None, r)):
        with pytest.raises(TypeError):
            f()
    for f in (lambda: ctx.picasso_layer_norm_forward(x, out=x), lambda: ctx.picasso_layer_norm_forward(x, eps=-1.0),
              lambda: ctx.picasso_layer_norm_forward(x, eps=math.nan), lambda: ctx.picasso_layer_norm_forward(x[:, :0].contiguous())):
        with pytest.raises(pk.PicassoError) as e:
            f()
        assert e.value.status == pk.PICASSO_ERR_INVALID_ARG


@pytest.fixture
def much_memory():
    """What a test of many gigabytes took is given back, also to what does not allocate through torch."""
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_more_rows_than_workgroups_of_one_launch(ctx, much_memory):
    """2^24 + 3 rows that take a workgroup each (2056 channels of bfloat16): 256 work items a row would be more than 2^32."""
    n, c, few = (1 << 24) + 3, 2056, 1 << 10
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("less than 150 GB free")
    small = torch.randn(few, c, device="cuda").bfloat16()
    want, m0, r0 = ctx.picasso_layer_norm_forward(small)
    x = torch.empty(n, c, dtype=torch.bfloat16, device="cuda")
    for part in x.split(few):
        part.copy_(small[:len(part)])
    y = torch.zeros_like(x)
    _, mean, rstd = ctx.picasso_layer_norm_forward(x, out=y)
    whole = n // few * few
    for p in y[:whole].view(-1, few, c).split(64):
        assert torch.equal(p, want.expand_as(p))
    assert torch.equal(y[whole:], want[:n - whole])
    assert torch.equal(mean[:whole].view(-1, few), m0.expand(whole // few, few)) and torch.equal(mean[whole:], m0[:n - whole])
    assert torch.equal(rstd[:whole].view(-1, few), r0.expand(whole // few, few)) and torch.equal(rstd[whole:], r0[:n - whole])


def test_more_columns_than_work_items_of_one_launch(ctx, much_memory):
    """2^27 + 5 channels: the columns' sums take 32 work items a channel, more than 2^32.  Features are +1 and -1, so that every sum over a
    row is exact and xh is the feature within 2e-5 (eps 1e-5, and a mean below 1e-7)."""
    c = (1 << 27) + 5
    x = torch.ones(2, c, dtype=torch.bfloat16, device="cuda")
    x[0, 1::2], x[1, 0::2] = -1, -1
    gy = torch.randint(-8, 9, (2, c), device="cuda").bfloat16()
    _, mean, rstd = ctx.picasso_layer_norm_forward(x)
    assert (mean.abs() <= 1e-7).all() and ((rstd - 1).abs() <= 2e-5).all()
    _, gg, gb = ctx.picasso_layer_norm_backward(gy, x, None, mean, rstd)
    assert torch.equal(gb, gy[0].float() + gy[1].float())
    want = gy[0].float() * x[0].float() + gy[1].float() * x[1].float()
    assert ((gg - want).abs() <= 2e-5 * 16 + 1e-6).all()


@pytest.mark.parametrize("n,c,dtype", [(1 << 20, 1028, "f32"), (1 << 18, 8200, "f32"), (1 << 19, 2056, "bf16"), (1 << 23, 6, "f32")])
def test_runs_of_the_columns_sums(ctx, much_memory, n, c, dtype):
    """However many rows there are, no more than 64 of them are added up in binary32 one behind the other, the rest in 64 bits: with a
    gradient of one value everywhere (whose sums round the same way each time) the sum is off by 64 u for a run, u for each of the two values that
    stand between the stages, and u for the result."""
    value = 0.3321608006954193
    x = torch.zeros(n, c, dtype=DTYPES[dtype], device="cuda")
    gy = torch.full((n, c), value, dtype=DTYPES[dtype], device="cuda")
    _, mean, rstd = ctx.picasso_layer_norm_forward(x)
    _, gg, gb = ctx.picasso_layer_norm_backward(gy, x, None, mean, rstd)
    want = float(gy[0, 0]) * n
    assert ((gb.double() - want).abs() <= 67 * U * want).all(), float((gb.double() - want).abs().max()) / want / U
    assert (gg == 0).all()
