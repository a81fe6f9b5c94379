"""The norm of many tensors together and clipping, against a plain implementation in 64 bits.

Bars: the norm is summed in 64 bits and rounded once (2^-24 relative, and 1e-12 for the sum); the factor is rounded once, the
product once in binary32 and once to the tensor's type: 2 u + h relative (u = 2^-24, h = half a step), half the smallest step where
a result is below the type's normal range."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    import paper_2103_15076_amd as pk
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    with pk.Context(64, 64, 1, device=0) as c:
        yield c


def tensors(sizes, dtypes, seed):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * 10.0 ** (-(k % 3))).to(dtypes[k % len(dtypes)]).cuda() for k, n in enumerate(sizes)]


def check(ctx, grads, max_norm, in_place):
    print(f"clip {len(grads)} tensors, {sum(g.numel() for g in grads)} values, max_norm={max_norm}, in_place={in_place}", flush=True)
    want_norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    c = min(1.0, max_norm / (want_norm + 1e-6))
    want = [c * g.double() for g in grads]
    norm = ctx.picasso_gradient_norm(grads)
    assert norm.shape == (1,) and abs(float(norm) - want_norm) <= (U + 1e-12) * want_norm
    before = [g.clone() for g in grads]
    out = None if in_place else [torch.empty_like(g) for g in grads]
    got_norm = ctx.picasso_clip_gradients(grads, max_norm, out=out)
    assert torch.equal(got_norm, norm)
    for k, (g, w) in enumerate(zip(grads if in_place else out, want)):
        f = torch.finfo(g.dtype)
        h = 0.0 if g.dtype == torch.float32 else f.eps / 2
        bar = (2 * U + h) * 1.001 * w.abs() + f.smallest_normal * f.eps / 2
        assert ((g.double() - w).abs() <= bar).all(), k
        if not in_place:
            assert torch.equal(grads[k], before[k])


F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtypes", [[F32], [BF16], [F16], [F32, BF16, F16]])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("max_norm", [0.7, 1e9])
def test_types(ctx, dtypes, in_place, max_norm):
    check(ctx, tensors([1, 2, 3, 5, 8, 64, 0, 100, 1023, 8191, 8192, 8193, 30000], dtypes, 1), max_norm, in_place)


@pytest.mark.parametrize("count", [1, 119, 120, 121, 240, 500])
def test_many_tensors(ctx, count):
    check(ctx, tensors([(37 * k) % 700 + 1 for k in range(count)], [F32, BF16], count), 1.5, False)


def test_large(ctx):
    check(ctx, tensors([20_000_001, 7, 3_000_000], [F32], 2), 10.0, True)
    check(ctx, tensors([30_000_001], [BF16], 2), 10.0, False)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_views_of_one_array_at_any_address(ctx, dtype):
    sizes = [5, 1, 70, 8192, 333, 10001]
    flat = torch.randn(sum(sizes) + 1, device="cuda").to(dtype)
    check(ctx, list(flat[1:].split(sizes)), 2.0, False)
    check(ctx, list(flat[1:].split(sizes)), 2.0, True)
    src = tensors(sizes, [dtype], 4)
    room = torch.full((sum(sizes) + 2,), 9.0, dtype=dtype, device="cuda")
    ctx.picasso_clip_gradients(src, 2.0, out=list(room[1:-1].split(sizes)))
    assert room[0] == 9 and room[-1] == 9  # nothing beside them


def test_values_whose_squares_leave_the_range(ctx):
    g = [torch.full((1000,), 1e30, device="cuda"), torch.full((10,), 1e-30, device="cuda")]
    norm = ctx.picasso_clip_gradients(g, 1.0)
    assert abs(float(norm) - 1e30 * math.sqrt(1000)) <= 1e-6 * 1e30 * math.sqrt(1000)
    assert torch.allclose(g[0], torch.full_like(g[0], 1 / math.sqrt(1000)), rtol=4 * U)


def test_non_finite(ctx):
    g = [torch.ones(100, device="cuda"), torch.ones(9, device="cuda").half()]
    g[0][5] = math.nan
    assert math.isnan(float(ctx.picasso_clip_gradients(g, 1.0))) and all(t.isnan().all() for t in g)
    g = [torch.ones(100, device="cuda"), torch.ones(9, device="cuda").half()]
    g[1][5] = math.inf
    assert float(ctx.picasso_clip_gradients(g, 1.0)) == math.inf
    assert (g[0] == 0).all() and g[1][5].isnan() and (g[1][:5] == 0).all()


def test_limits(ctx):
    g = tensors([10, 20], [F32], 1)
    before = [t.clone() for t in g]
    ctx.picasso_clip_gradients(g, math.inf)
    assert all(torch.equal(a, b) for a, b in zip(g, before))
    ctx.picasso_clip_gradients(g, 0.0)
    assert all((t == 0).all() for t in g)
    assert float(ctx.picasso_clip_gradients(g, 1.0)) == 0.0          # all zero
    assert float(ctx.picasso_clip_gradients([], 1.0)) == 0.0 and float(ctx.picasso_gradient_norm([])) == 0.0
    assert float(ctx.picasso_clip_gradients([torch.zeros(0, device="cuda")], 1.0)) == 0.0


def test_refusals(ctx):
    import paper_2103_15076_amd as pk
    a, b = torch.ones(10, device="cuda"), torch.ones(10, device="cuda")
    for f in (lambda: ctx.picasso_clip_gradients([a.double()], 1.0), lambda: ctx.picasso_clip_gradients([a[::2]], 1.0), lambda: ctx.picasso_clip_gradients([a.cpu()], 1.0),
              lambda: ctx.picasso_clip_gradients([a, None], 1.0), lambda: ctx.picasso_clip_gradients([a], 1.0, out=[a[:9]]),
              lambda: ctx.picasso_clip_gradients([a, b], 1.0, out=[a]), lambda: ctx.picasso_clip_gradients([a], 1.0, out=[a.half()]),
              lambda: ctx.picasso_clip_gradients(5, 1.0), lambda: ctx.picasso_gradient_norm([a.int()])):
        with pytest.raises(TypeError):
            f()
    flat = torch.ones(30, device="cuda")
    for f in (lambda: ctx.picasso_clip_gradients([a, a], 1.0), lambda: ctx.picasso_clip_gradients([flat[:20], flat[10:]], 1.0),
              lambda: ctx.picasso_clip_gradients([flat[:10], flat[10:20]], 1.0, out=[flat[10:20], flat[20:]]),
              lambda: ctx.picasso_clip_gradients([flat[:10]], 1.0, out=[flat[5:15]]), lambda: ctx.picasso_clip_gradients([a], -1.0),
              lambda: ctx.picasso_clip_gradients([a], math.nan)):
        with pytest.raises(pk.PicassoError) as e:
            f()
        assert e.value.status == pk.PICASSO_ERR_INVALID_ARG
    assert (a == 1).all() and (flat == 1).all()
    assert abs(float(ctx.picasso_gradient_norm([a, a])) - math.sqrt(20)) < 1e-5   # (read only: counted twice)


def test_tensors_that_only_a_generator_makes(ctx):
    """Outputs (and gradients) that nothing but the call holds: what the call allocates itself, the norm and the partial sums, is not laid
    into their memory.  (Sizes as of the norm's own block and of larger ones.)"""
    for n in (1, 100, 3000, 300_000):
        g = tensors([n, n, n], [F32], n)
        want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in g))
        for _ in range(3):
            norm = ctx.picasso_clip_gradients(g, 0.25, out=(torch.empty_like(t) for t in g))
            assert abs(float(norm) - want) <= (U + 1e-12) * want, n
            norm = ctx.picasso_clip_gradients((t.clone() for t in g), 0.25)
            assert abs(float(norm) - want) <= (U + 1e-12) * want, n
            assert abs(float(ctx.picasso_gradient_norm(map(torch.clone, g))) - want) <= (U + 1e-12) * want, n
    out = [torch.empty_like(t) for t in g]
    ctx.picasso_clip_gradients(iter(g), 0.25, out=(t.view(-1) for t in out))
    for t, o in zip(g, out):
        w = min(1.0, 0.25 / (want + 1e-6)) * t.double()
        assert ((o.double() - w).abs() <= 2.002 * U * w.abs() + 2.0 ** -149).all()


@pytest.mark.parametrize("count", [960, 2048, 2049, 6000])
def test_very_many_tensors(ctx, count):
    """As many partial sums as tensors, and more than one workgroup's share of them: they are added up once, not by every workgroup."""
    check(ctx, tensors([(53 * k) % 300 + 1 for k in range(count)], [F32, F16], count), 1.5, False)
    big = tensors([30_000 + k % 7 for k in range(count)], [BF16], count)   # (several workgroups a tensor)
    check(ctx, big, 1.5, True)
