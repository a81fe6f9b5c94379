"""What the calls on rows of features write into a caller's tensors raises those tensors' versions, as torch's own operations in
place do: a backward pass of torch's that saved the old contents refuses them, and inputs keep their versions."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    import paper_2103_15076_amd as pk
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    with pk.Context(64, 64, 1, device=0) as c:
        yield c


def test_versions_of_outputs_and_inputs(ctx):
    x, y = torch.randn(6, 8, device="cuda"), torch.empty(6, 8, device="cuda")
    ctx.picasso_layer_norm_forward(x, out=y)
    assert y._version == 1 and x._version == 0
    qkv, g = torch.randn(10, 6, 32, device="cuda"), torch.empty(10, 6, 32, device="cuda")
    q, k, v = qkv.split([2, 2, 2], dim=1)
    o = torch.tensor([0, 10], dtype=torch.int32, device="cuda")
    out = torch.empty(10, 2, 32, device="cuda")
    _, lse = ctx.picasso_attention_forward(q, k, v, o, out=out)
    assert out._version == 1 and qkv._version == 0
    ctx.picasso_attention_backward(out, q, k, v, out, lse, o, grads=g.split([2, 2, 2], dim=1))
    assert g._version == 3 and qkv._version == 0 and lse._version == 0  # (three parts of one array)
    a, b = [torch.ones(5, device="cuda"), torch.ones(9, device="cuda").half()], [torch.ones(5, device="cuda"), torch.ones(9, device="cuda").half()]
    ctx.picasso_clip_gradients(a, 1.0, out=b)
    assert [t._version for t in a] == [0, 0] and [t._version for t in b] == [1, 1]
    ctx.picasso_clip_gradients(a, 1.0)
    ctx.picasso_gradient_norm(a)
    assert [t._version for t in a] == [1, 1]


def test_what_torch_has_saved_is_not_silently_replaced(ctx):
    w = torch.randn(6, 8, device="cuda", requires_grad=True)
    y = (w * 2.0).detach()
    loss = (w * y).sum()          # torch keeps y for w's gradient
    ctx.picasso_layer_norm_forward(torch.randn(6, 8, device="cuda"), out=y)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_refused_calls_and_inference_tensors(ctx):
    import paper_2103_15076_amd as pk
    x = torch.ones(6, 8, device="cuda")
    with pytest.raises(pk.PicassoError):
        ctx.picasso_layer_norm_forward(x, out=x)
    assert x._version == 0
    with torch.inference_mode():
        t = torch.full((4,), 3.0, device="cuda")
        ctx.picasso_clip_gradients([t], 3.0)          # (a version that is not kept)
        assert torch.allclose(t, torch.full_like(t, 1.5), rtol=1e-5)
