"""Layer norm, attention and clipping as a program runs them: one behind the other as a block, on a stream of their own, recorded into a
graph and replayed with eager work between, from several threads on one context, and beside another current device.  Every
way gives the bits of the plain eager call."""
import threading

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


SIZES = [  # lengths, queries' heads, keys' heads, features of a head, type: splits in both passes, neither, single tokens
    ([700, 0, 1300], 2, 1, 32, torch.float32), ([300, 77], 4, 4, 64, torch.bfloat16), ([1, 1, 1], 4, 2, 128, torch.float16),
    ([900, 1100], 16, 8, 64, torch.bfloat16)]


class Block:
    """Norm -> attention -> gradients of both -> clipped: inputs that stay, and one training pass of it."""

    def __init__(self, lens, hq, hkv, d, t, seed):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g).to(t).cuda()  # noqa: E731
        T, self.heads, self.d = sum(lens), (hq, hkv), d
        self.x, self.go = r(T, (hq + 2 * hkv) * d), r(T, hq, d)
        self.gamma, self.beta = 1 + 0.1 * torch.randn(self.x.shape[1], generator=g).cuda(), 0.1 * torch.randn(self.x.shape[1], generator=g).cuda()
        o = [0]
        for n in lens:
            o.append(o[-1] + n)
        self.o = torch.tensor(o, dtype=torch.int32, device="cuda")

    def run(self, ctx, stream=None):
        hq, hkv = self.heads
        y, mean, rstd = ctx.picasso_layer_norm_forward(self.x, self.gamma, self.beta, stream=stream)
        q, k, v = y.view(-1, hq + 2 * hkv, self.d).split([hq, hkv, hkv], dim=1)
        out, lse = ctx.picasso_attention_forward(q, k, v, self.o, causal=True, stream=stream)
        # (the gradients of q, k, v as parts of y's)
        with torch.cuda.stream(stream):    # (this one is the program's own)
            gy = torch.empty_like(y)
        parts = gy.view(-1, hq + 2 * hkv, self.d).split([hq, hkv, hkv], dim=1)
        ctx.picasso_attention_backward(self.go, q, k, v, out, lse, self.o, causal=True, grads=parts, stream=stream)
        gx, gg, gb = ctx.picasso_layer_norm_backward(gy, self.x, self.gamma, mean, rstd, stream=stream)
        before = ctx.picasso_gradient_norm([gg, gb, gx], stream=stream)
        norm = ctx.picasso_clip_gradients([gg, gb, gx], 0.5, stream=stream)
        return y, mean, rstd, out, lse, gy, gx, gg, gb, before, norm

    def equal(self, got, want):
        return all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.fixture(params=SIZES, ids=lambda s: f"{s[0]}-{s[1]}-{s[2]}-{s[3]}-{s[4]}")
def block(request):
    return Block(*request.param, seed=3)


def test_as_a_block(ctx, block):
    """The bits of two passes agree, and the clipped gradients have the norm that they were clipped to."""
    want = block.run(ctx)
    assert block.equal(block.run(ctx), want)
    assert torch.equal(want[-1], want[-2]) and float(want[-1]) > 0.5
    clipped = torch.cat([t.double().reshape(-1) for t in want[6:9]]).norm()
    assert abs(float(clipped) - 0.5) <= 0.5 * torch.finfo(block.x.dtype).eps + 1e-6


def test_on_a_stream_of_its_own(ctx, block):
    want = block.run(ctx)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for given in (False, True):   # as the current one, and named while another is current
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            busy = torch.randn(1 << 24, device="cuda").sin_()   # (the stream has work in front)
            if not given:
                got = block.run(ctx)
        if given:
            got = block.run(ctx, stream=side)
        side.synchronize()
        assert block.equal(got, want), given
        del busy


def test_a_named_stream_is_told_to_the_allocator(ctx, block):
    """Results and workspaces of calls on a named stream, dropped at once, are not handed out again before that stream is through."""
    want = block.run(ctx)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    kept = []
    for _ in range(4):
        with torch.cuda.stream(side):
            torch.randn(1 << 25, device="cuda").sin_()
        got = block.run(ctx, stream=side)
        kept.append(got[-3:])
        del got
        junk = [torch.full_like(t, 9.0) for t in want]       # (on the current stream, into whatever the allocator has)
        del junk
    side.synchronize()
    for k in kept:
        assert block.equal(k, want[-3:])


def test_what_the_current_stream_still_writes_is_not_handed_out(ctx, block):
    """Memory that the current stream has freed while its own kernels on it are still to come is none for a call on a named stream, which does
    not wait for them; and a result that the current stream still reads when it is dropped is not handed out again before."""
    want = block.run(ctx)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        b = a
        for _ in range(20):
            b = b @ a                                            # (some milliseconds in front of what follows on this stream)
        junk = [torch.full_like(t, 9.0) for t in want]
        del junk, b
        got = block.run(ctx, stream=side)
        side.synchronize()
        torch.cuda.synchronize()
        assert block.equal(got, want)
        b = a
        for _ in range(20):
            b = b @ a
        got[5].record_stream(torch.cuda.current_stream())        # (gy, the program's own)
        copies = [t.clone() for t in got]                        # read by the current stream, late
        del got, b
        with torch.cuda.stream(side):
            junk = [torch.full_like(t, 9.0) for t in want]
        torch.cuda.synchronize()
        assert block.equal(copies, want)
        del junk, copies


def test_recorded_into_a_graph(ctx, block):
    want = block.run(ctx)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = block.run(ctx)
    other = Block([33, 200], 2, 2, 32, torch.float32, 9)
    first = other.run(ctx)
    x0, go0 = block.x.clone(), block.go.clone()
    for i in range(4):
        for t in got:
            t.fill_(-3.0)
        if i == 2:   # other inputs in the recorded places
            block.x.copy_(x0.flip(0)), block.go.copy_(go0.flip(0))
            want = block.run(ctx)
        graph.replay()
        assert other.equal(other.run(ctx), first)            # eager work right behind
        torch.cuda.synchronize()
        assert block.equal(got, want), f"replay {i}"
    block.x.copy_(x0), block.go.copy_(go0)


def test_two_graphs_and_eager_calls_together(ctx):
    """Two recorded passes on two streams beside an eager one on a third, again and again."""
    blocks = [Block(*s, seed=i) for i, s in enumerate(SIZES[:3])]
    want = [b.run(ctx) for b in blocks]
    torch.cuda.synchronize()
    graphs, got, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for b in blocks[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append(b.run(ctx))
    for i in range(5):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        eager = blocks[2].run(ctx)
        torch.cuda.synchronize()
        assert blocks[2].equal(eager, want[2])
        assert all(b.equal(x, w) for b, x, w in zip(blocks, got, want)), i


def test_from_several_threads_on_one_context(ctx):
    blocks = [Block(*s, seed=10 + i) for i, s in enumerate(SIZES)]
    want = [b.run(ctx) for b in blocks]
    torch.cuda.synchronize()
    wrong, gate = [], threading.Barrier(len(blocks))

    def work(i):
        try:
            s = torch.cuda.Stream()
            gate.wait()
            with torch.cuda.stream(s):
                for n in range(8):
                    got = blocks[i].run(ctx)
                    s.synchronize()
                    if not blocks[i].equal(got, want[i]):
                        wrong.append((i, n))
        except Exception as e:  # noqa: BLE001
            wrong.append((i, repr(e)))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(blocks))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_another_current_device(ctx, block):
    if torch.cuda.device_count() < 2:
        pytest.skip("one device")
    want = block.run(ctx)
    torch.cuda.synchronize(0)
    with torch.cuda.device(1):
        hq, hkv = block.heads
        y, mean, rstd = ctx.picasso_layer_norm_forward(block.x, block.gamma, block.beta)
        norm = ctx.picasso_gradient_norm([block.x])
        assert torch.cuda.current_device() == 1 and y.device.index == 0 and norm.device.index == 0
        torch.cuda.synchronize(0)
        assert torch.equal(y, want[0])
        with pytest.raises(TypeError):
            ctx.picasso_layer_norm_forward(block.x, stream=torch.cuda.Stream(device=1))
