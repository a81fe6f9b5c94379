"""CPU-only checks of the calls for layer norm, attention and gradient clipping: what they refuse, they refuse before anything
touches a device (the context handed over is memory that is only looked at by calls that are accepted)."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2103_15076_amd as pk
    if not os.path.exists(pk.binding.LIB_PATH):
        from paper_2103_15076_amd import build
        build.build_library()
    return pk.load_library()


@pytest.fixture(scope="module")
def pk():
    import paper_2103_15076_amd as p
    return p


CTX = ctypes.cast(ctypes.create_string_buffer(1 << 16), ctypes.c_void_p)
P = [ctypes.c_void_p(0x100000 * (k + 1)) for k in range(12)]   # addresses that no refused call reads
BIG = 1 << 40


def heads(pk, data=0x100000, row=64, head=32):
    return ctypes.byref(pk.picasso_heads(data, row, head))


def forward(lib, pk, **change):
    a = dict(ctx=CTX, type=0, q=heads(pk, 0x100000, 128), k=heads(pk, 0x200000), v=heads(pk, 0x300000), qo=P[5], ko=P[6], B=1, Tq=10, Tk=10, Hq=4,
             Hkv=2, D=32, scale=1.0, out=heads(pk, 0x400000, 128), ws=P[9], bytes=BIG)
    a.update(change)
    return lib.picasso_attention_forward(a["ctx"], None, a["type"], a["q"], a["k"], a["v"], a["qo"], a["ko"], a["B"], a["Tq"], a["Tk"], a["Hq"],
                                         a["Hkv"], a["D"], 0, a["scale"], 1, a["out"], None, a["ws"], a["bytes"])


@pytest.mark.parametrize("change", [
    dict(ctx=None), dict(type=3), dict(type=-1), dict(q=None), dict(qo=None), dict(ko=None), dict(B=0), dict(B=(1 << 24) + 1), dict(Tq=-1), dict(Tk=-1),
    dict(Tk=(1 << 30) + 1), dict(Tq=1 << 30, Hq=4), dict(Hq=0), dict(Hkv=0), dict(Hkv=3), dict(Hq=65536, Hkv=65536), dict(D=0), dict(D=12), dict(D=136), dict(scale=0.0),
    dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_attention_forward(lib, pk, change):
    assert forward(lib, pk, **change) == pk.PICASSO_ERR_INVALID_ARG


def test_attention_arrays(lib, pk):
    for bad in (heads(pk, 0), heads(pk, 0x100008), heads(pk, 0x100000, 130), heads(pk, 0x100000, 128, 34), heads(pk, 0x100000, -128), heads(pk, 0x100000, 1 << 41)):
        assert forward(lib, pk, q=bad) == pk.PICASSO_ERR_INVALID_ARG
        assert forward(lib, pk, v=bad) == pk.PICASSO_ERR_INVALID_ARG
    # rows of an output on top of one another, and an output over an input
    assert forward(lib, pk, out=heads(pk, 0x400000, 0)) == pk.PICASSO_ERR_INVALID_ARG
    assert forward(lib, pk, out=heads(pk, 0x400000, 128, 0)) == pk.PICASSO_ERR_INVALID_ARG
    assert forward(lib, pk, out=heads(pk, 0x200010, 128)) == pk.PICASSO_ERR_INVALID_ARG
    # 16-bit features: strides of 8
    assert forward(lib, pk, type=1, q=heads(pk, 0x100000, 132)) == pk.PICASSO_ERR_INVALID_ARG


def test_attention_workspace(lib, pk):
    need = lib.picasso_attention_workspace_bytes(0, 1, 1, 100000, 4, 2, 32, 0)
    assert need > 0
    one = dict(Tq=1, Tk=100000, k=heads(pk, 0x10000000), v=heads(pk, 0x20000000))
    assert forward(lib, pk, **one, ws=None) == pk.PICASSO_ERR_WORKSPACE
    assert forward(lib, pk, **one, bytes=need - 1) == pk.PICASSO_ERR_WORKSPACE
    assert forward(lib, pk, **one, ws=ctypes.c_void_p(0x900008)) == pk.PICASSO_ERR_WORKSPACE
    assert lib.picasso_attention_workspace_bytes(0, 0, 1, 1, 4, 2, 32, 0) == 0
    back = lib.picasso_attention_workspace_bytes(2, 3, 500, 700, 4, 2, 64, 1)
    h = [heads(pk, 0x1000000 * (k + 1), 256, 64) for k in range(8)]
    args = lambda ws, n: lib.picasso_attention_backward(CTX, None, 2, *h[:5], P[0], P[1], P[2], 3, 500, 700, 4, 2, 64, 0, 1.0, 1, *h[5:], ws, n)  # noqa: E731
    assert back >= 500 * 4 * 4
    assert args(None, back) == pk.PICASSO_ERR_WORKSPACE and args(P[11], back - 1) == pk.PICASSO_ERR_WORKSPACE
    # sizes at their limits are counted in 64 bits
    assert lib.picasso_attention_workspace_bytes(0, 1, 1 << 28, 1 << 28, 4, 4, 128, 1) >= (1 << 28) * 4 * 4


def test_attention_backward(lib, pk):
    def call(**change):
        a = dict(ctx=CTX, lse=P[0], qo=P[1], D=32, scale=1.0)
        names = ["gout", "q", "k", "v", "out", "gq", "gk", "gv"]
        for k, n in enumerate(names):
            a[n] = heads(pk, 0x1000000 * (k + 1), 64 if n in ("k", "v", "gk", "gv") else 128)
        a.update(change)
        return lib.picasso_attention_backward(a["ctx"], None, 0, *(a[n] for n in names[:5]), a["lse"], a["qo"], P[2], 1, 10, 10, 4, 2, a["D"], 0,
                                              a["scale"], 1, *(a[n] for n in names[5:]), P[9], BIG)
    for change in (dict(ctx=None), dict(lse=None), dict(qo=None), dict(D=33), dict(scale=0.0), dict(gq=None), dict(gout=heads(pk, 0)),
                   dict(gv=heads(pk, 0x1000000, 64)), dict(gk=heads(pk, 0x3000000, 64)), dict(gq=heads(pk, 0x1000000, 128))):
        assert call(**change) == pk.PICASSO_ERR_INVALID_ARG, change


def test_layer_norm(lib, pk):
    def forward(ctx=CTX, type=0, x=P[0], N=8, C=16, eps=1e-5, y=P[1]):
        return lib.picasso_layer_norm_forward(ctx, None, type, x, N, C, None, None, eps, y, None, None)
    for change in (dict(ctx=None), dict(type=7), dict(x=None), dict(y=None), dict(N=-1), dict(C=0), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")),
                   dict(y=P[0]), dict(y=ctypes.c_void_p(P[0].value + 4)), dict(x=ctypes.c_void_p(P[0].value + 2))):
        assert forward(**change) == pk.PICASSO_ERR_INVALID_ARG, change
    assert forward(N=0) == pk.PICASSO_OK                      # nothing to do: no device is touched

    need = lib.picasso_layer_norm_workspace_bytes(0, 1000, 64)
    assert need >= 2 * 64 * 4 and lib.picasso_layer_norm_workspace_bytes(0, 1000, 0) == 0

    def backward(ctx=CTX, gy=P[0], x=P[1], N=1000, C=64, mean=P[2], rstd=P[3], gx=P[4], gg=P[5], gb=P[6], ws=P[7], n=need):
        return lib.picasso_layer_norm_backward(ctx, None, 0, gy, x, N, C, None, mean, rstd, gx, gg, gb, ws, n)
    for change in (dict(ctx=None), dict(gy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(N=-1), dict(C=0), dict(gx=None, gg=None, gb=None),
                   dict(gx=P[0]), dict(gx=P[1])):
        assert backward(**change) == pk.PICASSO_ERR_INVALID_ARG, change
    assert backward(ws=None) == pk.PICASSO_ERR_WORKSPACE and backward(n=need - 1) == pk.PICASSO_ERR_WORKSPACE


def test_clipping(lib, pk):
    def call(grads, sizes, types, out, max_norm=1.0, ws=P[9], n=BIG, ctx=CTX):
        k = len(sizes)
        a = lambda t, v: (t * max(k, 1))(*v)  # noqa: E731
        return lib.picasso_clip_gradients(ctx, None, k, a(ctypes.c_void_p, grads), a(ctypes.c_int64, sizes), a(ctypes.c_int32, types), max_norm,
                                          a(ctypes.c_void_p, out), None, ws, n)
    x, y = 0x100000, 0x200000
    assert call([x], [4], [0], [x], ctx=None) == pk.PICASSO_ERR_INVALID_ARG
    for bad in (([0], [4], [0], [x]), ([x], [4], [0], [0]), ([x], [-1], [0], [x]), ([x], [4], [3], [x]), ([x + 2], [4], [0], [y]), ([x], [4], [0], [y + 2]),
                ([x, x], [4, 4], [0, 0], [x, x]), ([x, y], [4, 4], [0, 0], [x, x + 8]), ([x, y], [4, 4], [0, 0], [y, x]), ([x], [4], [0], [x + 4]),
                ([x], [1 << 45], [0], [x])):
        assert call(*bad) == pk.PICASSO_ERR_INVALID_ARG, bad
    for bound in (-1.0, float("nan")):
        assert call([x], [4], [0], [x], max_norm=bound) == pk.PICASSO_ERR_INVALID_ARG
    assert call([x], [4], [0], [x], ws=None) == pk.PICASSO_ERR_WORKSPACE
    sizes = (ctypes.c_int64 * 2)(100, 10_000_000)
    need = lib.picasso_gradients_workspace_bytes(2, sizes)
    assert 8 <= need <= 1 << 16 and lib.picasso_gradients_workspace_bytes(0, None) >= 8
    assert call([x, 0x10000000], [100, 10_000_000], [0, 0], [x, 0x10000000], n=need - 1) == pk.PICASSO_ERR_WORKSPACE
    one = (ctypes.c_void_p * 1)(x)
    four, kind = (ctypes.c_int64 * 1)(4), (ctypes.c_int32 * 1)(0)
    assert lib.picasso_gradient_norm(CTX, None, 1, one, four, kind, None, P[9], BIG) == pk.PICASSO_ERR_INVALID_ARG
    assert lib.picasso_gradient_norm(CTX, None, 1, one, four, kind, P[1], None, BIG) == pk.PICASSO_ERR_WORKSPACE


@pytest.mark.parametrize("name", ["PK_RW", "PK_FS", "PK_KS", "PK_QS"])
@pytest.mark.parametrize("value", ["0", "1", "7", "-1"])
def test_the_environment_changes_no_plan(lib, monkeypatch, name, value):
    sizes = [(t, b, tq, tk, 4, 2, 64) for t in (0, 1) for b, tq, tk in ((1, 1, 100000), (3, 24000, 24000), (16, 960, 960000), (2, 50, 60))]
    ask = lambda: [lib.picasso_attention_workspace_bytes(*s, back) for s in sizes for back in (0, 1)]  # noqa: E731
    before = ask()
    monkeypatch.setenv(name, value)
    assert ask() == before


# ---- outputs over other arrays of a call.  (No call here is accepted: where nothing overlaps the workspace is missing.)


def backward(lib, pk, arrays, Tq, Tk, Hq, Hkv, D, lse=0x40000000, ws=None):
    """arrays: {name: (address, row stride, head stride)}, the others far from everything; float32."""
    names = ["gout", "q", "k", "v", "out", "gq", "gk", "gv"]
    far = {n: (0x100000000 * (i + 1), 1 << 12, 1 << 6) for i, n in enumerate(names)}
    h = [ctypes.byref(pk.picasso_heads(*{**far, **arrays}[n])) for n in names]
    return lib.picasso_attention_backward(CTX, None, 0, *h[:5], ctypes.c_void_p(lse), ctypes.c_void_p(0x50000000), ctypes.c_void_p(0x60000000), 1, Tq, Tk, Hq,
                                          Hkv, D, 0, 1.0, 1, *h[5:], ctypes.c_void_p(ws), BIG if ws else 0)


def test_parts_of_one_array(lib, pk):
    INVALID, WS = pk.PICASSO_ERR_INVALID_ARG, pk.PICASSO_ERR_WORKSPACE
    T, H, D = 100, 4, 32
    at = lambda part, base=0x10000000: (base + 4 * part * H * D, 3 * H * D, D)  # noqa: E731  [T, 3, H, D]
    qkv = dict(q=at(0), k=at(1), v=at(2))
    grads = dict(gq=at(0, 0x20000000), gk=at(1, 0x20000000), gv=at(2, 0x20000000))
    assert backward(lib, pk, {**qkv, **grads}, T, T, H, H, D) == WS
    for name in ("q", "k", "v"):                       # a gradient in place of an input that other workgroups still read
        for g in ("gq", "gk", "gv"):
            assert backward(lib, pk, {**qkv, **grads, g: qkv[name]}, T, T, H, H, D) == INVALID, (name, g)
    assert backward(lib, pk, {**qkv, **grads, "gk": grads["gv"]}, T, T, H, H, D) == INVALID
    assert backward(lib, pk, {**qkv, **grads, "gk": grads["gq"]}, T, T, H, H, D) == INVALID
    per_head = lambda part, base=0x10000000: (base + 4 * part * D, 3 * H * D, 3 * D)  # noqa: E731  [T, H, 3, D]
    both = dict(q=per_head(0), k=per_head(1), v=per_head(2), gq=per_head(0, 0x20000000), gk=per_head(1, 0x20000000), gv=per_head(2, 0x20000000))
    assert backward(lib, pk, both, T, T, H, H, D) == WS
    assert backward(lib, pk, {**both, "gv": both["gq"]}, T, T, H, H, D) == INVALID
    outermost = lambda part, base=0x10000000: (base + 4 * part * H * T * D, D, T * D)  # noqa: E731  [3, H, T, D]
    both = dict(q=outermost(0), k=outermost(1), v=outermost(2), gq=outermost(0, 0x20000000), gk=outermost(1, 0x20000000), gv=outermost(2, 0x20000000))
    assert backward(lib, pk, both, T, T, H, H, D) == WS
    assert backward(lib, pk, {**both, "gk": both["v"]}, T, T, H, H, D) == INVALID
    # rows and heads of one output over one another
    assert backward(lib, pk, dict(gq=(0x20000000, D, D)), T, T, H, H, D) == INVALID
    assert backward(lib, pk, dict(gq=(0x20000000, 3 * D, 2 * D)), T, T, H, H, D) == INVALID
    assert backward(lib, pk, dict(gq=(0x20000000, 2 * D, 1 << 20)), T, T, H, H, D) == WS
    # the statistics and the workspace
    assert backward(lib, pk, {**qkv, **grads}, T, T, H, H, D, lse=0x20000000 + 64) == INVALID
    assert backward(lib, pk, {**qkv, **grads}, T, T, H, H, D, ws=0x10000000) == INVALID
    assert backward(lib, pk, {**qkv, **grads}, T, T, H, H, D, ws=0x20000000) == INVALID
    assert backward(lib, pk, {**qkv, **grads}, T, T, H, H, D, ws=0x50000000 - 1024) == INVALID


def test_overlaps_against_a_count_of_bytes(lib, pk):
    """Two arrays of heads at random places: refused exactly where a byte is in both, if their strides are alike; where they differ, never
    without one."""
    import random
    rng = random.Random(7)
    seen = {True: 0, False: 0}
    for _ in range(4000):
        D = rng.choice((8, 16))
        T, S, H, G = rng.randint(1, 6), rng.randint(1, 6), rng.randint(1, 4), rng.randint(1, 2)
        G = G if H % G == 0 else 1
        strides = [(rng.randint(D // 4, 60) * 4, rng.randint(D // 4, 60) * 4) for _ in range(2)]
        alike = rng.random() < 0.7
        (r0, h0), (r1, h1) = strides[0], strides[0] if alike else strides[1]
        base, other = 0x10000000, 0x10000000 + 16 * rng.randint(-120, 120)
        cells = lambda p, n, r, m, h: [p // 4 + i * r + j * h + d for i in range(n) for j in range(m) for d in range(D)]  # noqa: E731
        # gk [S, G, D] against q [T, H, D]
        a, b = cells(base, S, r0, G, h0), cells(other, T, r1, H, h1)
        over = len(set(a)) < len(a) or bool(set(a) & set(b))
        st = backward(lib, pk, dict(gk=(base, r0, h0), q=(other, r1, h1)), T, S, H, G, D)
        assert st in (pk.PICASSO_ERR_INVALID_ARG, pk.PICASSO_ERR_WORKSPACE)
        refused = st == pk.PICASSO_ERR_INVALID_ARG
        if alike:
            assert refused == over, (D, T, S, H, G, r0, h0, other - base)
        else:
            assert not refused or over, (D, T, S, H, G, strides, other - base)
        seen[refused] += 1
    assert min(seen.values()) > 500


def test_forward_overlaps(lib, pk):
    INVALID, WS = pk.PICASSO_ERR_INVALID_ARG, pk.PICASSO_ERR_WORKSPACE
    T, n = 8, 100000                                    # few queries over many keys: split, so a workspace is needed

    def call(out, lse=0x70000000, ws=None, **change):
        a = dict(q=(0x10000000, 128, 32), k=(0x20000000, 192, 32), v=(0x20000000 + 256, 192, 32))
        a.update(change)
        h = {k: ctypes.byref(pk.picasso_heads(*x)) for k, x in dict(a, out=out).items()}
        return lib.picasso_attention_forward(CTX, None, 0, h["q"], h["k"], h["v"], ctypes.c_void_p(0x50000000), ctypes.c_void_p(0x60000000), 1, T, n, 4, 2, 32, 0,
                                             1.0, 1, h["out"], ctypes.c_void_p(lse), ctypes.c_void_p(ws), BIG if ws else 0)
    assert call((0x40000000, 128, 32)) == WS
    assert call((0x20000000 + 512, 192, 16)) == INVALID             # (heads over one another)
    assert call((0x20000000 + 256, 192, 32)) == INVALID             # in place of v, a part of a projection's output
    assert call((0x10000000, 128, 32)) == INVALID
    assert call((0x40000000, 128, 32), lse=0x40000040) == INVALID
    assert call((0x40000000, 128, 32), lse=0x20000000) == INVALID
    assert call((0x40000000, 128, 32), ws=0x40000000 - 4096) == INVALID
    assert call((0x40000000, 128, 32), ws=0x20001000) == INVALID
    assert call((0x40000000, 1 << 40, 1 << 40), T) == INVALID       # (an array of 2^43 values and more)


def test_layer_norm_overlaps(lib, pk):
    x, y, a, b, c, d, e, ws = (0x10000000 * (k + 1) for k in range(8))
    V = ctypes.c_void_p

    def forward(gamma=a, beta=b, out=y, mean=c, rstd=d):
        return lib.picasso_layer_norm_forward(CTX, None, 0, V(x), 100, 64, V(gamma), V(beta), 1e-5, V(out), V(mean), V(rstd))
    for change in (dict(out=a + 16), dict(out=b), dict(mean=y + 400), dict(rstd=c), dict(mean=x), dict(rstd=a), dict(out=x + 4)):
        assert forward(**change) == pk.PICASSO_ERR_INVALID_ARG, change
    need = lib.picasso_layer_norm_workspace_bytes(0, 100, 64)

    def backward(gx=c, gg=d, gb=e, w=ws, n=need):
        return lib.picasso_layer_norm_backward(CTX, None, 0, V(x), V(y), 100, 64, V(a), V(b), V(b + 1024), V(gx), V(gg), V(gb), V(w), n)
    assert backward(n=need - 1) == pk.PICASSO_ERR_WORKSPACE
    for change in (dict(gx=x), dict(gx=y), dict(gx=a), dict(gg=e), dict(gg=a), dict(gb=b), dict(gg=c + 64), dict(w=c), dict(w=x + 1024), dict(w=b), dict(gb=ws)):
        assert backward(**change) == pk.PICASSO_ERR_INVALID_ARG, change


def test_clipping_overlaps(lib, pk):
    x, y, norm, ws = 0x10000000, 0x20000000, 0x30000000, 0x40000000
    two, sizes, types, V = (ctypes.c_void_p * 2)(x, y), (ctypes.c_int64 * 2)(1000, 2000), (ctypes.c_int32 * 2)(0, 1), ctypes.c_void_p

    def clip(norm=norm, ws=ws, out=two, n=BIG):
        return lib.picasso_clip_gradients(CTX, None, 2, two, sizes, types, 1.0, out, V(norm), V(ws), n)

    def plain(norm=norm, ws=ws, n=BIG):
        return lib.picasso_gradient_norm(CTX, None, 2, two, sizes, types, V(norm), V(ws), n)
    assert clip(n=0) == pk.PICASSO_ERR_WORKSPACE and plain(n=0) == pk.PICASSO_ERR_WORKSPACE
    for f in (clip, plain):
        for change in (dict(norm=x + 40), dict(norm=y + 3996), dict(ws=x + 8), dict(ws=y), dict(norm=ws)):
            assert f(**change) == pk.PICASSO_ERR_INVALID_ARG, change
    to = (ctypes.c_void_p * 2)(0x50000000, 0x60000000)
    for change in (dict(norm=x), dict(norm=0x50000000 + 400), dict(ws=0x60000000)):
        assert clip(out=to, **change) == pk.PICASSO_ERR_INVALID_ARG, change


def test_attention_sizes_that_no_launch_holds(lib, pk):
    """Fewer than 2^24 workgroups of 128 rows or keys; a sequence takes one at least."""
    ask = lambda B, Tq, Tk, Hq=1: lib.picasso_attention_workspace_bytes(1, B, Tq, Tk, Hq, 1, 8, 1)  # noqa: E731
    most = (1 << 24) - 3                                             # sequences without rows
    assert ask(most, 1, 1) > 0 and ask(most + 1, 1, 1) == 0
    assert ask(most - 1, 128, 1) > 0 and ask(most, 128, 1) == 0 and ask(most, 1, 128) == 0 and ask(most, 32, 1, 4) == 0
    assert ask((1 << 23) - 3, 1 << 30, 1 << 30) > 0 and ask((1 << 23) - 2, 1 << 30, 1) == 0 and ask((1 << 23) - 2, 1, 1 << 30) == 0
    far = dict(q=heads(pk, 0x100000000, 128), k=heads(pk, 0x200000000), v=heads(pk, 0x300000000), out=heads(pk, 0x400000000, 128))
    assert forward(lib, pk, **far, B=most + 1) == pk.PICASSO_ERR_INVALID_ARG


def test_more_values_than_can_be_numbered(lib, pk):
    """Two tensors of 2^43 values were accepted, and nothing was done to them."""
    two = (ctypes.c_int64 * 2)
    for sizes in ((1 << 43, 1), (1 << 43, 1 << 43), (1 << 62, 1 << 62), (1, 1 << 44)):
        assert lib.picasso_gradients_workspace_bytes(2, two(*sizes)) == 0
        at, types = (ctypes.c_void_p * 2)(1 << 20, 1 << 60), (ctypes.c_int32 * 2)(0, 0)
        assert lib.picasso_gradient_norm(CTX, None, 2, at, two(*sizes), types, P[0], P[9], BIG) == pk.PICASSO_ERR_INVALID_ARG
        assert lib.picasso_clip_gradients(CTX, None, 2, at, two(*sizes), types, 1.0, at, None, P[9], BIG) == pk.PICASSO_ERR_INVALID_ARG
    assert lib.picasso_gradients_workspace_bytes(2, two(1 << 42, 1 << 42)) >= 256 * 8


@pytest.mark.parametrize("name", ["layer_norm_forward", "layer_norm_backward", "attention_forward", "attention_backward", "gradient_norm", "clip_gradients"])
def test_streams_of_another_device(pk, name):
    """Refused before any other argument is looked at (this one has no more)."""
    pytest.importorskip("torch")
    call = getattr(pk.binding._load_host(), name)

    class Stream:
        cuda_stream, device_index = 0, 1
    with pytest.raises(TypeError, match="stream of the context's"):
        call(CTX.value, 0, Stream())
    Stream.device_index = 0
    with pytest.raises(TypeError, match="too few"):
        call(CTX.value, 0, Stream())


@pytest.mark.parametrize("scale", [2.5e38, 3.4e38])
def test_scales_that_leave_the_range_in_units_of_a_bit(lib, pk, scale):
    far = dict(q=heads(pk, 0x100000000, 128), k=heads(pk, 0x200000000), v=heads(pk, 0x300000000), out=heads(pk, 0x400000000, 128))
    one = dict(far, Tq=1, Tk=100000, ws=None)      # (a call that lacks its workspace, so that none is accepted)
    assert forward(lib, pk, **one, scale=scale) == pk.PICASSO_ERR_INVALID_ARG
    assert forward(lib, pk, **one, scale=2.0 ** 127) == pk.PICASSO_ERR_WORKSPACE
    assert forward(lib, pk, **one, scale=1e-45) == pk.PICASSO_ERR_WORKSPACE


def test_clipping_overlaps_against_a_count_of_bytes(lib, pk):
    """Tensors at random places in a short stretch of memory, some in place, in any order: refused exactly where a byte that is written is in
    another tensor or in the norm."""
    import random
    rng = random.Random(11)
    seen = {True: 0, False: 0}
    for _ in range(6000):
        n = rng.randint(1, 5)
        base, room = 0x10000000, rng.choice((60, 400, 4000))
        sizes, types = [rng.randint(0, 12) for _ in range(n)], [rng.randint(0, 2) for _ in range(n)]
        at = [base + 4 * rng.randrange(room) for _ in range(n)]
        to = [a if rng.random() < 0.5 else base + 4 * rng.randrange(room) for a in at]
        norm = base + 4 * rng.randrange(room) if rng.random() < 0.5 else 0
        cells = lambda p, k: set(range(p, p + sizes[k] * (4 if types[k] == 0 else 2)))  # noqa: E731
        written, read = [cells(to[k], k) for k in range(n)] + [set(range(norm, norm + 4)) if norm else set()], [cells(at[k], k) if to[k] != at[k] else set() for k in range(n)]
        over = sum(map(len, written)) > len(set().union(*written)) or bool(set().union(*written) & set().union(*read))
        st = lib.picasso_clip_gradients(CTX, None, n, (ctypes.c_void_p * n)(*at), (ctypes.c_int64 * n)(*sizes), (ctypes.c_int32 * n)(*types), 1.0,
                                        (ctypes.c_void_p * n)(*to), ctypes.c_void_p(norm), None, 0)
        assert st in (pk.PICASSO_ERR_INVALID_ARG, pk.PICASSO_ERR_WORKSPACE)
        assert (st == pk.PICASSO_ERR_INVALID_ARG) == over, (at, to, sizes, types, norm)
        seen[over] += 1
    assert min(seen.values()) > 1000
