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
