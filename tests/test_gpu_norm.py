"""The norms between two blocks on the GPU against their definition in 64 bits: types, widths, kinds, gates, strides, places."""
import numpy as np
import pytest

import paper_1802_10280_amd as esc
import feedforward as ff

gpu = pytest.mark.gpu
TYPES = pytest.mark.parametrize("type", [2, 1, 0], ids=["bf16", "f16", "f32"])
KINDS = [(1, 1), (2, 2), (0, 1), (0, 2), (1, 0), (2, 1), (0, 0)]


def draw(T, D, type, seed, post, pre, gate, params):
    """x, y, gate, weights and biases: rows with a mean of their own, as a residual stream has."""
    rng = np.random.default_rng(seed)
    t = lambda a: ff.rounded(a, type)
    x, y = (t(rng.standard_normal((T, D)) * 2 + rng.standard_normal((T, 1))) for _ in range(2))
    g = {None: None, "vector": t(rng.standard_normal(D)), "token": t(rng.standard_normal((T, D)))}[gate]
    vec = lambda shift, used: t(rng.standard_normal(D) * 0.2 + shift) if used else None
    return x, y, g, vec(1, params and post), vec(0, params and post), vec(1, params and pre), vec(0, params and pre)


def run(desc, type, x, y, g, pw, pb, nw, nb, h=True, n=True):
    import torch
    dev = lambda a: ff.to_dev(a, type)
    new = lambda: torch.full(x.shape, float("nan"), dtype=ff.torch_type(type), device="cuda")
    out = [new() if h else None, new() if n else None]
    esc.escoin_norm_forward(desc, dev(x), *out, d_y=dev(y), d_gate=dev(g), d_post_weight=dev(pw), d_post_bias=dev(pb), d_pre_weight=dev(nw), d_pre_bias=dev(nb))
    return out


def check(T, D, type, post=1, pre=1, gate="vector", params=True, seed=3, alpha=0.75, beta=-1.5, offset=0.0, eps=1e-5):
    a = draw(T, D, type, seed + D, post, pre, gate, params)
    d = esc.make_norm_desc(T, D, type, post, pre, int(gate == "token"), eps, alpha, beta, offset)
    f32 = lambda v: float(np.float32(v))
    want = ff.block64(*a[:3], type, post, pre, f32(eps), f32(alpha), f32(beta), f32(offset), *a[3:])
    for got, (ref, limit) in zip(run(d, type, *a), want):
        ff.within(got, ref, limit, f"T={T} D={D} {ff.NAMES[type]} post={post} pre={pre} gate={gate}")


@gpu
@TYPES
@pytest.mark.parametrize("D", [1, 2, 7, 8, 63, 64, 65, 255, 256, 257, 511, 512, 520, 1000, 1024, 2047, 2048, 2056, 4095, 4096, 4104, 5003, 8192, 8200, 12288, 16384, 16392,
                               20001, 32768, 32776, 40000, 70001])
def test_widths(type, D):
    check(3, D, type)
    check(2, D, type, 2, 2, "token")


@gpu
@TYPES
@pytest.mark.parametrize("post,pre", KINDS)
@pytest.mark.parametrize("gate", [None, "vector", "token"])
def test_kinds_and_gates(type, post, pre, gate):
    for D in (96, 333, 4096, 9001):
        check(4, D, type, post, pre, gate, params=True)
        check(4, D, type, post, pre, gate, params=False, offset=1.0)
    check(3, 128, type, post, pre, gate, offset=1.0)


@gpu
@TYPES
@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 63, 1000, 4099])
def test_tokens(type, T):
    check(T, 200, type)
    check(T, 131, type, 2, 2)
    if T >= 1000:
        check(T, 1003, type)
        check(T, 4091, type, 1, 2)


@gpu
@TYPES
@pytest.mark.parametrize("D", [64, 77, 1000, 4096, 6001, 40000])
def test_no_block_and_single_outputs(type, D):
    """The norm before the first block (no y), and calls that want h or n alone."""
    T = 3
    x, y, g, pw, pb, nw, nb = draw(T, D, type, 11, 1, 2, "vector", True)
    d = esc.make_norm_desc(T, D, type, esc.NORM_NONE, esc.NORM_LAYER, alpha=2.0)
    (h, dh), (n, dn) = ff.block64(x, None, None, type, 0, 2, float(np.float32(1e-5)), 2.0, 1.0, 0.0, None, None, nw, nb)
    both = run(d, type, x, None, None, None, None, nw, nb)
    ff.within(both[0], h, dh)
    ff.within(both[1], n, dn)
    assert (run(d, type, x, None, None, None, None, nw, nb, h=False)[1] == both[1]).all()
    assert (run(d, type, x, None, None, None, None, nw, nb, n=False)[0] == both[0]).all()
    d = esc.make_norm_desc(T, D, type, esc.NORM_RMS, esc.NORM_LAYER)
    both = run(d, type, x, y, g, pw, pb, nw, nb)
    assert (run(d, type, x, y, g, pw, pb, nw, nb, h=False)[1] == both[1]).all()
    assert (run(d, type, x, y, g, pw, pb, nw, nb, n=False)[0] == both[0]).all()


@gpu
@TYPES
@pytest.mark.parametrize("D,lead,pitch", [(96, 3, 5), (128, 8, 24), (2001, 1, 0), (4096, 0, 64), (40000, 5, 3)])
def test_strided_views(type, D, lead, pitch):
    """Columns of wider buffers that start anywhere; NaN beside them, which stays."""
    import torch
    T, ld = 5, D + lead + pitch
    a = draw(T, D, type, 4, 2, 1, "token", True)
    bufs = []
    for value in (a[0], a[1], a[2], None, None):
        buf = torch.full((T + 2, ld), float("nan"), dtype=ff.torch_type(type), device="cuda")
        if value is not None:
            buf[1:T + 1, lead:lead + D] = ff.to_dev(value, type)
        bufs.append(buf)
    x, y, g, h, n = (b[1:T + 1, lead:lead + D] for b in bufs)
    d = esc.make_norm_desc(T, D, type, 2, 1, 1, 1e-5, 1.0, 0.5, 0.0, ld, ld, ld, ld, ld)
    par = [ff.to_dev(v, type) for v in a[3:]]
    esc.escoin_norm_forward(d, x, h, n, d_y=y, d_gate=g, d_post_weight=par[0], d_post_bias=par[1], d_pre_weight=par[2], d_pre_bias=par[3])
    for got, buf, (ref, limit) in zip((h, n), bufs[3:], ff.block64(*a[:3], type, 2, 1, float(np.float32(1e-5)), 1.0, 0.5, 0.0, *a[3:])):
        ff.within(got, ref, limit)
        outside = buf.clone()
        outside[1:T + 1, lead:lead + D] = float("nan")
        assert outside.isnan().all()


@gpu
@TYPES
@pytest.mark.parametrize("D", [64, 1000, 4096, 16384, 40000])
@pytest.mark.parametrize("where", ["h=x", "h=y", "n=x", "n=y", "h=x n=y"])
def test_in_place(type, D, where):
    import torch
    T = 4
    a = draw(T, D, type, 9, 1, 1, "vector", True)
    d = esc.make_norm_desc(T, D, type, 1, 1)
    apart = run(d, type, *a)
    x, y, g, pw, pb, nw, nb = (ff.to_dev(v, type) for v in a)
    new = lambda: torch.empty_like(x)
    h = x if "h=x" in where else y if "h=y" in where else new()
    n = x if "n=x" in where else y if "n=y" in where else new()
    esc.escoin_norm_forward(d, x, h, n, d_y=y, d_gate=g, d_post_weight=pw, d_post_bias=pb, d_pre_weight=nw, d_pre_bias=nb)
    assert (h == apart[0]).all() and (n == apart[1]).all()


@gpu
@TYPES
def test_extremes(type):
    """Rows of zeros, of one large value beside small ones, with an Inf or NaN: each row is on its own."""
    D = 300
    x = np.zeros((6, D))
    x[1] = 3.0
    x[2, 5], x[2, 7] = 30000.0, 1e-3
    x[3, 9], x[4, 9] = np.inf, np.nan
    x[5] = np.linspace(-1, 1, D)
    x = ff.rounded(x, type)
    for kind in (1, 2):
        for eps in (1e-5, 0.0):
            d = esc.make_norm_desc(6, D, type, 0, kind, eps=eps)
            got = run(d, type, x, None, None, None, None, None, None)[1]
            rows = [2, 5] + ([0, 1] if eps else [])
            ref, dev = ff.norm64(x[rows], np.zeros((len(rows), D)), kind, None, None, float(np.float32(eps)), 0.0)
            ff.within(got[rows], ref, dev + ff.HALF[type] * np.abs(ref) + ff.TINY[type] + 2.0 ** -140)
            assert got[4].isnan().all() and got[3].isnan().any()


@gpu
@TYPES
def test_rows_far_apart(type):
    import torch
    T, D, ld = 3, 520, (1 << 31) + 8
    x, y, g, pw, pb, nw, nb = draw(T, D, type, 2, 1, 1, "vector", True)
    store = torch.empty((T - 1) * ld + D, dtype=ff.torch_type(type), device="cuda")
    far = store.as_strided((T, D), (ld, 1))
    far.copy_(ff.to_dev(x, type))
    d = esc.make_norm_desc(T, D, type, 0, 1, ld_x=ld, ld_h=ld)
    n = torch.empty((T, D), dtype=far.dtype, device="cuda")
    dev = lambda a: ff.to_dev(a, type)
    esc.escoin_norm_forward(d, far, far, n, d_y=dev(y), d_pre_weight=dev(nw))
    (h, dh), (m, dm) = ff.block64(x, y, None, type, 0, 1, float(np.float32(1e-5)), 1.0, 1.0, 0.0, None, None, nw, None)
    ff.within(far, h, dh)
    ff.within(n, m, dm)


@gpu
@TYPES
@pytest.mark.parametrize("T", [0, 1, 3000])
def test_graphs_and_streams(type, T):
    import torch
    D = 1024
    x = torch.randn(max(T, 1), D, device="cuda").to(ff.torch_type(type))[:T]
    y = torch.randn(max(T, 1), D, device="cuda").to(x.dtype)[:T]
    h, n = (torch.full((T + 1, D), 5.0, dtype=x.dtype, device="cuda") for _ in range(2))
    d = esc.make_norm_desc(T, D, type, 1, 2)
    call = lambda stream=None: esc.escoin_norm_forward(d, x, h[:T], n[:T], d_y=y, stream=stream)
    call()
    eager = h.clone(), n.clone()
    assert (h[T:] == 5.0).all() and (n[T:] == 5.0).all()
    if T == 0:
        return
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for k in range(3):
        h.fill_(float(k))
        n.fill_(float(k))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert (h[:T] == eager[0][:T]).all() and (n[:T] == eager[1][:T]).all() and (h[T:] == float(k)).all()
        assert x.float().sum().isfinite()
    h.zero_()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    assert (h[:T] == eager[0][:T]).all()


@gpu
def test_binding_refuses_what_does_not_fit():
    import torch
    T, D = 4, 64
    d = esc.make_norm_desc(T, D, esc.T_BF16, 0, 1)
    x = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(D, dtype=torch.bfloat16, device="cuda")
    for args, kw in (((x.float(), None, x), {}), ((x.cpu(), None, x), {}), ((x[:3], None, x), {}), ((x[:, :63], None, x), {}), ((x, None, x.t()), {}),
                     ((x, None, x), dict(d_pre_weight=v[:63])), ((x, None, x), dict(d_pre_weight=v.float())), ((x, None, x), dict(d_y=x, d_gate=x))):
        with pytest.raises(TypeError):
            esc.escoin_norm_forward(d, *args, **kw)
    with pytest.raises(esc.EscoinError):
        esc.escoin_norm_forward(d, x, None, None)
