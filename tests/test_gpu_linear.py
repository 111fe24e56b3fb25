"""Pruned linear layers on the GPU against their definition in 64 bits: types, sizes about every tile's edge, epilogues, strides,
what a call may and may not touch, streams and graphs."""
import numpy as np
import pytest

import paper_1802_10280_amd as esc
import feedforward as ff
from feedforward import BIAS, GELU, GELU_TANH, RELU, RESIDUAL, SILU

gpu = pytest.mark.gpu
TYPES = pytest.mark.parametrize("type", [2, 1, 0], ids=["bf16", "f16", "f32"])


class Layer:
    def __init__(self, K, M, type, gated=False, sparsity=0.6, most=1 << 20, seed=1):
        import torch
        self.K, self.M, self.type, self.gated = K, M, type, gated
        self.rows = 2 * M if gated else M
        self.w, csr = ff.pruned(self.rows, K, sparsity, seed, type)
        self.plan = esc.escoin_linear_plan_build(esc.make_linear_desc(most, K, M, type, gated), *csr)
        self.few = esc.linear_plan_header(self.plan)["few_tokens"]
        self.d_plan = torch.from_numpy(self.plan).cuda()
        rng = np.random.default_rng(seed + 1)
        self.bias = ff.rounded(rng.standard_normal(self.rows) * 0.3, type)

    def inputs(self, T, seed=5):
        rng = np.random.default_rng(seed)
        return ff.rounded(rng.standard_normal((T, self.K)), self.type), ff.rounded(rng.standard_normal((T, self.M)), self.type)

    def forward(self, x, flags, residual=None, out=None, bias=None, ld=(0, 0, 0), stream=None):
        import torch
        T = x.shape[0]
        if out is None:
            out = torch.full((T, self.M), float("nan"), dtype=ff.torch_type(self.type), device="cuda")
        if bias is None and flags & BIAS:
            bias = ff.to_dev(self.bias, self.type)
        d = esc.make_linear_desc(T, self.K, self.M, self.type, self.gated, *ld)
        esc.escoin_linear_forward(d, self.plan, self.d_plan, x, out, bias, residual, flags, stream)
        return out

    def check(self, T, flags, what="", seed=5):
        x, r = self.inputs(T, seed)
        out = self.forward(ff.to_dev(x, self.type), flags, ff.to_dev(r, self.type) if flags & RESIDUAL else None)
        ref, limit = ff.linear64(x, self.w, self.type, flags, self.gated, self.bias if flags & BIAS else None, r if flags & RESIDUAL else None)
        ff.within(out, ref, limit, f"{what} T={T} K={self.K} M={self.M} flags={flags} gated={self.gated} {ff.NAMES[self.type]}")


SIZES = [(1, 1), (7, 5), (8, 16), (64, 31), (127, 33), (128, 32), (129, 17), (256, 64), (520, 130), (1001, 129), (2048, 48)]


@gpu
@TYPES
@pytest.mark.parametrize("K,M", SIZES)
def test_sizes(type, K, M):
    layer = Layer(K, M, type)
    for T in (1, 2, 15, 16, 17, 33, 63, 64, 65, 96, 129):
        layer.check(T, 0)


@gpu
@TYPES
@pytest.mark.parametrize("K,M", [(1, 1), (40, 3), (129, 17), (512, 64), (777, 65)])
def test_gated_sizes(type, K, M):
    layer = Layer(K, M, type, gated=True)
    for T in (1, 3, 16, 31, 64, 65, 130):
        layer.check(T, BIAS | SILU)


@gpu
@TYPES
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", [0, RELU, SILU, GELU, GELU_TANH])
def test_epilogues(type, gated, act):
    layer = Layer(200, 36, type, gated)
    for T in (3, 70):
        for rest in (0, BIAS, RESIDUAL, BIAS | RESIDUAL):
            layer.check(T, act | rest)


@gpu
@TYPES
@pytest.mark.parametrize("sparsity", [0.0, 0.3, 0.95, 1.0])
def test_sparsities(type, sparsity):
    layer = Layer(300, 70, type, sparsity=sparsity)
    for T in (1, 40, 100):
        layer.check(T, BIAS)


@gpu
@TYPES
def test_larger(type):
    """Many tiles, more than one workgroup to a compute unit, a last tile that is not whole in either direction."""
    layer = Layer(1040, 1500, type, sparsity=0.7)
    for T in (1, 37, 64, 300, 1030):
        layer.check(T, BIAS | RESIDUAL | GELU)
    layer = Layer(1000, 700, type, gated=True, sparsity=0.5)
    for T in (5, 600):
        layer.check(T, SILU)


@gpu
@TYPES
def test_rows_that_are_empty_or_full(type):
    import torch
    K, M = 260, 40
    w = np.zeros((M, K))
    w[3] = w[17, 100:] = 0.5
    w[39, 259] = -2.0
    layer = Layer(K, M, type)
    layer.w = w
    layer.plan = esc.escoin_linear_plan_build(esc.make_linear_desc(1000, K, M, type), *ff.to_csr(w))
    layer.d_plan = torch.from_numpy(layer.plan).cuda()
    for T in (1, 20, 90):
        layer.check(T, BIAS)


@gpu
@TYPES
@pytest.mark.parametrize("T", [1, 30, 64, 100])
@pytest.mark.parametrize("K,M,lead,pitch,gated", [(96, 40, 3, 7, False), (100, 21, 8, 24, False), (129, 33, 1, 0, True), (64, 64, 0, 64, True)])
def test_strided_and_unaligned_views(type, T, K, M, lead, pitch, gated):
    """Input, output and residual as columns of wider buffers that start anywhere; what lies beside them is NaN and stays as it was."""
    import torch
    layer = Layer(K, M, type, gated)
    x, r = layer.inputs(T)
    wide = {}
    for name, cols, value in (("in", K, x), ("out", M, None), ("residual", M, r)):
        ld = cols + lead + pitch
        buf = torch.full((T + 2, ld), float("nan"), dtype=ff.torch_type(type), device="cuda")
        view = buf[1:T + 1, lead:lead + cols]
        if value is not None:
            view.copy_(ff.to_dev(value, type))
        wide[name] = (buf, view, ld)
    layer.forward(wide["in"][1], BIAS | RESIDUAL | SILU, wide["residual"][1], out=wide["out"][1], ld=tuple(wide[k][2] for k in ("in", "out", "residual")))
    ref, limit = ff.linear64(x, layer.w, type, BIAS | RESIDUAL | SILU, gated, layer.bias, r)
    ff.within(wide["out"][1], ref, limit)
    outside = wide["out"][0].clone()
    outside[1:T + 1, lead:lead + M] = float("nan")
    assert outside.isnan().all()


@gpu
@TYPES
@pytest.mark.parametrize("T", [2, 64, 150])
def test_the_residual_in_place(type, T):
    layer = Layer(300, 68, type)
    x, r = layer.inputs(T)
    out = ff.to_dev(r, type)
    layer.forward(ff.to_dev(x, type), RESIDUAL, out, out=out)
    ff.within(out, *ff.linear64(x, layer.w, type, RESIDUAL, False, None, r))


@gpu
@TYPES
@pytest.mark.parametrize("T", [3, 40, 140])
def test_inf_and_nan_stay_with_their_token(type, T):
    layer = Layer(200, 50, type, sparsity=0.5)
    x, _ = layer.inputs(T)
    bad = x.copy()
    bad[1, 77], bad[T - 1, 0] = np.inf, np.nan
    good = layer.forward(ff.to_dev(x, type), 0)
    got = layer.forward(ff.to_dev(bad, type), 0)
    rest = [t for t in range(T) if t not in (1, T - 1)]
    assert (got[rest].float() == good[rest].float()).all()
    assert not got[T - 1].isfinite().any() and not got[1].isfinite().any()


@gpu
@TYPES
def test_tokens_do_not_meet(type):
    """A token's outputs are the same bits whichever tokens stand beside it in a call of the same size."""
    layer = Layer(500, 60, type)
    for T in (20, 64, 200):
        x, _ = layer.inputs(T)
        x = ff.to_dev(x, type)
        whole = layer.forward(x, BIAS)
        turned = layer.forward(x.flip(0).contiguous(), BIAS)
        assert (turned.flip(0).float() == whole.float()).all()


@gpu
@TYPES
def test_rows_far_apart(type):
    """Offsets that pass 32 bits, counted in elements and in bytes."""
    import torch
    T, K, M = 3, 72, 40
    ld = (1 << 31) + 8
    layer = Layer(K, M, type)
    x, r = layer.inputs(T)
    store = torch.empty((T - 1) * ld + max(K, M), dtype=ff.torch_type(type), device="cuda")
    far = store.as_strided((T, K), (ld, 1))
    far.copy_(ff.to_dev(x, type))
    near = layer.forward(far, 0, ld=(ld, 0, 0))
    ref, limit = ff.linear64(x, layer.w, type, 0, False)
    ff.within(near, ref, limit)
    out = store.as_strided((T, M), (ld, 1))
    layer.forward(ff.to_dev(x, type), 0, out=out, ld=(0, ld, 0))
    ff.within(out, ref, limit)
    if type:      # the same with a plan and a batch that take the tiled kernel
        T = layer.few + 2
        ld = ((1 << 32) // T + 8) & ~7
        x, r = layer.inputs(T)
        far = store[:(T - 1) * ld + K].as_strided((T, K), (ld, 1))
        far.copy_(ff.to_dev(x, type))
        ff.within(layer.forward(far, 0, ld=(ld, 0, 0)), *ff.linear64(x, layer.w, type, 0, False))


@gpu
@TYPES
@pytest.mark.parametrize("T", [0, 1, 64, 200])
def test_graphs_and_streams(type, T):
    """Captured on a side stream, replayed with eager work between; equal calls give equal bits."""
    import torch
    layer = Layer(384, 96, type, gated=True)
    x = ff.to_dev(layer.inputs(max(T, 1))[0], type)[:T]
    out = torch.full((T + 1, layer.M), 7.0, dtype=ff.torch_type(type), device="cuda")
    layer.forward(x, SILU, out=out[:T])
    eager = out.clone()
    assert (out[T:] == 7.0).all()
    if T == 0:
        return
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer.forward(x, SILU, out=out[:T])
    for k in range(3):
        out.fill_(float(k))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert (out[:T] == eager[:T]).all() and (out[T:] == float(k)).all()
        assert (layer.forward(x * (k + 1), SILU).isfinite()).all()
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    layer.forward(x, SILU, out=out[:T], stream=side)
    side.synchronize()
    assert (out[:T] == eager[:T]).all()


@gpu
@pytest.mark.parametrize("K,M,T", [(1024, 2048, 64), (256, 4096, 1000), (256, 4096, 2048), (256, 8192, 2048)])
def test_graphs_of_kernels_with_much_lds(K, M, T):
    import torch
    layer = Layer(K, M, 2, sparsity=0.3)
    x = ff.to_dev(layer.inputs(T)[0], 2)
    out = torch.empty((T, M), dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(x, RELU, out=out)
    eager = layer.forward(x, RELU)
    for k in range(3):
        out.fill_(-1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert (out == eager).all()
        assert layer.forward(x, 0).isfinite().all()


@gpu
def test_one_plan_for_calls_of_every_length():
    layer = Layer(640, 80, 2)
    for T in (300, 1, 64, 65, 17, 2):
        layer.check(T, BIAS | GELU)
    few = Layer(640, 80, 2, most=10)
    few.check(10, 0)
    with pytest.raises(esc.EscoinError) as e:
        few.check(11, 0)
    assert e.value.code == esc.EINVAL


@gpu
def test_binding_refuses_what_does_not_fit():
    import torch
    layer = Layer(64, 16, 2)
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros(4, 16, dtype=torch.bfloat16, device="cuda")
    d = esc.make_linear_desc(4, 64, 16, esc.T_BF16)
    bias = torch.zeros(16, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(d_in=x.float()), dict(d_in=x.cpu()), dict(d_in=x[:3]), dict(d_in=x[:, :63]), dict(d_in=x.t().contiguous().t()), dict(d_out=out[:, :15]),
                dict(d_out=out.float()), dict(d_bias=bias[:15], flags=BIAS), dict(d_residual=out[:2], flags=RESIDUAL), dict(d_plan=layer.d_plan[:-1]),
                dict(d_plan=layer.d_plan.cpu())):
        kw = dict(plan_host=layer.plan, d_plan=layer.d_plan, d_in=x, d_out=out)
        kw.update(bad)
        with pytest.raises(TypeError):
            esc.escoin_linear_forward(d, **kw)


# The tiles of the kernel for many tokens, which goes by how they fill 256 compute units: 64 by 32, 64 by 64, one of 128 by 128 a
# unit, two, 256 by 256; a last step, row block and token block that are not whole.
@gpu
@pytest.mark.parametrize("type,K,M,T,gated", [
    (2, 200, 300, 300, False), (2, 200, 1020, 500, False), (2, 200, 4090, 1000, False), (2, 264, 4090, 2041, False), (1, 136, 8180, 2041, False),
    (2, 328, 4090, 2041, True), (1, 72, 2040, 1000, True), (2, 201, 4090, 1000, False), (1, 203, 2050, 300, True), (0, 100, 1500, 100, False),
    (0, 100, 2000, 500, False), (0, 100, 2040, 2041, False), (0, 101, 2040, 2041, False), (0, 68, 1020, 2041, True)])
def test_every_tile(type, K, M, T, gated):
    layer = Layer(K, M, type, gated)
    layer.check(T, BIAS | RESIDUAL | SILU)


@gpu
@pytest.mark.parametrize("type,K", [(2, 140001), (1, 140008), (0, 70003), (0, 70004)])
def test_long_rows(type, K):
    """More tiles to a wave than it has lanes to keep their starts in."""
    layer = Layer(K, 5, type, sparsity=0.97)
    for T in (1, 6, 20, 300):
        layer.check(T, 0)


@gpu
@pytest.mark.parametrize("type,K,M,T,gated", [(2, 12288, 1500, 100, False), (1, 12280, 750, 128, True), (0, 4096, 1024, 150, False), (0, 4097, 1000, 70, False)])
def test_kept_weights_for_many_tokens(type, K, M, T, gated):
    """Long rows, few of them: the kept weights are read for more tokens than a workgroup takes."""
    layer = Layer(K, M, type, gated, sparsity=0.9)
    assert layer.few >= T
    layer.check(T, BIAS | RESIDUAL | GELU_TANH)


@gpu
@TYPES
@pytest.mark.parametrize("act", [SILU, GELU_TANH])
@pytest.mark.parametrize("T", [3, 300])
def test_activations_far_below_zero(type, act, T):
    """z / (1 + exp(-u)) as long as the type holds it, where exp(-u) is beyond fp32.  Relative to the value: u is off by six half steps of
    itself (SiLU: by none), its product with log2 e and that one's distance from 64 by three more, each worth |u| of the value; an
    exponential and three products by eight."""
    K = 64
    layer = Layer(K, K, type)
    layer.w = np.eye(K)
    layer.plan = esc.escoin_linear_plan_build(esc.make_linear_desc(1000, K, K, type), *ff.to_csr(layer.w))
    import torch
    layer.d_plan = torch.from_numpy(layer.plan).cuda()
    z = ff.rounded(np.linspace(-110.0 if act == SILU else -11.0, 4.0, T * K).reshape(T, K), type)
    got = layer.forward(ff.to_dev(z, type), act).double().cpu().numpy()
    u = z if act == SILU else 2 * np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)
    ref = z / (1 + np.exp(-u))
    off = np.abs(ref) * ((9 if act == GELU_TANH else 3) * np.abs(u) + 8) * ff.F32
    ff.within(got, ref, off + ff.HALF[type] * (np.abs(ref) + off) + ff.TINY[type])
