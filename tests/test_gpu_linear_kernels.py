"""Every kernel of the linear layers on the GPU, each by a call that the library says it takes, against the definition in 64 bits."""
import numpy as np
import pytest

import paper_1802_10280_amd as esc
import feedforward as ff
import linear_cases as lc
from feedforward import BIAS, RESIDUAL, SILU

pytestmark = pytest.mark.gpu
FLAGS = BIAS | RESIDUAL | SILU


def run(type, gated, place, K, rows, T, sparsity, seed):
    """A call whose input rows lie at `place` in wider ones, NaN beside them; returns what the library told of its kernel."""
    import torch
    M = rows // 2 if gated else rows
    w, csr = ff.pruned(rows, K, sparsity, seed, type)
    desc = esc.make_linear_desc(1 << 20, K, M, type, gated)
    plan = esc.escoin_linear_plan_build(desc, *csr)
    rng = np.random.default_rng(seed + 1)
    x, r, bias = (ff.rounded(rng.standard_normal(s), type) for s in ((T, K), (T, M), (rows,)))
    ld = (K + 8 + 7) // 8 * 8
    wide = torch.full((T, ld), float("nan"), dtype=ff.torch_type(type), device="cuda")
    wide[:, place:place + K] = ff.to_dev(x, type)
    d_in = wide[:, place:place + K]
    out = torch.full((T + 1, M), float("nan"), dtype=wide.dtype, device="cuda")
    d = esc.make_linear_desc(T, K, M, type, gated, ld_in=ld)
    told = esc.escoin_linear_kernel(d, plan, d_in.data_ptr())
    call = lambda to: esc.escoin_linear_forward(d, plan, torch.from_numpy(plan).cuda(), d_in, to, ff.to_dev(bias, type), ff.to_dev(r, type), FLAGS)
    call(out)
    again = torch.empty_like(out)
    call(again)
    assert out[T:].isnan().all() and (out[:T] == again[:T]).all()
    within(out[:T], x, w, type, gated, bias, r)
    return told


def within(got, x, w, type, gated, bias, residual):
    """feedforward.linear64's definition and limit for FLAGS, on the GPU in 64 bits (its matrices are large here)."""
    import torch
    up = lambda a: torch.from_numpy(a).cuda()
    x, w, bias, residual = up(x), up(w), up(bias), up(residual)
    n = (w != 0).sum(1)[None, :] + 16
    dz = (n * 2 + 1) * ff.F32 * (x.abs() @ w.abs().t().contiguous())
    z = x @ w.t().contiguous() + bias
    dz += ff.F32 * 2 * (z.abs() + bias.abs())
    M = w.shape[0] // 2 if gated else w.shape[0]
    z, u = z[:, :M], z[:, M:]
    a = z / (1 + torch.exp(-z))
    da = 1.13 * dz[:, :M] + 16 * ff.F32 * z.abs()
    if gated:
        du = dz[:, M:]
        da = da * (u.abs() + du) + a.abs() * du + ff.F32 * (a * u).abs()
        a = a * u
    a = a + residual
    da = da + ff.F32 * a.abs()
    limit = da + ff.HALF[type] * (a.abs() + da) + ff.TINY[type] + 2.0 ** -140
    err = (got.double() - a).abs()
    bad = ~(err <= limit)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}"


def cases(table):
    return [pytest.param(*c[1:], type, gated, id="-".join([ff.NAMES[type], "gated" if gated else "plain", "wide" if c[1] == lc.WIDE else "any",
                                                           *map(str, c[5])]))
            for c in table for type in lc.TYPES[c[0]] for gated in (False, True)]


@pytest.mark.parametrize("place,K,rows,T,kernel,type,gated", cases(lc.MANY))
def test_tiled_kernels(place, K, rows, T, kernel, type, gated):
    k = run(type, gated, place, K, rows, T, 0.5, 70 + K)
    assert (k["kept"], k["rows"], k["tokens"], k["steps"], k["step_bytes"]) == (0, *kernel)


@pytest.mark.parametrize("place,K,rows,T,kernel,type,gated", cases(lc.FEW))
def test_kernels_for_few_tokens(place, K, rows, T, kernel, type, gated):
    for pieces, sparsity in lc.PIECES[4 if type == 0 else 2].items():
        k = run(type, gated, place, K, rows, T, sparsity, K + rows + pieces)
        assert (k["kept"], k["inputs"], k["tokens"], k["pieces"]) == (1, *kernel, pieces)


@pytest.mark.parametrize("K,M,T,kept", [(1032, 2124, 29, 1), (1032, 300, 13, 1), (2328, 522, 240, 1), (256, 4096, 1000, 0), (256, 8192, 2048, 0)])
def test_graphs_of_kernels_with_more_than_64_kb_of_lds(K, M, T, kept):
    import torch
    _, csr = ff.pruned(M, K, 0.3, K + T, 2)
    plan = esc.escoin_linear_plan_build(esc.make_linear_desc(1 << 20, K, M, esc.T_BF16), *csr)
    d_plan = torch.from_numpy(plan).cuda()
    d = esc.make_linear_desc(T, K, M, esc.T_BF16)
    x = torch.randn(T, K, device="cuda").bfloat16()
    out = torch.empty(T, M, dtype=torch.bfloat16, device="cuda")
    told = esc.escoin_linear_kernel(d, plan, x.data_ptr())
    assert told["kept"] == kept and told["lds_bytes"] > 64 * 1024
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        esc.escoin_linear_forward(d, plan, d_plan, x, out, flags=SILU)
    eager = torch.empty_like(out)
    for k in range(3):
        out.fill_(-1.0)
        eager.fill_(1.0)
        esc.escoin_linear_forward(d, plan, d_plan, x, eager, flags=SILU)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert (out == eager).all() and eager.isfinite().all()
        x.mul_(0.5)
