"""The linear layers' and norms' host side: descriptors, plans (decoded here from their documented layout), refusals."""
import ctypes

import numpy as np
import pytest

import paper_1802_10280_amd as esc
import feedforward as ff


def unrounded(raw, type):
    """Values of a type from a plan's bytes."""
    if type == 0:
        return raw.view(np.float32).astype(np.float64)
    if type == 1:
        return raw.view(np.float16).astype(np.float64)
    return (raw.view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def internal(w, gated):
    """Rows in the plan's order: a gate's, its partner's, and so on."""
    return w if not gated else np.stack([w[:len(w) // 2], w[len(w) // 2:]], axis=1).reshape(w.shape)


def decode_kept(plan, h, rows, K):
    size = 4 if h["type"] == 0 else 2
    rt, ct = -(-rows // 16), -(-K // 128)
    mask = plan[h["off_mask"]:h["off_mask"] + rt * ct * 256].view(np.uint32).reshape(rt, ct, 64)
    start = plan[h["off_start"]:h["off_start"] + (rt * ct + 1) * 4].view(np.uint32)
    out = np.zeros((rt * 16, ct * 128))
    most = 0
    for r in range(rt):
        for c in range(ct):
            t = r * ct + c
            n = sum(bin(int(m)).count("1") for m in mask[r, c])
            at = h["off_kept"] + int(start[t]) * 16
            taken = -(-n * size // 16) * 16
            # runs of 2048 rows start where they would with the most padding
            assert int(start[t + 1]) * 16 - int(start[t]) * 16 == taken or ((r + 1) % 128 == 0 and c == ct - 1 and int(start[t + 1]) * 16 >= int(start[t]) * 16 + taken)
            assert not plan[at + n * size:h["off_kept"] + int(start[t + 1]) * 16].any()
            values = iter(unrounded(plan[at:at + n * size], h["type"]))
            begin = 0
            for lane in range(64):
                n = bin(int(mask[r, c, lane])).count("1")
                most = max(most, (begin % 4 + n * size + 3) // 4)
                begin += n * size
                for bit in range(32):
                    if mask[r, c, lane] >> bit & 1:
                        out[r * 16 + lane % 16, c * 128 + bit // 8 * 32 + lane // 16 * 8 + bit % 8] = next(values)
    assert most == h["most_lane_words"]
    return out


def decode_whole(plan, h, rows, K):
    size = 4 if h["type"] == 0 else 2
    rf, cf, half = -(-rows // 32), -(-K * size // 128) * 4, 16 // size
    raw = unrounded(plan[h["off_whole"]:h["off_whole"] + rf * cf * 1024], h["type"]).reshape(rf, cf, 2, 32, half)
    return raw.transpose(0, 3, 1, 2, 4).reshape(rf * 32, cf * 2 * half)


@pytest.mark.parametrize("type", [0, 1, 2])
@pytest.mark.parametrize("K,M,gated,sparsity", [(1, 1, False, 0.0), (7, 5, True, 0.5), (128, 16, False, 0.0), (129, 33, False, 0.7),
                                                 (300, 20, True, 0.9), (64, 40, False, 1.0), (65, 3, True, 0.3), (130, 2100, False, 0.8),
                                                 (9, 2500, True, 0.5), (3, 6200, False, 0.4)])
def test_plan_holds_the_weights(type, K, M, gated, sparsity):
    rows = 2 * M if gated else M
    w, (rowptr, colidx, value) = ff.pruned(rows, K, sparsity, 7 * K + M, type)
    for T in (1, 100000):
        d = esc.make_linear_desc(T, K, M, type, gated)
        size = esc.escoin_linear_plan_size(d, rowptr, colidx)
        plan = np.full(size + 64, 0xA5, dtype=np.uint8)
        esc.escoin_linear_plan_build(d, rowptr, colidx, value, plan[:size])
        assert (plan[size:] == 0xA5).all()
        h = esc.linear_plan_header(plan)
        assert h["total_bytes"] == size and h["most_tokens"] == T and esc.escoin_linear_few_tokens(d, plan) == h["few_tokens"]
        assert not plan[h["off_zero"]:h["off_zero"] + 256].any()
        want = internal(w, gated)
        got = decode_kept(plan, h, rows, K)
        np.testing.assert_array_equal(got[:rows, :K], want)
        assert not got[rows:].any() and not got[:, K:].any()
        if T > h["few_tokens"]:
            got = decode_whole(plan, h, rows, K)
            np.testing.assert_array_equal(got[:rows, :K], want)
            assert not got[rows:].any() and not got[:, K:].any()


def test_equal_builds_give_equal_bytes():
    d = esc.make_linear_desc(1000, 70, 9000, esc.T_F16)
    _, csr = ff.pruned(9000, 70, 0.6, 5, 1)
    n = esc.escoin_linear_plan_size(d, *csr[:2])
    first = esc.escoin_linear_plan_build(d, *csr, plan=np.full(n, 0x5A, dtype=np.uint8))
    for fill in (0, 0xFF):
        assert (esc.escoin_linear_plan_build(d, *csr, plan=np.full(n, fill, dtype=np.uint8)) == first).all()


def test_plan_takes_any_order_and_adds_up_repeats():
    K, M = 200, 3
    rowptr = np.array([0, 5, 5, 8], dtype=np.int32)
    colidx = np.array([199, 3, 3, 0, 3, 7, 7, 150], dtype=np.int32)
    value = np.array([1.0, 0.5, 0.25, 2.0, 0.125, 3.0, -3.0, 0.0], dtype=np.float32)
    d = esc.make_linear_desc(1, K, M, esc.T_F32)
    plan = esc.escoin_linear_plan_build(d, rowptr, colidx, value)
    got = decode_kept(plan, esc.linear_plan_header(plan), M, K)
    want = np.zeros((16, 256))
    want[0, [199, 3, 0]] = [1.0, 0.875, 2.0]
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("type", [1, 2])
def test_plan_rounds_weights_to_nearest_even(type):
    import torch
    rng = np.random.default_rng(3)
    bits = np.concatenate([rng.integers(0, 2 ** 32, 20000, dtype=np.uint64).astype(np.uint32),
                           # ties, the subnormals' edges, the largest numbers, infinities, NaN
                           (np.arange(0x33000000 - 3, 0x33000000 + 3)).astype(np.uint32), np.arange(0x387fe000, 0x38802000, 0x800, dtype=np.uint32),
                           np.arange(0x477fe000, 0x47801000, 0x200, dtype=np.uint32), np.array([0x7f800000, 0xff800000, 0x7fc00000, 0x7f800001, 0x7f7fffff, 0x3f808000, 0x3f818000,
                                                                                                 0x3f801000, 0x3f803000, 1, 0x80000000], dtype=np.uint32)])
    v = bits.view(np.float32)
    want = torch.from_numpy(v.copy()).to(ff.torch_type(type)).double().numpy()
    d = esc.make_linear_desc(1, len(v), 1, type)
    plan = esc.escoin_linear_plan_build(d, np.array([0, len(v)], dtype=np.int32), np.arange(len(v), dtype=np.int32), v)
    np.testing.assert_array_equal(decode_kept(plan, esc.linear_plan_header(plan), 1, len(v))[0, :len(v)], want)


def test_linear_descriptors():
    ok = dict(T=3, K=10, M=4, type=esc.T_BF16)
    assert esc.escoin_linear_check_desc(esc.make_linear_desc(**ok)) == esc.OK
    assert esc.escoin_linear_check_desc(esc.make_linear_desc(**{**ok, "T": 0})) == esc.OK
    for bad in (dict(T=-1), dict(K=0), dict(M=-5), dict(type=3), dict(type=-1), dict(gated=2), dict(ld_in=9), dict(ld_out=3), dict(ld_residual=-4)):
        assert esc.escoin_linear_check_desc(esc.make_linear_desc(**{**ok, **bad})) == esc.EINVAL, bad
    for far in (dict(K=1 << 22), dict(M=1 << 29), dict(ld_in=1 << 40), dict(K=(1 << 22) - 1, M=1 << 28)):
        assert esc.escoin_linear_check_desc(esc.make_linear_desc(**{**ok, **far})) == esc.ERANGE, far
    assert esc.lib().escoin_linear_check_desc(None) == esc.EINVAL


def test_plan_refusals():
    d = esc.make_linear_desc(1, 6, 2, esc.T_F32)
    rp, ci, v = np.array([0, 1, 3], dtype=np.int32), np.array([0, 5, 2], dtype=np.int32), np.ones(3, dtype=np.float32)
    good = esc.escoin_linear_plan_build(d, rp, ci, v)
    for rowptr, colidx in (([1, 1, 3], [0, 5, 2]), ([0, 2, 1], [0, 5, 2]), ([0, 1, 3], [0, 6, 2]), ([0, 1, 3], [0, -1, 2])):
        with pytest.raises(esc.EscoinError) as e:
            esc.escoin_linear_plan_build(d, np.array(rowptr, dtype=np.int32), np.array(colidx, dtype=np.int32), v)
        assert e.value.code == esc.EINVAL
    with pytest.raises(esc.EscoinError) as e:
        esc.escoin_linear_plan_build(d, rp, ci, v, good[:-1].copy())
    assert e.value.code == esc.ESIZE
    for args in ((rp[:2], ci, v), (rp, ci[:2], v), (rp, ci, v[:2]), (rp.astype(np.int64), ci, v), (rp, ci, v.astype(np.float64))):
        with pytest.raises(TypeError):
            esc.escoin_linear_plan_build(d, *args)
    L, n = esc.lib(), ctypes.c_size_t(0)
    assert L.escoin_linear_plan_size(ctypes.byref(d), None, None, ctypes.byref(n)) == esc.EINVAL
    assert L.escoin_linear_plan_size(ctypes.byref(d), rp.ctypes.data, ci.ctypes.data, None) == esc.EINVAL
    assert L.escoin_linear_plan_build(ctypes.byref(d), rp.ctypes.data, ci.ctypes.data, None, good.ctypes.data, good.nbytes) == esc.EINVAL
    assert L.escoin_linear_plan_build(ctypes.byref(d), rp.ctypes.data, ci.ctypes.data, v.ctypes.data, None, 1 << 20) == esc.EINVAL
    with pytest.raises(TypeError):
        esc.escoin_linear_few_tokens(d, good[:16].copy())


def test_forward_refuses_before_any_launch():
    L, one, two = esc.lib(), ctypes.c_void_p(256), ctypes.c_void_p(512)
    d = esc.make_linear_desc(4, 6, 2, esc.T_F32)
    rp, ci, v = np.array([0, 1, 3], dtype=np.int32), np.array([0, 5, 2], dtype=np.int32), np.ones(3, dtype=np.float32)
    plan = esc.escoin_linear_plan_build(d, rp, ci, v)

    def call(desc=d, plan=plan, d_plan=one, d_in=one, d_out=two, bias=None, residual=None, flags=0):
        return L.escoin_linear_forward(ctypes.byref(desc), plan.ctypes.data if plan is not None else None, d_plan, d_in, d_out, bias, residual, flags, None)

    other = plan.copy()
    other[0] ^= 1
    for kw in (dict(plan=None), dict(plan=other), dict(d_plan=None), dict(d_in=None), dict(d_out=None), dict(d_out=one),
               dict(flags=esc.F_BIAS), dict(flags=esc.F_RESIDUAL), dict(flags=64), dict(flags=esc.F_RELU | esc.F_SILU), dict(flags=esc.F_GELU | esc.F_GELU_TANH),
               dict(d_plan=ctypes.c_void_p(264)), dict(d_in=ctypes.c_void_p(258)), dict(d_out=ctypes.c_void_p(514)),
               dict(flags=esc.F_BIAS, bias=ctypes.c_void_p(257)), dict(flags=esc.F_RESIDUAL, residual=ctypes.c_void_p(1026)),
               dict(desc=esc.make_linear_desc(4, 6, 2, esc.T_F32, ld_out=3), flags=esc.F_RESIDUAL, residual=two),
               # a plan of another layer, or for fewer tokens
               dict(desc=esc.make_linear_desc(5, 6, 2, esc.T_F32)), dict(desc=esc.make_linear_desc(4, 7, 2, esc.T_F32)),
               dict(desc=esc.make_linear_desc(4, 6, 1, esc.T_F32)), dict(desc=esc.make_linear_desc(4, 6, 2, esc.T_BF16)),
               dict(desc=esc.make_linear_desc(4, 6, 2, esc.T_F32, gated=True)), dict(desc=esc.make_linear_desc(4, 0, 2, esc.T_F32))):
        assert call(**kw) == esc.EINVAL, kw
    assert call(desc=esc.make_linear_desc(0, 6, 2, esc.T_F32), d_in=None, d_out=None) == esc.OK      # nothing to do


def test_norm_refuses_before_any_launch():
    L, p = esc.lib(), [ctypes.c_void_p(256 * (i + 1)) for i in range(4)]
    ok = dict(T=2, D=8, type=esc.T_BF16, post=esc.NORM_RMS, pre=esc.NORM_RMS)
    assert esc.escoin_norm_check_desc(esc.make_norm_desc(**ok)) == esc.OK
    for bad in (dict(T=-1), dict(D=0), dict(type=7), dict(post=3), dict(pre=-1), dict(gate_rows=2), dict(eps=-1.0), dict(eps=float("nan")),
                dict(alpha=float("inf")), dict(beta=float("nan")), dict(weight_offset=float("inf")), dict(ld_x=7), dict(ld_n=-8), dict(ld_gate=1)):
        assert esc.escoin_norm_check_desc(esc.make_norm_desc(**{**ok, **bad})) == esc.EINVAL, bad
    assert esc.escoin_norm_check_desc(esc.make_norm_desc(**{**ok, "ld_y": 1 << 40})) == esc.ERANGE
    assert esc.escoin_norm_check_desc(esc.make_norm_desc(**{**ok, "D": 1 << 30})) == esc.ERANGE

    def call(desc=ok, x=p[0], y=p[1], gate=None, pw=None, pb=None, nw=None, nb=None, h=p[2], n=p[3]):
        d = esc.make_norm_desc(**desc)
        return L.escoin_norm_forward(ctypes.byref(d), x, y, gate, pw, pb, nw, nb, h, n, None)

    none = {**ok, "post": esc.NORM_NONE, "pre": esc.NORM_NONE}
    odd = ctypes.c_void_p(4097)
    for kw in (dict(x=None), dict(y=None), dict(h=None, n=None), dict(n=p[2]), dict(desc=none, pw=p[0]), dict(desc=none, nb=p[0]),
               dict(desc={**ok, "post": esc.NORM_NONE}, y=None, gate=p[1]), dict(x=odd), dict(y=odd), dict(gate=odd), dict(pw=odd), dict(pb=odd),
               dict(nw=odd), dict(nb=odd), dict(h=odd), dict(n=odd), dict(desc={**ok, "ld_h": 9}, h=p[0]), dict(desc={**ok, "ld_y": 9}, n=p[1])):
        assert call(**kw) == esc.EINVAL, kw
    assert call(desc={**ok, "T": 0}, x=None) == esc.OK


def test_the_convolutions_refuse_the_new_flags():
    d = esc.make_desc(1, 3, 8, 9, 4, 3, 3, 2, 1)
    one = ctypes.c_void_p(256)
    for flag in (esc.F_RESIDUAL, esc.F_SILU, esc.F_GELU, esc.F_GELU_TANH):
        assert esc.lib().escoin_sconv_forward(ctypes.byref(d), one, one, one, one, one, one, flag, None) == esc.EINVAL


class Tensor:
    """What the binding looks at of a device tensor, without a device."""

    def __init__(self, shape, type=2, device=0, stride=None):
        self.shape, self.dtype, self.device = tuple(shape), ff.torch_type(type), device
        self.strides = stride or tuple(int(np.prod(shape[i + 1:])) for i in range(len(shape)))

    def get_device(self):
        return self.device

    def stride(self):
        return self.strides

    def numel(self):
        return int(np.prod(self.shape))

    def is_contiguous(self):
        return self.strides == tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))

    @property
    def nbytes(self):
        return self.numel() * (4 if self.dtype == ff.torch_type(0) else 2)

    def data_ptr(self):
        return 4096


def test_a_call_without_tensors_is_refused():
    with pytest.raises(TypeError):
        esc.escoin_norm_forward(esc.make_norm_desc(2, 8, esc.T_F32), None, None, None)


class Reached(Exception):
    pass


def test_the_binding_refuses_tensors_that_do_not_fit(monkeypatch):
    """Every refusal is raised before the library is called; the calls that are not refused reach it."""
    from paper_1802_10280_amd import binding

    def call(self, where, fn, *args, stream):
        raise Reached

    monkeypatch.setattr(binding._Rows, "call", call)
    T, K, M = 4, 64, 16
    d = esc.make_linear_desc(T, K, M, esc.T_BF16)
    _, csr = ff.pruned(M, K, 0.5, 1, 2)
    plan = esc.escoin_linear_plan_build(d, *csr)
    ok = dict(plan_host=plan, d_plan=Tensor([plan.nbytes // 2]), d_in=Tensor([T, K]), d_out=Tensor([T, M]), d_bias=Tensor([M]), d_residual=Tensor([T, M]))
    for good in ({}, dict(d_bias=None, d_residual=None), dict(d_in=Tensor([T + 1, K])), dict(d_plan=Tensor([plan.nbytes]))):
        with pytest.raises(Reached):
            esc.escoin_linear_forward(d, **{**ok, **good})
    for name, t in ok.items():
        if name == "plan_host":
            bad = [None, plan[:40], plan.astype(np.int8), plan[::2]]
        elif name == "d_plan":
            bad = [Tensor([plan.nbytes // 2], device=-1), Tensor([plan.nbytes // 2], device=1), Tensor([plan.nbytes // 2 - 1]), Tensor([plan.nbytes // 2], stride=(2,))]
        else:
            s = t.shape
            bad = [Tensor(s, 0), Tensor(s, 1), Tensor(s, device=-1), Tensor(s[:-1] + (s[-1] - 1,)), Tensor(s[:-1] + (s[-1] + 1,))]
            if len(s) == 2:
                bad += [Tensor((T - 1, s[1])), Tensor(s, stride=(1, T)), Tensor(s, stride=(s[1] + 1, 1)), Tensor((T * s[1],))]
            else:
                bad += [Tensor(s, stride=(2,))]
            if name != "d_in":
                bad += [Tensor(s, device=1)]
        for b in bad:
            with pytest.raises(TypeError):
                esc.escoin_linear_forward(d, **{**ok, name: b})
    wide = esc.make_linear_desc(T, K, M, esc.T_BF16, ld_in=K + 8)
    with pytest.raises(Reached):
        esc.escoin_linear_forward(wide, **{**ok, "d_in": Tensor([T, K], stride=(K + 8, 1))})
    with pytest.raises(TypeError):
        esc.escoin_linear_forward(wide, **ok)

    with pytest.raises(TypeError):
        esc.escoin_linear_forward(d, plan, ok["d_plan"], None, None)
    with pytest.raises(TypeError):
        esc.escoin_linear_forward(d, plan, ok["d_plan"], Tensor([T, K], device=-1), Tensor([T, M], device=-1))

    D = 24
    for rows in (0, 1):
        d = esc.make_norm_desc(T, D, esc.T_BF16, esc.NORM_RMS, esc.NORM_RMS, rows)
        gate = [T, D] if rows else [D]
        ok = dict(d_x=Tensor([T, D]), d_h=Tensor([T, D]), d_n=Tensor([T, D]), d_y=Tensor([T, D]), d_gate=Tensor(gate), d_post_weight=Tensor([D]),
                  d_post_bias=Tensor([D]), d_pre_weight=Tensor([D]), d_pre_bias=Tensor([D]))
        for good in ({}, dict(d_h=None), dict(d_n=None, d_pre_bias=None), dict(d_gate=None)):
            with pytest.raises(Reached):
                esc.escoin_norm_forward(d, **{**ok, **good})
        for name, t in ok.items():
            s = t.shape
            bad = [Tensor(s, 1), Tensor(s, device=-1), Tensor(s, device=1) if name != "d_gate" else Tensor(s, 0), Tensor(s[:-1] + (D - 1,)), Tensor(s[:-1] + (D + 1,))]
            bad += [Tensor((T - 1, D)), Tensor(s, stride=(1, T)), Tensor((T * D,))] if len(s) == 2 else [Tensor(s, stride=(2,)), Tensor((T, D))]
            for b in bad:
                with pytest.raises(TypeError):
                    esc.escoin_norm_forward(d, **{**ok, name: b})


def test_a_plans_copy_is_as_long_as_its_header_says(monkeypatch):
    """The host's part may be the header alone; the device's copy is what kernels read, and has to be whole all the same."""
    from paper_1802_10280_amd import binding

    def call(self, where, fn, *args, stream):
        raise Reached

    monkeypatch.setattr(binding._Rows, "call", call)
    T, K, M = 4, 640, 48
    d = esc.make_linear_desc(T, K, M, esc.T_BF16)
    plan = esc.escoin_linear_plan_build(d, *ff.pruned(M, K, 0.5, 1, 2)[1])
    x, out = Tensor([T, K]), Tensor([T, M])
    for host in (plan, plan[:256], np.concatenate([plan, plan[:64]])):
        with pytest.raises(Reached):
            esc.escoin_linear_forward(d, host, Tensor([plan.nbytes // 2]), x, out)
        for short in (128, plan.nbytes // 2 - 1):
            with pytest.raises(TypeError):
                esc.escoin_linear_forward(d, host, Tensor([short]), x, out)
    with pytest.raises(TypeError):
        esc.escoin_linear_forward(d, plan, None, x, out)


@pytest.mark.parametrize("type", [-1, 3, 99])
def test_the_binding_refuses_unknown_types_as_the_library_does(type):
    _, csr = ff.pruned(16, 64, 0.5, 1, 2)
    plan = esc.escoin_linear_plan_build(esc.make_linear_desc(4, 64, 16, esc.T_BF16), *csr)
    for call in (lambda: esc.escoin_linear_forward(esc.make_linear_desc(4, 64, 16, type), plan, Tensor([plan.nbytes // 2]), Tensor([4, 64]), Tensor([4, 16])),
                 lambda: esc.escoin_norm_forward(esc.make_norm_desc(4, 64, type), Tensor([4, 64]), None, Tensor([4, 64]))):
        with pytest.raises(esc.EscoinError) as e:
            call()
        assert e.value.code == esc.EINVAL
