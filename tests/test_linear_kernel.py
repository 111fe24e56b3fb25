"""Which kernel a linear layer's call takes, as the library tells it, and that what such a kernel reads of its LDS is its own."""
import ctypes
import re
import shutil
import subprocess

import numpy as np
import pytest

import paper_1802_10280_amd as esc
import feedforward as ff
import linear_cases as lc


def words_read(plan, rows, K, type):
    """The most words of its column that any lane reads while it unfolds a tile: 16-bit values four places at a time, three words from the
    next value's on; fp32 ones place by place."""
    h = esc.linear_plan_header(plan)
    tiles = -(-rows // 16) * -(-K // 128)
    mask = plan[h["off_mask"]:h["off_mask"] + tiles * 256].view(np.uint32).reshape(tiles, 64)
    there = (mask[:, :, None] >> np.arange(32, dtype=np.uint32) & 1).astype(np.int64)
    before = np.cumsum(there, 2) - there                    # of the lane, at each place
    if type == 0:
        return int(before.max()) + 1
    counts = there.sum(2)
    odd = (np.cumsum(counts, 1) - counts) & 1               # whether a lane's values start in the middle of a word
    return int(((before[:, :, ::4] + odd[:, :, None]) // 2).max()) + 3


def first_places(n):
    """A row of 128 columns in which each lane's first n places are kept."""
    w = np.zeros((16, 128))
    for lane in range(64):
        for b in range(n):
            w[lane % 16, b // 8 * 32 + lane // 16 * 8 + b % 8] = 1.0
    return w


def check(plan, desc, rows):
    seen = set()
    size = 4 if desc.type == 0 else 2
    most = esc.escoin_linear_few_tokens(desc, plan)
    for T in (1, 4, 5, 16, 17, 32, 33, 64, most):
        for address in (0, 2 * size):
            if T > min(most, desc.T):
                continue
            d = esc.make_linear_desc(T, desc.K, desc.M, desc.type, desc.gated)
            k = esc.escoin_linear_kernel(d, plan, address)
            assert k["kept"] and k["pieces"] * 4 >= min(esc.linear_plan_header(plan)["most_lane_words"], 32)
            assert words_read(plan, rows, desc.K, desc.type) <= k["lane_words"] and k["pieces"] * 4 <= k["lane_words"]
            inputs = k["tokens"] * 128 * size if k["inputs"] == 2 else 0
            assert 128 + k["waves"] * (k["lane_words"] * 256 + inputs) <= k["lds_bytes"] <= 160 * 1024
            assert 128 + k["waves"] * k["tokens"] * 64 <= k["lds_bytes"]         # the sums of all waves
            seen.add(k["pieces"])
    return seen


@pytest.mark.parametrize("type", [0, 1, 2])
@pytest.mark.parametrize("n", range(33))
def test_lanes_read_their_own_columns(type, n):
    """Every count of values, all in a lane's first places: the later ones are empty, and read behind the last value."""
    d = esc.make_linear_desc(64, 128, 16, type)
    plan = esc.escoin_linear_plan_build(d, *ff.to_csr(first_places(n)))
    check(plan, d, 16)


@pytest.mark.parametrize("type", [0, 1, 2])
def test_lanes_read_their_own_columns_at_any_sparsity(type):
    seen = set()
    for k, sparsity in enumerate((0.0, 0.2, 0.4, 0.5, 0.6, 0.7, 0.8, 0.9, 0.95, 0.97, 0.99, 1.0, 0.01)):
        d = esc.make_linear_desc(256, 700, 40, type, k % 2)
        plan = esc.escoin_linear_plan_build(d, *ff.pruned(80 if k % 2 else 40, 700, sparsity, 60 + k, type)[1])
        seen |= check(plan, d, 80 if k % 2 else 40)
    assert seen == ({1, 2, 3, 4, 5, 8} if type == 0 else {1, 2, 3, 4, 5})


def test_kernel_refusals():
    d = esc.make_linear_desc(4, 6, 2, esc.T_F32)
    plan = esc.escoin_linear_plan_build(d, *ff.pruned(2, 6, 0.5, 1, 0)[1])
    L, info = esc.lib(), esc.escoin_linear_kernel_info()
    call = lambda desc=d, plan=plan, at=None, to=info: L.escoin_linear_kernel(ctypes.byref(desc), None if plan is None else plan.ctypes.data, at, to and ctypes.byref(to))
    assert call() == esc.OK and info.kept == 1 and info.inputs == 0
    for kw in (dict(plan=None), dict(at=2), dict(to=None), dict(desc=esc.make_linear_desc(5, 6, 2, esc.T_F32)), dict(desc=esc.make_linear_desc(4, 7, 2, esc.T_F32)),
               dict(desc=esc.make_linear_desc(-1, 6, 2, esc.T_F32))):
        assert call(**kw) == esc.EINVAL, kw
    assert not any(esc.escoin_linear_kernel(esc.make_linear_desc(0, 6, 2, esc.T_F32), plan).values())


def compiled_kernels():
    """The names of the linear layers' kernels in the built library: waves multiplied out."""
    nm = shutil.which("nm")
    if nm is None:
        pytest.skip("no nm here")
    text = subprocess.run([nm, "-C", esc.binding.LIB_PATH], check=True, capture_output=True, text=True, timeout=120).stdout
    names = set(re.findall(r" (linear_(?:few|many)_kernel<[^>]*>)", text.replace("::", " ")))
    out = set()
    for n in names:
        if n.startswith("linear_many"):
            a = n[len("linear_many_kernel<"):-1].split(", ")
            n = f"linear_many_kernel<{', '.join(a[:5])}, {int(a[5]) * int(a[6]) * int(a[7])} waves, {a[8]}, {a[9]}>"
        out.add(n)
    assert len(out) == len(names)
    return out


def test_every_kernel_in_the_library_is_one_that_a_tested_call_takes():
    reached = set()
    for size, types in lc.TYPES.items():
        for type in types:
            for gated in (False, True):
                for case in [*lc.MANY, *lc.FEW]:
                    if case[0] != size:
                        continue
                    _, place, K, rows, T, kernel = case
                    d = esc.make_linear_desc(0, K, rows // 2 if gated else rows, type, gated)
                    empty = esc.escoin_linear_plan_build(d, np.zeros(rows + 1, np.int32), np.zeros(0, np.int32), np.zeros(0, np.float32))
                    for pieces in lc.PIECES[size] if case in lc.FEW else (1,):
                        k = lc.kernel_of(d, lc.header_with(empty, most_tokens=1 << 20, most_lane_words=4 * pieces), T, place)
                        if case in lc.FEW:
                            assert (k["kept"], k["inputs"], k["tokens"], k["pieces"]) == (1, *kernel, pieces), (case, k)
                        else:
                            assert (k["kept"], k["rows"], k["tokens"], k["steps"], k["step_bytes"]) == (0, *kernel), (case, k)
                        reached.add(lc.named(k, type, gated))
    assert reached == compiled_kernels()
