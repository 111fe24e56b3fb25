"""The check of a feed-forward block that smoke() makes: right hand-overs pass it, a mistake in any of them does not."""
import numpy as np
import pytest

import __graft_entry__ as entry
import feedforward as ff
from paper_1802_10280_amd import workloads as wl

NAMES = ["n", "g", "d", "h", "after"]


def handed_over(block):
    """What each step hands over, from its definition in 64 bits and rounded to bf16."""
    s = block.spec
    r = lambda a: ff.rounded(a, 2)

    def dense(csr, cols):
        w = np.zeros((len(csr[0]) - 1, cols))
        for m in range(len(w)):
            w[m, csr[1][csr[0][m]:csr[0][m + 1]]] = r(csr[2][csr[0][m]:csr[0][m + 1]])
        return w

    norm = lambda v, w: v / np.sqrt(np.square(v).sum(1, keepdims=True) / s.D + 1e-5) * r(w)
    x = r(block.x)
    n = r(norm(x, block.norm))
    z = n @ dense(block.up, s.D).T
    g = r(ff.act64(z[:, :s.F], ff.SILU) * z[:, s.F:])
    d = r(g @ dense(block.down, s.F).T)
    h = x + r(block.gate) * norm(d, block.post_norm)
    return dict(n=n, g=g, d=d, h=r(h), after=r(norm(h, block.next_norm)))


@pytest.fixture(scope="module", params=[3, 40])
def block(request):
    b = wl.make_block(wl.BlockSpec("t", request.param, 192, 320, "bf16", 0.6))
    return b, handed_over(b)


def test_right_hand_overs_pass(block):
    assert 0.0 < entry.check_block(block[0], **block[1]) <= 1.0


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("kind", ["scaled", "shifted", "one", "zeros", "nan", "other"])
def test_a_mistake_is_seen(block, name, kind):
    b, right = block
    v = right[name].copy()
    if kind == "scaled":
        v *= 1.05
    elif kind == "shifted":
        v = np.roll(v, 1, axis=1)
    elif kind == "one":
        i = np.unravel_index(np.argmax(np.abs(v)), v.shape)
        v[i] *= 1.02
    elif kind == "zeros":
        v[-1] = 0.0
    elif kind == "nan":
        v[0, 0] = np.nan
    else:
        v = np.random.default_rng(1).standard_normal(v.shape)
    with pytest.raises(AssertionError):
        entry.check_block(b, **{**right, name: v})
