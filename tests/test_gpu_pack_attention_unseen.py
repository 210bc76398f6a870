"""What a position does not see, in every width of head: undefined, infinite and very large elements of hidden tokens, keys that weigh nothing.

Bounds are those of the packed attention's other tests, of the elements that are compared."""
import numpy as np
import pytest

from oracle import block as ob
from test_gpu_pack_attention import FLOOR, HALF, Call, check_backward, check_forward, close, sb  # noqa: F401  (sb: the fixture)

pytestmark = pytest.mark.gpu
WIDTHS = [(4, 2, 32), (4, 2, 64), (7, 1, 128)]


def check_dq(c, rows):
    """dq of these rows, whose own bound no other row takes part in."""
    half, floor = HALF[c.dtype], FLOOR[c.dtype]
    q, k, v, dout, got = c.host("q", "k", "v", "dout", "dq")
    g, size = ob.attention_grad(q, k, v, dout, c.lens, c.scale)
    E = c.errors().T[rows][:, :, None] + q.shape[2] * 2.0 ** -23
    want, s = g[0][rows], size[0][rows]
    assert np.isfinite(want).all()
    most = np.abs(k[np.isfinite(k)]).max()
    close(got[rows], want, (2 * half + 6 * E) * s + half * np.abs(want) * (1 + half) + floor * (1 + max(c.lens) * c.scale * most), "dq")


@pytest.mark.parametrize("name,row,value", [("v", 70, np.nan), ("v", 12, np.inf), ("v", 99, -np.inf), ("k", 70, np.nan), ("k", 150, np.inf), ("q", 33, np.nan), ("dout", 65, np.nan), ("v", 159, np.nan)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("hq,hkv,hd", WIDTHS)
def test_hidden_elements(sb, name, row, value, dtype, hq, hkv, hd):  # noqa: F811
    """An undefined or infinite element: exactly what depends on it is undefined; dq of the rows before it in its tile is the oracle's."""
    import torch
    c = Call(sb, [40, 120, 35], hq, hkv, hd, dtype, seed=9)
    t = getattr(c, name)
    t[row, min(1, t.shape[1] - 1), hd - 3] = value
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    check_forward(c)
    first = 0 if row < 40 else 40
    check_dq(c, np.r_[0:row, first + (40, 120)[first > 0]:c.n])
    if not (name == "v" and np.isinf(value)):                # inf - inf somewhere along the row: which gradient is undefined is left open
        check_backward(c)
    else:
        q, k, v, dout = c.host("q", "k", "v", "dout")
        g, _ = ob.attention_grad(q, k, v, dout, c.lens, c.scale)
        others = np.r_[0:first, first + (40, 120)[first > 0]:c.n]
        for x, w in zip(c.host("dk", "dv"), g[1:]):
            assert np.isfinite(x[others]).all() and np.isfinite(w[others]).all()
    c.free()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("hq,hkv,hd", WIDTHS)
def test_rows_before_a_key_that_weighs_nothing(sb, dtype, hq, hkv, hd):  # noqa: F811
    """Keys with an element of -inf: rows behind them meet 0 times infinity in dq, those before them do not, in the same tile either."""
    import torch
    c = Call(sb, [50, 70, 33], hq, hkv, hd, dtype, seed=37)
    c.q[:, :, hd - 3] = c.q[:, :, hd - 3].abs() + 1
    c.k[torch.tensor([30, 49, 88, 118, 137, 152], device="cuda"), :, hd - 3] = -float("inf")
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    check_dq(c, np.r_[0:30, 50:88, 120:137])
    check_backward(c)
    c.free()


@pytest.mark.parametrize("hq,hkv,hd", WIDTHS + [(2, 2, 64), (16, 1, 32)])
def test_large_values_that_rows_do_not_see(sb, hq, hkv, hd):  # noqa: F811
    """A value whose product with the gradients of rows before it passes 32 bits: it is finite and hidden from them, its own rows have no gradient, so dk and dv of it are 0."""
    import torch
    c = Call(sb, [40, 101], hq, hkv, hd, "bfloat16", seed=51)
    tokens = [20, 39, 40 + 45, 40 + 100]
    for a, b, token in ((0, 20, 20), (40, 85, 85)):
        c.dout[a:b] = 100.0
        c.v[token] = 3e37
    c.v[39], c.v[140] = 3e37, 3e37
    c.dout[20:40] = 0.0
    c.dout[85:] = 0.0
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    check_backward(c)
    for t in (c.dq, c.dk, c.dv):
        assert torch.isfinite(t).all()
    assert not c.dk[tokens].any() and not c.dv[tokens].any()
    c.free()
