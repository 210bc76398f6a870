"""Weights far below half precision's normal range: a first token that takes nearly all of every row leaves the others 2^-20.

Bounds are those of the packed attention's other tests without what they grant weights below half precision's normal range."""
import numpy as np
import pytest

from oracle import block as ob
from test_gpu_pack_attention import HALF, Call, close, sb  # noqa: F401  (sb: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 32), (2, 2, 64), (4, 2, 64), (3, 3, 128), (7, 1, 128)])
@pytest.mark.parametrize("undefined", [False, True])
def test_values_of_small_weights(sb, dtype, hq, hkv, hd, undefined):  # noqa: F811
    """dv of tokens that every row weighs 2^-20: each weight is rounded by half a step of itself, also by heads shared out and where a row is undefined."""
    import torch
    lens = [200, 33]
    c = Call(sb, lens, hq, hkv, hd, dtype, seed=61, dscale=1024.0)
    c.q[:, :, 0] = 4.0
    c.k[:, :, 0] = 0.0
    c.k[[0, 200], :, 0] = 14.0 * float(np.sqrt(hd)) / 4.0
    if undefined:
        c.dout[70, 0, 1] = float("nan")
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    half = HALF[dtype]
    q, k, v, dout, got = c.host("q", "k", "v", "dout", "dv")
    (_, _, want), (_, _, size) = ob.attention_grad(q, k, v, dout, lens, c.scale)
    E = c.errors().max() + hd * 2.0 ** -23
    allowed = (half + 4 * E) * np.where(np.isfinite(size), size, 0) + half * np.abs(np.where(np.isfinite(want), want, 0)) * (1 + half) + 2.0 ** -25
    if dtype == "float16":                                    # the first token's own passes its range, as an infinity
        past = np.abs(want) > 65520 + allowed
        assert (got[past] == np.copysign(np.inf, want[past])).all()
        near = (np.abs(want) > 65504 - allowed) & ~past
        want = np.where(past | near, np.inf, want)
    close(got, want, allowed, "dv")
    for x in c.host("dq", "dk")[:2 * (not undefined)]:
        assert np.isfinite(x).all()
    c.free()


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 32), (2, 2, 64), (7, 1, 128)])
def test_outputs_of_small_weights(sb, dtype, hq, hkv, hd):  # noqa: F811
    """A first token that takes nearly all and is 0 itself: what remains are the others, of 2^-20 of its weight each, all rounded alike."""
    import torch
    lens = [200, 33, 500]
    c = Call(sb, lens, hq, hkv, hd, dtype, seed=67)
    c.q[:, :, 0] = 4.0
    c.k.zero_()
    first = torch.tensor([0, 200, 233], device="cuda")
    c.k[first, :, 0] = 14.03 * float(np.sqrt(hd)) / 4.0
    c.v[first] = 0.0
    c.forward()
    torch.cuda.synchronize()
    half = HALF[dtype]
    q, k, v, out = c.host("q", "k", "v", "out")
    want, size = (ob.attention(q, k, x, lens, c.scale)[0] for x in (v, np.abs(v)))
    close(out, want, (half + 2 * c.errors().T[:, :, None]) * size + half * np.abs(want) * (1 + half) + 2.0 ** -25, "out")
    c.free()


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_equal_scores_of_ten_millions(sb, dtype, hd):  # noqa: F811
    """One bit of a score is a unit there, but equal keys have the same bits: every row's output is the mean of what it sees, none of its weights past half precision's range."""
    import torch
    lens = [150, 40]
    c = Call(sb, lens, 4, 2, hd, dtype, seed=73)
    c.q.zero_()
    c.k.zero_()
    c.q[:, :, 0], c.k[:, :, 0] = 3000.0, 2.0 ** 15 * float(np.sqrt(hd / 64))
    c.forward()
    torch.cuda.synchronize()
    half = HALF[dtype]
    v, out = (x.astype(np.float64) for x in c.host("v", "out"))
    for a, n in ((0, 150), (150, 40)):
        count = np.arange(1, n + 1)[:, None, None]
        want, size = (np.repeat(np.cumsum(x[a:a + n], axis=0) / count, 2, axis=1) for x in (v, np.abs(v)))
        close(out[a:a + n], want, (half + 2.0 ** -24 * (n + 64)) * size + half * np.abs(want) * (1 + half) + 2.0 ** -25, "out")
    c.free()
