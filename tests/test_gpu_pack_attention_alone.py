"""Rows of packed attention with all their weight on one token: dp - D is 0 there, so are dq and dk, however large the scores are.

Bounds: dp and D are sums of hd products in 32 bits and D is a quotient of such, so dp - D is off by at most (2 hd + 8) 2^-24 of sum |dout||v|, with p no more than 1.01;
t is rounded by half a step and results once, in half precision by 2^-25 at least."""
import numpy as np
import pytest

from test_gpu_pack_attention import FLOOR, HALF, Call, sb  # noqa: F401  (sb: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 32), (2, 2, 64), (7, 1, 128)])
@pytest.mark.parametrize("lens", [[1] * 90, [64, 1, 40, 3, 0, 64]])
def test_no_gradient_of_a_weight_of_one(sb, lens, dtype, hq, hkv, hd):  # noqa: F811
    """Scores of 3,000 of each sequence's first token; the others' are some tens, their weights 0."""
    import torch
    c = Call(sb, lens, hq, hkv, hd, dtype, seed=71)
    big = float(np.sqrt(3000.0 * np.sqrt(hd)))
    first = np.concatenate([[0], np.cumsum(lens)[:-1]])[np.array(lens) > 0]
    c.q[:, :, 0] = big
    c.k[:, :, 0] = 0.0
    c.k[torch.from_numpy(first).cuda(), :, 0] = big
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    q, k, v, dout, dq, dk = (x.astype(np.float64) for x in c.host("q", "k", "v", "dout", "dq", "dk"))
    G, half, floor = hq // hkv, HALF[dtype], FLOOR[dtype]
    at = np.repeat(first, np.array(lens)[np.array(lens) > 0])                    # of each row, its sequence's first
    w = (np.abs(dout) * np.abs(np.repeat(v[at], G, axis=1))).sum(2, keepdims=True)
    t = c.scale * 1.01 * (2 * hd + 8) * 2.0 ** -24 * w * (1 + half) + c.scale * floor
    assert (np.abs(dq) <= t * np.abs(np.repeat(k[at], G, axis=1)) * (1 + half) + floor).all()
    of_first = np.zeros_like(k)
    np.add.at(of_first, at, (t * np.abs(q)).reshape(c.n, hkv, G, hd).sum(2))
    assert (np.abs(dk) <= of_first * (1 + half) + floor).all()
    c.free()
