"""The learner's operators on more rows, or sequences, than one launch has workgroups or a second dimension for: the last ones against the definition."""
import numpy as np
import pytest

from test_gpu_block_rows import U, sb  # noqa: F401  (sb: the fixture)

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


@pytest.mark.parametrize("n,d", [((1 << 24) + 4999, 8), ((1 << 22) + 1001, 5), ((1 << 24) + 77, 11)])
def test_norm(sb, n, d):  # noqa: F811
    import torch
    torch.manual_seed(1)
    x, gain = torch.randn((n, d), device="cuda").bfloat16(), 1 + 0.3 * torch.randn(d, device="cuda")
    out, rstd = torch.zeros_like(x), torch.zeros(n, device="cuda")
    codes, scale = torch.zeros((n, d), dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros(n, device="cuda")
    sb.spiral_add_rmsnorm(x, None, gain, 1e-6, out, None, None, rstd)
    sb.spiral_add_rmsnorm(x, None, gain, 1e-6, codes, scale)
    for rows in (slice(0, 5000), slice(n - 6000, n)):
        h = x[rows].double()
        r = 1 / (h.square().mean(1, keepdim=True) + float(np.float32(1e-6))).sqrt()
        want = h * r * gain.double()
        assert ((rstd[rows].double() - r[:, 0]).abs() <= 24 * U * r[:, 0]).all()
        assert ((out[rows].double() - want).abs() <= (HALF + 32 * U) * want.abs() * (1 + HALF) + 2.0 ** -133).all()
        p = h * gain.double()
        v = p * (448.0 / p.abs().amax(1, keepdim=True))
        step = torch.exp2(torch.clamp(torch.frexp(v)[1] - 1, min=-6).double() - 3)
        assert torch.equal(codes[rows].double(), torch.round(v / step) * step)
        assert ((scale[rows].double() - (p.abs().amax(1) * r[:, 0] / 448)).abs() <= 32 * U * scale[rows].double()).all()
    # every row written: the norm of none is 0
    assert (out.float().abs().amax(1) > 0).all() and (rstd > 0).all() and (scale > 0).all()


def test_rotation(sb):  # noqa: F811
    import torch
    n, hd = (1 << 24) + 515, 32
    torch.manual_seed(2)
    q, k = (torch.randn((n, 1, hd), device="cuda").bfloat16() for _ in range(2))
    pos = torch.arange(n, device="cuda", dtype=torch.int32)
    oq, ok = torch.zeros_like(q), torch.zeros_like(k)
    sb.spiral_norm_rope(q, k, None, None, 1e-6, 1e4, pos, oq, ok)
    for rows in (slice(0, 4000), slice(n - 4000, n)):
        a = pos[rows].double()[:, None] * 1e4 ** (-2.0 * torch.arange(hd // 2, device="cuda", dtype=torch.float64) / hd)
        for x, out in ((q, oq), (k, ok)):
            lo, hi = x[rows, 0].double().split(hd // 2, 1)
            want = torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], 1)
            size = torch.cat([lo.abs() + hi.abs()] * 2, 1)
            assert ((out[rows, 0].double() - want).abs() <= HALF * want.abs() * (1 + HALF) + 33 * U * size).all()
    assert (oq.float().abs().amax(2) > 0).all() and (ok.float().abs().amax(2) > 0).all()


def test_attention(sb):  # noqa: F811
    """70,001 sequences of one or two positions, with heads of a group: a position alone is its value, its dq and dk are nearly 0 and its dv the group's sum."""
    import torch
    torch.manual_seed(3)
    B, hq, hkv, hd = 70001, 4, 2, 32
    lens = np.where(np.arange(B) % 9 == 4, 2, 1).astype(np.int32)
    n = int(lens.sum())
    q, k, v, dout = (torch.randn((n, h, hd), device="cuda").bfloat16() for h in (hq, hkv, hkv, hq))
    out, dq, dk, dv = (torch.full_like(t, 7.0) for t in (q, q, k, v))
    lse = torch.full((hq, n), 7.0, device="cuda")
    mem = torch.empty(sb.spiral_attention_plan_bytes(lens, hq, hkv, hd), dtype=torch.uint8, device="cuda")
    plan = sb.spiral_attention_plan_create(lens, hq, hkv, hd, mem)
    ws = torch.empty(sb.spiral_attention_backward_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    scale = float(np.float32(hd ** -0.5))
    sb.spiral_attention_forward(plan, q, k, v, scale, out, lse)
    sb.spiral_attention_backward(plan, q, k, v, out, lse, dout, scale, dq, dk, dv, ws)
    torch.cuda.synchronize()
    starts = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)[:-1]])).cuda()
    ones = starts[torch.from_numpy(lens == 1).cuda()]
    v4, k4 = v.repeat_interleave(2, 1), k.repeat_interleave(2, 1)
    assert torch.equal(out[ones], v4[ones])
    s = (q.double() * k4.double()).sum(2) * scale
    assert ((lse.T[ones].double() - s[ones]).abs() <= 2.0 ** -24 * (2 * hd + 80) * ((q.double() * k4.double()).abs().sum(2)[ones] * scale + 1)).all()
    # dp - D: two sums of 32 bits of the same 32 products, p off by as many
    w = (dout.double() * v4.double()).abs().sum(2)
    small = (2 * hd + 80) * 2.0 ** -24 * 8 * w[ones][:, :, None] * scale
    assert (dq[ones].double().abs() <= small * k4[ones].double().abs() + 2.0 ** -133).all()
    assert (dk[ones].double().abs() <= (small * q[ones].double().abs()).unflatten(1, (2, 2)).sum(2) + 2.0 ** -133).all()
    want = dout[ones].double().unflatten(1, (2, 2)).sum(2)
    size = dout[ones].double().abs().unflatten(1, (2, 2)).sum(2)
    assert ((dv[ones].double() - want).abs() <= HALF * want.abs() * (1 + HALF) + (HALF + 2.0 ** -12) * size).all()
    # pairs: the second row's softmax over two
    b = starts[torch.from_numpy(lens == 2).cuda()] + 1
    x, y = (q[b].double() * k4[b - 1].double()).sum(2) * scale, s[b]
    p = torch.sigmoid(y - x)[:, :, None]
    want = (1 - p) * v4[b - 1].double() + p * v4[b].double()
    size = (1 - p) * v4[b - 1].double().abs() + p * v4[b].double().abs()
    assert ((out[b].double() - want).abs() <= (HALF + 2.0 ** -12) * size + HALF * want.abs() * (1 + HALF)).all()
    for t in (out, dq, dk, dv, lse):
        assert torch.isfinite(t).all() and not (t == 7.0).flatten(1).all(1).any()
    sb.spiral_attention_plan_free(plan)
