"""Every form of the gradient's kernels against the float64 oracle, with the bounds of tests/test_gpu_policy_gradient.py: long uncut rows of each width (what a thread keeps in
registers, and the second sweep behind that), rows in slices, rows without a distribution in each of them, slices in a captured graph."""
import numpy as np
import pytest

from oracle import update as ou
from test_gpu_policy_gradient import check, make, matrix, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,V,dtype,pad,offset", [(97, 151937, "float32", 3, 1), (98, 50257, "float32", 0, 0), (97, 81924, "float32", 0, 0), (101, 100003, "float16", 1, 1),
                                                  (99, 65543, "float16", 0, 0), (97, 152064, "bfloat16", 8, 0), (96, 131077, "bfloat16", 1, 1), (50, 70003, "float32", 2, 1)])
@pytest.mark.parametrize("ratio", [True, False])
def test_long_rows_of_every_form(n, V, dtype, pad, offset, ratio):
    import torch
    from paper_2506_24119_amd import binding as sb
    rng = np.random.default_rng(n + V)
    x, y, adv, mask = make(rng, n, V, masked=0.8)
    mask[[0, n - 1]] = 1                                               # the first and the last row count
    y[[0, n - 1]] = [0, V - 1]
    whole, rows = matrix(n, V, dtype, pad, offset)
    rows.copy_(torch.from_numpy(x))
    live = np.flatnonzero((mask != 0) & (y >= 0))
    x = rows[torch.from_numpy(live).cuda()].float().cpu().numpy()
    old = None
    if ratio:
        old = np.zeros(n, np.float32)
        old[live] = ou.objective(x, y[live], None, adv[live], None, 0.8, 0)[1] + 0.2 * rng.normal(size=len(live))
    gw, grad = matrix(n, V, dtype, pad, offset)
    lp = run(sb, rows, y, old, adv, mask, 0.8, 0.2, 1.0 / n, grad)
    g = grad[torch.from_numpy(live).cuda()].float().cpu().numpy()
    check(x, y[live], None if old is None else old[live], adv[live], None, 0.8, float(np.float32(0.2)), float(np.float32(1.0 / n)), lp[live], g, dtype)
    dead = np.setdiff1d(np.arange(n), live)
    assert (lp[dead] == 0).all() and (grad[torch.from_numpy(dead).cuda()] == 0).all().item()
    lp2 = run(sb, rows, y, old, adv, mask, 0.8, 0.2, 1.0 / n, rows)    # in place
    assert np.array_equal(lp, lp2) and torch.equal(grad, rows)


@pytest.mark.parametrize("times,V,dtype", [(1, 70000, "float32"), (1, 140000, "bfloat16"), (1, 131077, "float16"), (7, 70001, "float32"), (7, 90000, "float32"), (7, 70001, "bfloat16")])
@pytest.mark.parametrize("ratio", [True, False])
def test_odd_rows_of_every_form(times, V, dtype, ratio):
    """14 rows, in slices, and seven times 14, which are not cut."""
    import torch
    from paper_2506_24119_amd import binding as sb
    rng = np.random.default_rng(V)
    n = 14
    x, y, adv, _ = make(rng, n, V, masked=0.0)
    y[:] = np.maximum(y, 0)
    old = np.full(n, -3.0, np.float32) if ratio else None
    x[0] = -np.inf                                                     # no distribution
    x[1, V - 1] = np.nan                                               # in the last, scalar part or the last slice
    x[2, V // 2] = np.inf
    y[3], y[4], y[5] = V, 0x7FFFFFFF, -5                               # no such entry, twice; no target
    x[6, y[6]] = -np.inf                                               # the target is masked out
    x[7] = -np.inf
    x[7, y[7]] = 4.0                                                   # nothing but the target
    x[8] = float(torch.finfo(getattr(torch, dtype)).min)               # masked by the type's lowest value
    x[8, 3] = 0.0
    x[9] = -1e4
    x[10] = 0.0
    x[11, rng.random(V) < 0.9] = -np.inf
    x[11, : V // 2] = -np.inf                                          # whole slices of nothing
    x[11, y[11]] = 1.0
    mask = np.ones(n, np.int32)
    mask[12] = 0
    x[12] = np.nan                                                     # does not count: not looked at
    rep = lambda a: None if a is None else np.tile(a, times)  # noqa: E731
    N = n * times
    whole, rows = matrix(N, V, dtype, 0, 0)
    rows.copy_(torch.from_numpy(x).repeat(times, 1))
    _, grad = matrix(N, V, dtype, 0, 0)
    lp = run(sb, rows, rep(y), rep(old), rep(adv), rep(mask), 1.0, 0.2, 0.5, grad)
    g = grad.view(times, n, V)
    bits = torch.int32 if dtype == "float32" else torch.int16
    for t in range(1, times):                                          # each of the copies is the first
        assert torch.equal(g[t].view(bits), g[0].view(bits))
        assert np.array_equal(lp[t * n:(t + 1) * n], lp[:n], equal_nan=True)
    x, lp, g = rows[:n].float().cpu().numpy(), lp[:n], g[0].float().cpu().numpy()
    for i in (0, 1, 2, 3, 4):
        assert np.isnan(lp[i]) and np.isnan(g[i]).all(), i
    assert lp[5] == lp[12] == 0 and (g[5] == 0).all() and (g[12] == 0).all()
    assert np.isneginf(lp[6])
    good = [6, 7, 8, 9, 10, 11, 13]
    sub = lambda a: None if a is None else a[good]  # noqa: E731
    check(x[good], y[good], sub(old), adv[good], None, 1.0, float(np.float32(0.2)), 0.5, lp[good], g[good], dtype)


@pytest.mark.parametrize("n,V,dtype", [(3, 140000, "bfloat16"), (40, 70001, "float32"), (97, 90001, "float32")])
def test_captured_slices_and_long_rows_replay(n, V, dtype):
    import torch
    from paper_2506_24119_amd import binding as sb
    rng = np.random.default_rng(10)
    x, y, adv, mask = make(rng, n, V)
    whole, rows = matrix(n, V, dtype, 0, 0)
    _, grad = matrix(n, V, dtype, 0, 0)
    first = torch.from_numpy(x).cuda()
    rows.copy_(first)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    yt, at, mt = dev(y), dev(adv), dev(mask)
    logp = torch.empty(n, device="cuda")
    ws = torch.empty(sb.spiral_policy_gradient_workspace_bytes(n, V), dtype=torch.uint8, device="cuda")
    call = lambda gr: sb.spiral_policy_gradient(rows, yt, None, at, mt, 1.0, 0.0, 1.0, logp, gr, ws)  # noqa: E731
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(grad)
    torch.cuda.synchronize()
    gph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gph, stream=side):
        call(grad)
    for r in range(4):
        rows.copy_(first.roll(r, 1))
        at.copy_(dev(np.roll(adv, r)))
        grad.fill_(9.0)
        ws.fill_(0xA5)
        gph.replay()
        torch.cuda.synchronize()
        got, lp = grad.clone(), logp.clone()
        again = torch.empty_like(got)
        call(again)
        torch.cuda.synchronize()
        assert torch.equal(got, again) and torch.equal(lp, logp)
