"""spiral_policy_gradient against the float64 oracle.

Bounds, in units of eps = 2^-24 (half a step of fp32): z = l / T is off by 2 |z|, an exponential's argument by 4 max|z| and the exponential by
that and 4 more; a sum of V such terms in runs of at most V / 256 adds V / 256 + 16.  The log-probability is off by R = eps (8 max|z| + 2 |logp| + V / 256 + 64),
the softmax and the slope relatively by as much again each (the ratio has the error of logp and of the given old one's 2 |old|), and the
result is rounded once to the output's type."""
import numpy as np
import pytest

from oracle import update as ou

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


@pytest.fixture(scope="module")
def sb():
    import torch
    assert torch.cuda.is_available()
    from paper_2506_24119_amd import binding
    binding.load_library()
    return binding


def matrix(n, V, dtype, pad, offset):
    import torch
    t = torch.full((n * (V + pad) + offset + 8,), 77.0, dtype=getattr(torch, dtype), device="cuda")
    return t, t[offset:offset + n * (V + pad)].view(n, V + pad)[:, :V]


def make(rng, n, V, masked=0.3, spread=2.0):
    y = rng.integers(0, V, n).astype(np.int32)
    x = (rng.normal(size=(n, V)) * spread).astype(np.float32)
    x[np.arange(n), y] += rng.uniform(0, 8, n).astype(np.float32)
    y[rng.random(n) < masked / 3] = -1
    return x, y, rng.normal(size=n).astype(np.float32), (rng.random(n) >= masked).astype(np.int32) * 3


def run(sb, rows, y, old, adv, mask, T, clip, scale, grad, stream=None):
    import torch
    n, V = rows.shape
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    logp = torch.full((n + 2,), 5.0, device="cuda")
    ws = torch.full((sb.spiral_policy_gradient_workspace_bytes(n, V),), 0xA5, dtype=torch.uint8, device="cuda")
    sb.spiral_policy_gradient(rows, dev(y), dev(old), dev(adv), dev(mask), T, clip, scale, logp[1:-1], grad, ws)
    torch.cuda.synchronize()
    lp = logp.cpu().numpy()
    assert lp[0] == lp[-1] == 5.0
    return lp[1:-1]


def check(x, y, old, adv, mask, T, clip, scale, lp, grad, dtype):
    want_lp, want, p, s = ou.policy_gradient(x, y, old, adv, mask, T, clip, scale)
    n, V = x.shape
    half = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[dtype]
    least = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}[dtype]
    z = np.abs(np.where(np.isfinite(x), x, 0).astype(np.float64)).max(axis=1) / T
    R = EPS * (8 * z + 2 * np.abs(np.nan_to_num(want_lp, neginf=0)) + V / 256 + 64)
    assert np.array_equal(np.isnan(lp), np.isnan(want_lp)) and np.array_equal(np.isneginf(lp), np.isneginf(want_lp))
    fine = np.isfinite(want_lp)
    assert (np.abs(lp - want_lp)[fine] <= R[fine]).all(), np.abs((lp - want_lp) / R)[fine].max()
    R = R + EPS * (2 * np.abs(np.nan_to_num(old, neginf=0)) if old is not None else 0)
    size = np.abs(want) + np.abs(s)[:, None] * p                       # at the target p - 1: each part has its own error
    allowed = 3 * R[:, None] * (size + np.abs(want)) + half * np.abs(want) * (1 + 3 * R[:, None]) + least
    bad = ~(np.abs(grad - want) <= allowed) & ~(np.isnan(grad) & np.isnan(want))
    # rows whose ratio is as near to the clip's edge as its error: either side of the kink is right
    if old is not None:
        r = np.exp(want_lp - old)
        edge = np.minimum(np.abs(r - (1 - clip)), np.abs(r - (1 + clip))) <= 2 * R
        assert edge.sum() <= 1 + n // 50
        bad[edge] = False
    assert not bad.any(), (np.argwhere(bad)[:4], grad[bad][:4], want[bad][:4])


@pytest.mark.parametrize("n,V,dtype,pad,offset", [(1, 151936, "float32", 0, 0), (3, 152064, "bfloat16", 0, 0), (5, 151937, "float16", 3, 1), (40, 40003, "bfloat16", 1, 0),
                                                  (9, 8209, "float32", 0, 1), (700, 1000, "float32", 0, 0), (257, 2048, "bfloat16", 8, 0), (4, 1, "float32", 0, 0),
                                                  (6, 3, "bfloat16", 0, 1), (33, 130, "float16", 2, 1), (2, 70000, "float32", 4, 4), (600, 16385, "bfloat16", 0, 0)])
@pytest.mark.parametrize("clip,T", [(0.2, 1.0), (None, 0.7), (0.0, 1.3)])
def test_log_probabilities_and_gradient(sb, n, V, dtype, pad, offset, clip, T):
    import torch
    rng = np.random.default_rng(n + V)
    x, y, adv, mask = make(rng, n, V, masked=0.3 if n > 3 else 0.0)
    whole, rows = matrix(n, V, dtype, pad, offset)
    rows.copy_(torch.from_numpy(x))
    x = rows.float().cpu().numpy()
    old = None
    if clip is not None:
        old = (ou.objective(x, y, None, adv, None, T, 0)[1] + 0.2 * rng.normal(size=n)).astype(np.float32)
    if n > 3:
        adv[1] = 0.0
    gw, grad = matrix(n, V, dtype, (pad * 3) % 7, offset)
    scale = 1.0 / n
    lp = run(sb, rows, y, old, adv, mask if n > 3 else None, T, clip or 0.0, scale, grad)
    check(x, y, old, adv, mask if n > 3 else None, T, clip or 0.0, np.float32(scale), lp, grad.float().cpu().numpy(), dtype)
    g = gw.float().cpu().numpy()                                       # what lies between and behind the rows is left as it was
    inside = np.zeros(g.shape, bool)
    step = V + (pad * 3) % 7
    for i in range(n):
        inside[offset + i * step:offset + i * step + V] = True
    assert (g[~inside] == 77.0).all()
    first = grad.clone()
    lp2 = run(sb, rows, y, old, adv, mask if n > 3 else None, T, clip or 0.0, scale, grad)
    assert np.array_equal(lp, lp2) and torch.equal(first, grad)        # bit for bit
    lp3 = run(sb, rows, y, old, adv, mask if n > 3 else None, T, clip or 0.0, scale, rows)          # in place
    assert np.array_equal(lp, lp3) and torch.equal(first, rows)


@pytest.mark.parametrize("n,V", [(14, 300), (14, 20000)])
@pytest.mark.parametrize("ratio", [True, False])
def test_odd_rows(sb, n, V, ratio):
    import torch
    rng = np.random.default_rng(8)
    x, y, adv, _ = make(rng, n, V, masked=0.0)
    y[:] = np.maximum(y, 0)
    old = np.full(n, -3.0, np.float32) if ratio else None
    x[0] = -np.inf                                                     # no distribution
    x[1, 5] = np.nan
    x[2, 7] = np.inf
    y[3] = V                                                           # no such entry
    y[4] = 0x7FFFFFFF
    y[5] = -5
    x[6, y[6]] = -np.inf                                               # the target is masked out
    x[7] = -np.inf; x[7, y[7]] = 4.0                                   # nothing but the target
    x[8] = np.finfo(np.float32).min; x[8, 3] = 0.0                     # masked by the type's lowest value
    x[9] = -1e4
    x[10] = 0.0
    x[11, rng.random(V) < 0.9] = -np.inf
    x[11, y[11]] = 1.0
    mask = np.ones(n, np.int32)
    mask[12] = 0
    x[12] = np.nan                                                     # does not count: not looked at
    whole, rows = matrix(n, V, "float32", 0, 0)
    rows.copy_(torch.from_numpy(x))
    _, grad = matrix(n, V, "float32", 0, 0)
    lp = run(sb, rows, y, old, adv, mask, 1.0, 0.2, 0.5, grad)
    g = grad.cpu().numpy()
    for i in (0, 1, 2, 3, 4):
        assert np.isnan(lp[i]) and np.isnan(g[i]).all(), i
    assert lp[5] == lp[12] == 0 and (g[5] == 0).all() and (g[12] == 0).all()
    assert np.isneginf(lp[6])
    good = [6, 7, 8, 9, 10, 11, 13]
    sub = lambda a: None if a is None else a[good]  # noqa: E731
    check(x[good], y[good], sub(old), adv[good], None, 1.0, 0.2, 0.5, lp[good], g[good], "float32")


def test_objective_values_follow_from_the_log_probabilities(sb):
    """What the learner calls together: the gradient, and the sums of the objective from its log-probabilities."""
    import torch
    rng = np.random.default_rng(9)
    n, V = 120, 5000
    x, y, adv, mask = make(rng, n, V)
    mask[y < 0] = 0
    old = (ou.objective(x, y, None, adv, None, 1.0, 0)[1] + 0.3 * rng.normal(size=n)).astype(np.float32)
    whole, rows = matrix(n, V, "float32", 0, 0)
    rows.copy_(torch.from_numpy(x))
    lp = run(sb, rows, y, old, adv, mask, 1.0, 0.2, 1.0, rows)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    out = torch.zeros(2, dtype=torch.float64, device="cuda")
    sb.spiral_policy_objective(dev(lp), dev(old), dev(adv), dev(mask), n, 0.2, out)
    J, _, _ = ou.objective(x, y, old, adv, mask, 1.0, float(np.float32(0.2)))
    assert abs(out[0].item() - J) <= 1e-5 * np.abs(adv).sum()          # 120 log-probabilities, each off by less than 3e-6


def test_rows_beyond_32_bit_offsets(sb):
    """A gradient of more than 2^32 bytes, and 2^31 elements: rows at both ends."""
    import torch
    n, V = 14200, 151936
    g = torch.Generator(device="cuda"); g.manual_seed(1)
    rows = torch.empty((n, V), dtype=torch.bfloat16, device="cuda")
    some = [0, 1, 7066, 14133, 14134, n - 1]                           # 14134 rows reach 2^31 elements
    y = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    for i in some:
        rows[i] = torch.randn(V, device="cuda", generator=g) * 2
        y[i] = (i * 7919) % V
    grad = torch.full((n, V), 1.0, dtype=torch.bfloat16, device="cuda")
    adv = torch.ones(n, device="cuda")
    logp = torch.empty(n, device="cuda")
    ws = torch.empty(sb.spiral_policy_gradient_workspace_bytes(n, V), dtype=torch.uint8, device="cuda")
    sb.spiral_policy_gradient(rows, y, None, adv, None, 1.0, 0.0, 1.0, logp, grad, ws)
    torch.cuda.synchronize()
    x = rows[some].float().cpu().numpy()
    check(x, y[some].cpu().numpy(), None, np.ones(len(some), np.float32), None, 1.0, 0.0, 1.0, logp[some].cpu().numpy(), grad[some].float().cpu().numpy(), "bfloat16")
    assert grad[2].float().abs().max().item() == 0 and grad[n - 2].float().abs().max().item() == 0


@pytest.mark.parametrize("n", [3, 700])
def test_captured_gradient_replays(sb, n):
    import torch
    rng = np.random.default_rng(10)
    V = 9001
    x, y, adv, mask = make(rng, n, V)
    whole, rows = matrix(n, V, "bfloat16", 0, 0)
    _, grad = matrix(n, V, "bfloat16", 0, 0)
    rows.copy_(torch.from_numpy(x))
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
        rows.copy_(torch.from_numpy(np.roll(x, r, axis=1)))
        at.copy_(dev(np.roll(adv, r)))
        grad.fill_(9.0)
        gph.replay()
        torch.cuda.synchronize()
        got, lp = grad.clone(), logp.clone()
        again = torch.empty((n, V), dtype=torch.bfloat16, device="cuda")
        call(again)
        torch.cuda.synchronize()
        assert torch.equal(got, again) and torch.equal(lp, logp)


def test_more_rows_than_a_launch_takes(sb):
    """2^20 rows of three logits, and five more."""
    import torch
    n, V = (1 << 20) + 5, 3
    g = torch.Generator().manual_seed(3)
    x = torch.randn((n, V), generator=g)
    y = torch.randint(0, V, (n,), generator=g, dtype=torch.int32)
    adv = torch.randn(n, generator=g)
    mask = (torch.rand(n, generator=g) < 0.7).int()
    logp, grad = torch.empty(n, device="cuda"), torch.full((n, V), 9.0, device="cuda")
    ws = torch.empty(sb.spiral_policy_gradient_workspace_bytes(n, V), dtype=torch.uint8, device="cuda")
    sb.spiral_policy_gradient(x.cuda(), y.cuda(), None, adv.cuda(), mask.cuda(), 1.0, 0.0, 1.0, logp, grad, ws)
    ls = torch.log_softmax(x.double(), -1)
    want = -(adv * mask).double()[:, None] * (torch.nn.functional.one_hot(y.long(), V) - ls.exp())
    assert (logp.cpu().double() - ls.gather(1, y.long()[:, None])[:, 0] * mask).abs().max().item() <= EPS * (8 * 6 + 2 * 12 + 64)
    assert (grad.cpu().double() - want).abs().max().item() <= 6 * 3 * EPS * (8 * 6 + 2 * 12 + 64)


def test_no_advantage_no_gradient_whatever_the_ratio(sb):
    import torch
    n, V = 4, 50
    rng = np.random.default_rng(11)
    x = rng.normal(size=(n, V)).astype(np.float32)
    y = np.arange(n, dtype=np.int32)
    old = np.array([-1000.0, -np.inf, -3.0, 0.0], np.float32)             # ratios without end, and ordinary ones
    whole, rows = matrix(n, V, "float32", 0, 0)
    rows.copy_(torch.from_numpy(x))
    _, grad = matrix(n, V, "float32", 0, 0)
    run(sb, rows, y, old, np.zeros(n, np.float32), None, 1.0, 0.2, 1.0, grad)
    assert (grad == 0).all()
    run(sb, rows, y, old, np.ones(n, np.float32), None, 1.0, 0.2, 1.0, grad)
    assert (grad[:2] == 0).all() and (grad[2:] != 0).any()                # clipped from above
