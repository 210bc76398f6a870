"""spiral_add_rmsnorm and spiral_norm_rope, forward and backward, against the float64 oracle.

Bounds, in units of u = 2^-24: a sum of d squares adds d / 64 + 16 (partial sums of at most that many terms) and its square root halves that, so 1 / rms is off by at
most R = u (d / 128 + 16) and a normed value by R and four roundings more; results are rounded once to their type.  A gradient's row sum of products is off by
u (d / 64 + 16) of the sum of magnitudes.  Sums over rows are off by u (rows / 8 + 64) of the sum of magnitudes."""
import numpy as np
import pytest

from oracle import block as ob

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {"float32": U, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
LEAST = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}


@pytest.fixture(scope="module")
def sb():
    import torch
    assert torch.cuda.is_available()
    from paper_2506_24119_amd import binding
    binding.load_library()
    return binding


def matrix(n, d, dtype, pad=0, offset=0, values=None):
    """(the whole buffer, its rows): what lies around the rows is 77."""
    import torch
    t = torch.full((n * (d + pad) + offset + 8,), 77.0, device="cuda").to(getattr(torch, dtype))
    rows = t[offset:offset + n * (d + pad)].view(n, d + pad)[:, :d]
    if values is not None:
        rows.copy_(torch.from_numpy(np.asarray(values, dtype=np.float32)))
    return t, rows


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def around(whole, n, d, pad, offset):
    h = host(whole)
    inside = np.zeros(h.shape, bool)
    for i in range(n):
        inside[offset + i * (d + pad):offset + i * (d + pad) + d] = True
    return h[~inside]


def near(got, want, allowed, what):
    bad = ~(np.abs(got - want) <= allowed) & ~(np.isnan(got) & np.isnan(want)) & ~(got == want)
    assert not bad.any(), (what, np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], np.broadcast_to(allowed, got.shape)[bad][:4])


ROWS = [(1, 1, 0, 0), (3, 7, 1, 1), (5, 2560, 0, 0), (70, 893, 3, 1), (33, 4096, 8, 8), (2, 20011, 1, 0), (129, 256, 0, 4), (9, 8192, 0, 0), (4, 16384, 8, 0), (300, 64, 0, 0), (17, 3584, 5, 3),
        (2, 40000, 0, 0), (2100, 130, 1, 1), (2049, 2559, 3, 1), (2048, 9, 0, 0), (2050, 4090, 0, 0), (6, 8, 0, 1)]


@pytest.mark.parametrize("n,d,pad,offset", ROWS)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("residual,out8", [(True, False), (False, False), (True, True), (False, True)])
def test_add_rmsnorm(sb, n, d, pad, offset, dtype, residual, out8):
    import torch
    rng = np.random.default_rng(n + d)
    _, x = matrix(n, d, dtype, pad, offset, rng.normal(size=(n, d)))
    _, res = matrix(n, d, dtype, (pad * 3) % 7, offset, rng.normal(size=(n, d)) * 10 ** rng.uniform(-2, 2, (n, 1)))
    if not residual:
        res = None
    gain = torch.from_numpy((1 + 0.3 * rng.normal(size=d)).astype(np.float32)).cuda()
    sw, total = matrix(n, d, dtype, pad, offset)
    ow, out = matrix(n, d, "float8_e4m3fn" if out8 else dtype, pad, offset)
    edge = host(ow)[-1]
    scale = torch.full((n + 2,), 5.0, device="cuda")
    rstd = torch.full((n + 2,), 5.0, device="cuda")
    eps = 1e-5
    sb.spiral_add_rmsnorm(x, res, gain, eps, out, scale[1:-1] if out8 else None, total, rstd[1:-1])
    torch.cuda.synchronize()
    h, y, r = ob.add_rmsnorm(host(x), None if res is None else host(res), host(gain), eps)
    half, R = HALF[dtype], U * (d / 128 + 16)
    near(host(total), h, (half + 2 * U) * np.abs(h) * (1 + half) + LEAST[dtype], "sum")
    # an element whose parts nearly cancel carries their rounding
    parts = U * (np.abs(host(x)) + (0 if res is None else np.abs(host(res)))) * r[:, None] * np.abs(host(gain))
    near(host(rstd)[1:-1], r, (R + 4 * U) * r + U * r * np.abs(r), "rstd")
    if out8:
        s = host(scale)[1:-1]
        most = np.abs(y).max(axis=1)
        near(s, most / 448, (R + 8 * U) * most / 448, "scale")
        code = host(out)
        # within half a step of the value that it stands for, a step being 2^-3 of it or 2^-9 near zero
        near(code * s[:, None], y, (2.0 ** -4 * np.abs(y) + 2.0 ** -10 * s[:, None]) * (1 + 4 * R + 64 * U) + parts, "codes")
        assert host(scale)[0] == host(scale)[-1] == 5.0
    else:
        near(host(out), y, (half + R + 8 * U) * np.abs(y) * (1 + half) + parts + LEAST[dtype], "out")
    assert (around(ow, n, d, pad, offset) == edge).all() and (around(sw, n, d, pad, offset) == 77.0).all() and host(rstd)[0] == host(rstd)[-1] == 5.0
    # without the optional outputs, and with the sum in place, the same bits
    first = out.clone().view(torch.uint8), total.clone()
    out.view(torch.uint8).zero_()
    sb.spiral_add_rmsnorm(x, res, gain, eps, out, scale[1:-1] if out8 else None)
    assert torch.equal(out.view(torch.uint8), first[0])
    over = x if res is None or n % 2 else res
    sb.spiral_add_rmsnorm(x, res, gain, eps, out, scale[1:-1] if out8 else None, over)
    assert torch.equal(out.view(torch.uint8), first[0]) and torch.equal(over, first[1])


@pytest.mark.parametrize("out8", [False, True])
@pytest.mark.parametrize("d", [100, 4096, 20000])
def test_odd_rows_of_the_norm(sb, d, out8):
    """Rows of zeros, of one element, with an undefined or infinite element: each row is its own."""
    import torch
    x = np.ones((6, d), np.float32)
    x[0] = 0
    x[1] = 0
    x[1, d - 1] = 3e-20
    x[2, d // 2] = np.nan
    x[3, 1] = np.inf
    x[4] = 1e-12
    _, rows = matrix(6, d, "float32", values=x)
    gain = torch.ones(d, device="cuda")
    _, out = matrix(6, d, "float8_e4m3fn" if out8 else "float32")
    scale = torch.zeros(6, device="cuda")
    sb.spiral_add_rmsnorm(rows, None, gain, 1e-6, out, scale if out8 else None)
    got, s = host(out), host(scale)
    if out8:
        assert s[0] == 0 and (got[0] == 0).all() and np.isnan(s[2]) and np.isnan(got[2]).all() and np.isnan(s[3]) and np.isnan(got[3]).all()
        got = got * s[:, None]
        near(got[[1, 4, 5]], ob.add_rmsnorm(x[[1, 4, 5]], None, np.ones(d), 1e-6)[1], 2.0 ** -4 * np.abs(x[[1, 4, 5]]) * 1e3 + 1e-30, "codes")
        assert got[1, d - 1] > 2.7e-17
    else:
        want = ob.add_rmsnorm(x, None, np.ones(d), 1e-6)[1]
        near(got, want, 1e-6 * np.abs(np.nan_to_num(want)) + d * U * np.abs(np.nan_to_num(want)), "out")
    assert (host(out)[5] == host(out)[5, 0]).all()


@pytest.mark.parametrize("n,d,pad,offset", ROWS + [(1000, 130, 0, 0), (5000, 33, 1, 0)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("branch", [True, False])
def test_add_rmsnorm_backward(sb, n, d, pad, offset, dtype, branch):
    import torch
    rng = np.random.default_rng(n * 3 + d)
    _, dy = matrix(n, d, dtype, pad, offset, rng.normal(size=(n, d)) * 0.1)
    _, total = matrix(n, d, dtype, (pad * 5) % 11, offset, rng.normal(size=(n, d)) * 10 ** rng.uniform(-1, 1, (n, 1)))
    _, dsum = matrix(n, d, dtype, pad, offset, rng.normal(size=(n, d)) * 0.1)
    if not branch:
        dsum = None
    gain = torch.from_numpy((1 + 0.3 * rng.normal(size=d)).astype(np.float32)).cuda()
    rstd = torch.from_numpy((1 / np.sqrt((host(total) ** 2).mean(1) + 1e-5)).astype(np.float32)).cuda()
    dw, dx = matrix(n, d, dtype, pad, offset)
    dg = torch.full((d + 2,), 5.0, device="cuda")
    ws = torch.full((sb.spiral_add_rmsnorm_backward_workspace_bytes(n, d),), 0xA5, dtype=torch.uint8, device="cuda")
    sb.spiral_add_rmsnorm_backward(dy, total, gain, rstd, dsum, dx, dg[1:-1], ws)
    torch.cuda.synchronize()
    keep = dx.clone()
    want, wg = ob.add_rmsnorm_grad(host(dy), host(total), host(gain), host(rstd), None if dsum is None else host(dsum))
    u = np.abs(host(total)) * host(rstd)[:, None]
    a = np.abs(host(dy) * host(gain))
    size = host(rstd)[:, None] * (a + u * (a * u).mean(1, keepdims=True))
    half = HALF[dtype]
    near(host(dx), want, half * np.abs(want) * (1 + half) + U * (d / 64 + 32) * size + 2 * U * (0 if dsum is None else np.abs(host(dsum))) + LEAST[dtype], "dx")
    assert dg[0] == dg[-1] == 5.0
    near(host(dg)[1:-1], wg, U * (n / 8 + 64) * (np.abs(host(dy)) * u).sum(0) + 1e-37, "dgain")
    assert (around(dw, n, d, pad, offset) == 77.0).all()
    # again, without the gain's gradient, and in place: the same bits
    again = torch.empty(d, device="cuda")
    sb.spiral_add_rmsnorm_backward(dy, total, gain, rstd, dsum, dx, again, ws)
    assert torch.equal(keep, dx) and torch.equal(again, dg[1:-1])
    over = dy if dsum is None or n % 2 else dsum
    sb.spiral_add_rmsnorm_backward(dy, total, gain, rstd, dsum, over, None, None)
    assert torch.equal(over, keep)


HEADS = [(1, 1, 1, 32), (7, 4, 2, 64), (33, 16, 8, 128), (130, 7, 1, 128), (5, 3, 3, 32), (400, 2, 1, 64), (65, 32, 8, 128), (2000, 5, 1, 32)]


@pytest.mark.parametrize("n,hq,hkv,hd", HEADS)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("norm,pad,offset", [((True, True), 0, 0), ((False, False), 3, 1), ((True, False), 8, 8), ((False, True), 0, 0)])
def test_norm_rope(sb, n, hq, hkv, hd, dtype, norm, pad, offset):
    """Forward and backward, out of place and in place, the heads of one fused row."""
    import torch
    rng = np.random.default_rng(n + hq + hd)
    width = (hq + hkv) * hd

    def fused(values=None):
        whole, rows = matrix(n, width, dtype, pad, offset, values)
        return whole, [rows[:, :hq * hd].unflatten(1, (hq, hd)), rows[:, hq * hd:].unflatten(1, (hkv, hd))]

    _, x = fused(rng.normal(size=(n, width)) * 2)
    gains = [torch.from_numpy((1 + 0.3 * rng.normal(size=hd)).astype(np.float32)).cuda() if g else None for g in norm]
    pos = rng.integers(0, 40_000, n).astype(np.int32)
    pos[0] = 0
    if n > 4:
        pos[1], pos[2], pos[3] = 1_999_999, -5, 2 ** 31 - 1
    dpos = torch.from_numpy(pos).cuda()
    theta, eps = (1e6, 1e-6) if n % 2 else (1e4, 1e-5)
    ow, out = fused()
    sb.spiral_norm_rope(x[0], x[1], gains[0], gains[1], eps, theta, dpos, out[0], out[1])
    dw, dx = fused()
    _, dy = fused(rng.normal(size=(n, width)))
    ws = torch.full((sb.spiral_norm_rope_backward_workspace_bytes(n, hq, hkv, hd),), 0xA5, dtype=torch.uint8, device="cuda")
    dg = [None if g is None else torch.full((hd,), 5.0, device="cuda") for g in gains]
    sb.spiral_norm_rope_backward(x[0], x[1], dy[0], dy[1], gains[0], gains[1], eps, theta, dpos, dx[0], dx[1], dg[0], dg[1], ws)
    torch.cuda.synchronize()
    half = HALF[dtype]
    for i in range(2):
        g = None if gains[i] is None else host(gains[i])
        h = lambda t: host(t.contiguous()).reshape(t.shape)  # noqa: E731
        want = ob.norm_rope(h(x[i]), g, eps, theta, pos)
        lo, hi = np.split(np.abs(ob.norm_rope(h(x[i]), g, eps, theta, 0 * pos)), 2, axis=-1)
        size = np.concatenate([lo + hi, lo + hi], axis=-1)
        near(h(out[i]), want, half * np.abs(want) * (1 + half) + U * (hd / 32 + 32) * size + LEAST[dtype], f"out {i}")
        wdx, wdg = ob.norm_rope_grad(h(x[i]), h(dy[i]), g, eps, theta, pos)
        lo, hi = np.split(np.abs(h(dy[i])), 2, axis=-1)
        d = np.concatenate([lo + hi, lo + hi], axis=-1)
        if g is None:
            size = d
        else:
            r = 1 / np.sqrt((h(x[i]) ** 2).mean(-1, keepdims=True) + eps)
            u = np.abs(h(x[i])) * r
            size = r * (d * np.abs(g) + u * (d * np.abs(g) * u).mean(-1, keepdims=True))
            near(host(dg[i]), wdg, U * (n * (hq, hkv)[i] / 8 + 96) * (d * u).sum((0, 1)) + 1e-37, f"dgain {i}")
        near(h(dx[i]), wdx, half * np.abs(wdx) * (1 + half) + U * (hd / 16 + 48) * size + LEAST[dtype], f"dx {i}")
    assert (around(ow, n, width, pad, offset) == 77.0).all() and (around(dw, n, width, pad, offset) == 77.0).all()
    keep = [t.clone() for t in (*out, *dx, *[t for t in dg if t is not None])]
    sb.spiral_norm_rope_backward(x[0], x[1], dy[0], dy[1], gains[0], gains[1], eps, theta, dpos, dy[0], dy[1], dg[0], dg[1], ws)
    sb.spiral_norm_rope(x[0], x[1], gains[0], gains[1], eps, theta, dpos, x[0], x[1])
    assert all(torch.equal(a, b) for a, b in zip(keep, (*x, *dy, *[t for t in dg if t is not None])))


def test_rows_far_apart(sb):
    """Rows 2^26 elements apart, the last ones behind 2^31: the bits of the same calls on rows back to back."""
    import torch
    rng = np.random.default_rng(6)
    n, d = 36, 128
    _, x = matrix(n, d, "bfloat16", values=rng.normal(size=(n, d)))
    far = torch.empty(n << 26, dtype=torch.bfloat16, device="cuda").view(n, 1 << 26)[:, :d]
    far.copy_(x)
    gain = torch.from_numpy((1 + 0.3 * rng.normal(size=d)).astype(np.float32)).cuda()
    outs = []
    for t in (x, far):
        out, total, rstd, dx, dg = torch.empty_like(x), torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty_like(x), torch.empty(d, device="cuda")
        ws = torch.empty(sb.spiral_add_rmsnorm_backward_workspace_bytes(n, d), dtype=torch.uint8, device="cuda")
        sb.spiral_add_rmsnorm(t, t, gain, 1e-6, out, None, total, rstd)
        sb.spiral_add_rmsnorm_backward(t, total, gain, rstd, t, dx, dg, ws)
        heads = t.unflatten(1, (2, 64))
        oq, ok, pos = torch.empty((n, 1, 64), dtype=torch.bfloat16, device="cuda"), torch.empty((n, 1, 64), dtype=torch.bfloat16, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda")
        sb.spiral_norm_rope(heads[:, :1], heads[:, 1:], gain[:64], gain[64:], 1e-6, 1e4, pos, oq, ok)
        outs.append([out, total, rstd, dx, dg, oq, ok])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("dtype,n,d,residual", [("bfloat16", 3000, 2560, True), ("float16", 2100, 4097, False), ("float32", 2500, 2047, False), ("bfloat16", 700, 8200, True), ("float32", 600, 7001, False),
                                                ("bfloat16", 300, 16384, True), ("bfloat16", 250, 20001, True), ("float16", 2000000, 5, True)])
def test_codes_are_those_of_exact_products(sb, dtype, n, d, residual):
    """5 to 10 million codes, every one that of the 64-bit quotient (32 bits alone have two in three million on a border's other side), also where the sum is written over x."""
    import torch
    torch.manual_seed(12)
    dt = getattr(torch, dtype)
    some = lambda: (torch.empty((n, d), device="cuda").uniform_(-6, 6).exp2() * torch.randn((n, d), device="cuda").sign()).to(dt)  # noqa: E731
    x, res = some(), some() if residual else None
    gain = 1 + 0.3 * torch.randn(d, device="cuda")
    p = (x.double() + (res.double() if residual else 0)) * gain.double()         # at most 20 bits (one type's without residual) times 24: exact
    out, scale = torch.empty((n, d), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(n, device="cuda")
    sb.spiral_add_rmsnorm(x, res, gain, 1e-6, out, scale, x, None)
    v = p * (448.0 / p.abs().amax(1, keepdim=True))
    step = torch.exp2(torch.clamp(torch.frexp(v)[1] - 1, min=-6).double() - 3)
    assert torch.equal(out.double(), torch.round(v / step) * step)


@pytest.mark.parametrize("dtype,n,d,pad,offset", [("bfloat16", 12288, 2051, 5, 1), ("float32", 8192, 2048, 0, 0), ("float16", 8200, 5002, 3, 0)])
def test_more_than_the_caches_keep(sb, dtype, n, d, pad, offset):
    """Calls of 200 to 650 MB: of rows, what a call on each quarter of them gives (40 to 110 MB), bit for bit; of the gains, those calls' sums."""
    import torch
    torch.manual_seed(9)
    dt = getattr(torch, dtype)

    def rows(fill=None):
        whole = torch.full((n * (d + pad) + offset + 8,), 77.0, device="cuda").to(dt)
        t = whole[offset:offset + n * (d + pad)].view(n, d + pad)[:, :d]
        if fill is None:
            t.normal_()
        return whole, t

    (_, x), (_, res), (_, dy), (_, ds) = (rows() for _ in range(4))
    gain = 1 + 0.3 * torch.randn(d, device="cuda")
    hd, heads = 64, d // 64
    gq, gk = 1 + 0.3 * torch.randn(hd, device="cuda"), 1 + 0.3 * torch.randn(hd, device="cuda")
    pos = torch.randint(0, 40000, (n,), device="cuda", dtype=torch.int32)
    q, g = (torch.randn((n, heads, hd), device="cuda").to(dt) for _ in range(2))

    def call(a, b):
        outs = [rows(0) for _ in range(3)]                    # whole buffers of all rows, of which a call writes its own
        (_, out), (_, total), (_, dx) = outs
        out8 = torch.zeros((n, d), dtype=torch.float8_e4m3fn, device="cuda")
        scale, rstd, dg, dgq, dgk = (torch.zeros(m, device="cuda") for m in (n, n, d, hd, hd))
        oq, dq = torch.zeros_like(q), torch.zeros_like(q)
        m = b - a
        ws = torch.empty(sb.spiral_add_rmsnorm_backward_workspace_bytes(m, d), dtype=torch.uint8, device="cuda")
        sb.spiral_add_rmsnorm(x[a:b], res[a:b], gain, 1e-6, out[a:b], None, total[a:b], rstd[a:b])
        sb.spiral_add_rmsnorm(x[a:b], res[a:b], gain, 1e-6, out8[a:b], scale[a:b], None, None)
        sb.spiral_add_rmsnorm_backward(dy[a:b], total[a:b], gain, rstd[a:b], ds[a:b], dx[a:b], dg, ws)
        ws = torch.empty(sb.spiral_norm_rope_backward_workspace_bytes(m, heads - 1, 1, hd), dtype=torch.uint8, device="cuda")
        sides = lambda t: (t[a:b, :-1], t[a:b, -1:])  # noqa: E731
        sb.spiral_norm_rope(*sides(q), gq, gk, 1e-6, 1e4, pos[a:b], *sides(oq))
        sb.spiral_norm_rope_backward(*sides(q), *sides(g), gq, gk, 1e-6, 1e4, pos[a:b], *sides(dq), dgq, dgk, ws)
        return [o[0] for o in outs] + [out8.view(torch.uint8), scale, rstd, oq, dq], [dg, dgq, dgk]

    whole, sums = call(0, n)
    first = [t.clone() for t in whole]
    for t in whole[:3]:
        assert (t[:offset] == 77).all() and (t[-8:] == 77).all() and (not pad or (t[offset:-8].view(n, d + pad)[:, d:] == 77).all())
    parts = [torch.zeros_like(t, dtype=torch.float64) for t in sums]
    for i in range(4):
        a, b = n * i // 4, n * (i + 1) // 4
        piece, add = call(a, b)
        for j, (w, p) in enumerate(zip(first, piece)):
            if j < 3:
                w, p = (t[offset:-8].view(n, d + pad)[a:b, :d] for t in (w, p))
            else:
                w, p = w[a:b], p[a:b]
            assert torch.equal(w, p), j
        for t, y in zip(parts, add):
            t += y.double()
    # Sums of the gains: a term passes at most 128 additions of 32 bits, of its wave's rows and heads (6 to 30), waves, 16 parts and 32 groups of them, in either order.
    total = whole[1][offset:-8].view(n, d + pad)[:, :d].double()
    size = [(dy.double() * total / (total.square().mean(1, keepdim=True) + 1e-6).sqrt()).abs().sum(0)]
    y, xn = g.double().abs(), (q.double() / (q.double().square().mean(2, keepdim=True) + 1e-6).sqrt()).abs()
    y += y.roll(hd // 2, 2)                                   # no rotation makes more of a pair
    size += [(y * xn)[:, :-1].sum((0, 1)), (y * xn)[:, -1].sum(0)]
    for t, w, m in zip(parts, sums, size):
        assert ((t - w.double()).abs() <= 2 * 128 * U * m).all()


def test_gradients_of_rows_are_those_of_differences(sb):
    import torch
    rng = np.random.default_rng(3)
    n, d = 9, 96
    _, h = matrix(n, d, "float32", values=rng.normal(size=(n, d)))
    _, dy = matrix(n, d, "float32", values=rng.normal(size=(n, d)))
    _, dx = matrix(n, d, "float32")
    gain = torch.from_numpy((1 + 0.2 * rng.normal(size=d)).astype(np.float32)).cuda()
    _, _, r = ob.add_rmsnorm(host(h), None, host(gain), 1e-6)
    dg = torch.empty(d, device="cuda")
    ws = torch.empty(sb.spiral_add_rmsnorm_backward_workspace_bytes(n, d), dtype=torch.uint8, device="cuda")
    sb.spiral_add_rmsnorm_backward(dy, h, gain, torch.from_numpy(r.astype(np.float32)).cuda(), None, dx, dg, ws)
    t, tg = rng.normal(size=(n, d)), rng.normal(size=d)
    f = lambda s, sg: (host(dy) * ob.add_rmsnorm(host(h) + s * t, None, host(gain) + sg * tg, 1e-6)[1]).sum()  # noqa: E731
    assert abs((f(1e-5, 0) - f(-1e-5, 0)) / 2e-5 - (host(dx) * t).sum()) <= 1e-5 * np.abs(host(dx) * t).sum()
    assert abs((f(0, 1e-5) - f(0, -1e-5)) / 2e-5 - (host(dg) * tg).sum()) <= 1e-5 * np.abs(host(dg) * tg).sum()


def test_streams_and_graphs(sb):
    """Rows' operators on two streams at once and replayed from graphs: what each gives alone."""
    import torch
    rng = np.random.default_rng(4)

    class Work:
        def __init__(self, n, d, hq, hkv, hd):
            put = lambda *s: torch.from_numpy(rng.normal(size=s).astype(np.float32)).cuda().bfloat16()  # noqa: E731
            self.x, self.res, self.dy, self.ds = put(n, d), put(n, d), put(n, d), put(n, d)
            self.gain = torch.ones(d, device="cuda")
            self.sum, self.out, self.dx = (torch.zeros_like(self.x) for _ in range(3))
            self.out8 = torch.zeros((n, d), dtype=torch.float8_e4m3fn, device="cuda")
            self.scale, self.rstd, self.dg = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(d, device="cuda")
            self.ws = torch.zeros(sb.spiral_add_rmsnorm_backward_workspace_bytes(n, d), dtype=torch.uint8, device="cuda")
            self.q, self.k, self.dq, self.dk = put(n, hq, hd), put(n, hkv, hd), put(n, hq, hd), put(n, hkv, hd)
            self.oq, self.ok, self.gq, self.gk = (torch.zeros_like(t) for t in (self.q, self.k, self.q, self.k))
            self.g = [torch.ones(hd, device="cuda") for _ in range(2)]
            self.dgs = [torch.zeros(hd, device="cuda") for _ in range(2)]
            self.pos = torch.arange(n, device="cuda", dtype=torch.int32)
            self.ws2 = torch.zeros(sb.spiral_norm_rope_backward_workspace_bytes(n, hq, hkv, hd), dtype=torch.uint8, device="cuda")

        def run(self):
            sb.spiral_add_rmsnorm(self.x, self.res, self.gain, 1e-6, self.out, None, self.sum, self.rstd)
            sb.spiral_add_rmsnorm(self.x, self.res, self.gain, 1e-6, self.out8, self.scale)
            sb.spiral_add_rmsnorm_backward(self.dy, self.sum, self.gain, self.rstd, self.ds, self.dx, self.dg, self.ws)
            sb.spiral_norm_rope(self.q, self.k, *self.g, 1e-6, 1e6, self.pos, self.oq, self.ok)
            sb.spiral_norm_rope_backward(self.q, self.k, self.dq, self.dk, *self.g, 1e-6, 1e6, self.pos, self.gq, self.gk, *self.dgs, self.ws2)

        def outs(self):
            return [self.sum, self.out, self.out8.view(torch.uint8), self.scale, self.rstd, self.dx, self.dg, self.oq, self.ok, self.gq, self.gk, *self.dgs]

    works = [Work(700, 2560, 8, 2, 128), Work(129, 900, 4, 4, 64)]
    alone = []
    for w in works:
        w.run()
        torch.cuda.synchronize()
        alone.append([t.clone() for t in w.outs()])
    same = lambda: all(torch.equal(a, b) for w, r in zip(works, alone) for a, b in zip(w.outs(), r))  # noqa: E731

    def clear():
        for w in works:
            for t in w.outs():
                t.zero_()
        torch.cuda.synchronize()

    streams = [torch.cuda.Stream() for _ in works]
    clear()
    for w, st in zip(works, streams):
        with torch.cuda.stream(st):
            w.run()
    torch.cuda.synchronize()
    assert same()
    graphs = []
    for w, st in zip(works, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            w.run()
        graphs.append(g)
    for _ in range(3):
        clear()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        assert same()
