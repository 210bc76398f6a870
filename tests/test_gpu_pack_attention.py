"""spiral_attention_forward and _backward against the float64 oracle.

Bounds.  A score is off by E = 2^-24 (2 hd A + 8 max|s| + len + 64), A the largest scale sum |q||k| of the row: products summed in 32 bits, the exponent's
argument and the sum of the row; the softmax's weights relatively by as much.  Weights are rounded to the operands' type (`half` a step), and in fp16 are
off by 2^-25 at least: an output by (half + 2 E) sum p|v| + 2^-25 sum |v|, and rounded once itself.  In the gradients w = p (|dout||v| + |dout||out|) bounds both
|t| and what the rounding of `out` does to D, so dq and dk are off by (2 half + 6 E) of the same sum over w, dv by (half + 4 E) of its own, and are rounded once."""
import numpy as np
import pytest

from oracle import block as ob

pytestmark = pytest.mark.gpu
HALF = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
FLOOR = {"bfloat16": 2.0 ** -133, "float16": 2.0 ** -25}


@pytest.fixture(scope="module")
def sb():
    import torch
    assert torch.cuda.is_available()
    from paper_2506_24119_amd import binding
    binding.load_library()
    return binding


def heads(n, counts, hd, dtype, fused, behind=3, pad=0):
    """[n, heads, hd] views for each count, in one row or apart, gaps and rows behind filled with 77."""
    import torch
    dt = getattr(torch, dtype)
    if fused:
        whole = torch.full((n + behind, sum(counts) * hd + pad), 77.0, dtype=dt, device="cuda")
        at = np.concatenate([[0], np.cumsum(counts)]) * hd
        return [whole], [whole[:n, a:a + c * hd].unflatten(1, (c, hd)) for a, c in zip(at, counts)]
    whole = [torch.full((n + behind, c * hd + pad), 77.0, dtype=dt, device="cuda") for c in counts]
    return whole, [w[:n, :c * hd].unflatten(1, (c, hd)) for w, c in zip(whole, counts)]


class Call:
    def __init__(self, sb, lens, hq, hkv, hd, dtype, fused=True, pad=0, seed=0, sharp=1.0, dscale=None):
        import torch
        self.sb, self.lens, self.dtype, self.scale = sb, lens, dtype, float(np.float32(1.0 / np.sqrt(hd)))
        n = self.n = sum(lens)
        rng = np.random.default_rng(seed)
        self.wholes, (self.q, self.k, self.v) = heads(n, [hq, hkv, hkv], hd, dtype, fused, pad=pad)
        w, (self.out, self.dout) = heads(n, [hq, hq], hd, dtype, False, pad=pad)
        self.gwholes, (self.dq, self.dk, self.dv) = heads(n, [hq, hkv, hkv], hd, dtype, fused, pad=pad)
        self.owhole = w[0]
        put = lambda t, x: t.copy_(torch.from_numpy(x.astype(np.float32)))  # noqa: E731
        put(self.q, rng.normal(size=self.q.shape) * sharp)
        put(self.k, rng.normal(size=self.k.shape))
        put(self.v, rng.normal(size=self.v.shape) + 0.3)
        put(self.dout, rng.normal(size=self.out.shape) * (dscale or 1.0))
        self.lse = torch.full((hq, n), 5.0, device="cuda")
        self.mem = torch.full((sb.spiral_attention_plan_bytes(lens, hq, hkv, hd),), 0xA5, dtype=torch.uint8, device="cuda")
        self.plan = sb.spiral_attention_plan_create(lens, hq, hkv, hd, self.mem)
        self.ws = torch.full((sb.spiral_attention_backward_workspace_bytes(self.plan),), 0xA5, dtype=torch.uint8, device="cuda")

    def forward(self):
        self.sb.spiral_attention_forward(self.plan, self.q, self.k, self.v, self.scale, self.out, self.lse)

    def backward(self):
        self.sb.spiral_attention_backward(self.plan, self.q, self.k, self.v, self.out, self.lse, self.dout, self.scale, self.dq, self.dk, self.dv, self.ws)

    def results(self):
        return [t.clone() for t in (self.out, self.lse, self.dq, self.dk, self.dv)]

    def host(self, *names):
        return [getattr(self, x).float().cpu().numpy() for x in names]

    def errors(self):
        """[heads, rows] bound E of every row's scores."""
        q, k = self.host("q", "k")
        G, hd = q.shape[1] // k.shape[1], q.shape[2]
        E, a = np.zeros((q.shape[1], self.n)), 0
        for m in self.lens:
            for h in range(q.shape[1] if m else 0):
                size = np.tril(np.nan_to_num(np.abs(q[a:a + m, h]) @ np.abs(k[a:a + m, h // G]).T, posinf=0) * self.scale)
                E[h, a:a + m] = 2.0 ** -24 * (2 * hd * size.max(1) + 8 * size.max(1) + m + 64)
            a += m
        return E

    def free(self):
        self.sb.spiral_attention_plan_free(self.plan)


def close(got, want, allowed, what):
    assert np.array_equal(np.isnan(got), np.isnan(want)), (what, np.argwhere(np.isnan(got) != np.isnan(want))[:4])
    fine = np.isfinite(want)
    bad = fine & ~(np.abs(got - np.where(fine, want, 0)) <= allowed)
    assert not bad.any(), (what, np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], np.broadcast_to(allowed, got.shape)[bad][:4])


def check_forward(c):
    half, floor = HALF[c.dtype], FLOOR[c.dtype]
    q, k, v, out, lse = c.host("q", "k", "v", "out", "lse")
    want, wlse, ps = ob.attention(q, k, v, c.lens, c.scale)
    E, G = c.errors(), q.shape[1] // k.shape[1]
    size = ob.attention(q, k, np.abs(v), c.lens, c.scale)[0]
    Er = E.T[:, :, None]
    many = max(c.lens)
    close(out, want, (half + 2 * Er) * size + half * np.abs(want) * (1 + half) + floor * (1 + many * np.nanmax(np.where(np.isfinite(v), np.abs(v), 0))), "out")
    close(lse, wlse, 2 * E + 2.0 ** -22 * np.abs(wlse), "lse")


def check_backward(c):
    half, floor = HALF[c.dtype], FLOOR[c.dtype]
    q, k, v, dout = c.host("q", "k", "v", "dout")
    g, size = ob.attention_grad(q, k, v, dout, c.lens, c.scale)
    E, G = c.errors(), q.shape[1] // k.shape[1]
    worst = np.zeros(c.n)                                     # of the rows of a sequence, for the sums over rows
    a = 0
    for m in c.lens:
        worst[a:a + m] = E[:, a:a + m].max() if m else 0
        a += m
    # 128 products of 32 bits with |dout||v| + |dout||out| are in w too
    E3 = worst[:, None, None] + q.shape[2] * 2.0 ** -23
    most = lambda t: np.abs(t[np.isfinite(t)]).max()  # noqa: E731
    many = max(c.lens)
    for name, want, s, f, extra in (("dq", g[0], size[0], 2 * half + 6 * E3, c.scale * most(k)), ("dk", g[1], size[1], 2 * half + 6 * E3, G * c.scale * most(q)),
                                    ("dv", g[2], size[2], half + 4 * E3, G * most(dout))):
        got, = c.host(name)
        close(got, want, f * np.where(np.isfinite(s), s, 0) + half * np.abs(np.where(np.isfinite(want), want, 0)) * (1 + half) + floor * (1 + many * extra), name)


def untouched(c):
    for w, parts in ((c.owhole, [c.out]), *([(c.gwholes[0], [c.dq, c.dk, c.dv])] if len(c.gwholes) == 1 else [(x, [y]) for x, y in zip(c.gwholes, (c.dq, c.dk, c.dv))])):
        h = w.float().cpu().numpy()
        cols = sum(p.shape[1] * p.shape[2] for p in parts)
        assert (h[c.n:] == 77.0).all() and (h[:, cols:] == 77.0).all()


# the last four: a group's heads shared out over workgroups of their own, evenly and not, beside many short sequences that are not
SHAPES = [([1], 1, 1, 32), ([5, 0, 1, 33], 4, 2, 32), ([64, 65, 63], 2, 1, 64), ([130, 1, 31, 32], 6, 2, 128), ([257, 40], 7, 1, 128), ([0, 200, 0], 3, 3, 64),
          ([129, 127, 128], 8, 2, 64), ([96], 16, 1, 128), ([300, 17], 5, 5, 128), ([2] * 40, 4, 4, 32), ([31, 321], 9, 3, 32), ([70, 191], 12, 4, 128), ([500], 7, 1, 64), ([390, 3, 200], 6, 2, 128),
          ([129] * 12, 16, 2, 32), ([700, 1, 650, 0, 33], 5, 1, 32), ([70, 35], 64, 1, 32), ([150], 40, 1, 64), ([33, 64, 1], 12, 12, 128)]


@pytest.mark.parametrize("lens,hq,hkv,hd", SHAPES)
@pytest.mark.parametrize("dtype,fused,pad", [("bfloat16", True, 0), ("float16", False, 8), ("bfloat16", False, 24), ("float16", True, 40)])
def test_against_the_oracle(sb, lens, hq, hkv, hd, dtype, fused, pad):
    import torch
    c = Call(sb, lens, hq, hkv, hd, dtype, fused, pad, seed=len(lens) + hd, sharp=1.5)
    c.forward()
    torch.cuda.synchronize()
    check_forward(c)
    c.backward()
    torch.cuda.synchronize()
    check_backward(c)
    untouched(c)
    first = c.results()
    for t in (c.out, c.lse, c.dq, c.dk, c.dv):
        t.fill_(3.0)
    c.forward()
    c.backward()
    assert all(torch.equal(x, y) for x, y in zip(first, c.results()))         # bit for bit
    c.free()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_sharp_and_large_scores(sb, dtype):
    """Rows whose weight is on a token or two, scores of some hundreds, a maximum that rises along the row."""
    import torch
    c = Call(sb, [200, 77], 4, 2, 64, dtype, seed=5, sharp=20.0)
    up = torch.linspace(0.2, 3.0, 200, device="cuda")[:, None, None]
    c.k[:200] = (c.k[:200].float() * up).to(c.k.dtype)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    check_forward(c)
    check_backward(c)
    c.free()


@pytest.mark.parametrize("name,row,value", [("v", 70, np.nan), ("v", 12, np.inf), ("k", 70, np.nan), ("k", 150, np.inf), ("q", 33, np.nan), ("dout", 65, np.nan), ("q", 0, np.nan), ("v", 159, np.nan)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_what_a_row_does_not_see_does_not_reach_it(sb, name, row, value, dtype):
    """An undefined or infinite element in one sequence: exactly what depends on it is undefined."""
    import torch
    c = Call(sb, [40, 120, 35], 4, 2, 32, dtype, seed=9)
    getattr(c, name)[row, 1, 3] = value
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    check_forward(c)
    if not (name == "v" and value == np.inf):                # inf - inf somewhere along the row: which element is undefined is left open
        check_backward(c)
    else:
        q, k, v, dout = c.host("q", "k", "v", "dout")
        g, _ = ob.attention_grad(q, k, v, dout, c.lens, c.scale)
        for t, w in zip(c.host("dq", "dk", "dv"), g):
            assert np.isfinite(t[40:]).all() and np.isfinite(w[40:]).all()
    c.free()


@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 64), (7, 1, 128), (2, 2, 32)])
def test_infinite_gradients_stay_where_they_belong(sb, hq, hkv, hd):
    """Every third row of a sequence up to row 80 with an infinite element in its output's gradient: dq of the other rows, dk and dv of the tokens behind, and
    the other sequences are what they are without."""
    import torch
    lens = [50, 100, 33]
    c = Call(sb, lens, hq, hkv, hd, "float16", seed=31)
    c.forward()
    c.backward()
    clean = c.results()
    rows = torch.arange(50, 131, 3, device="cuda")
    c.dout[rows, 0, 5] = float("inf")
    c.backward()
    got = c.results()
    keep = torch.ones(c.n, dtype=torch.bool, device="cuda")
    keep[rows] = False
    assert torch.equal(got[2][keep], clean[2][keep])
    behind = torch.ones(c.n, dtype=torch.bool, device="cuda")
    behind[50:rows[-1] + 1] = False
    # added pair by pair, a tile's weights are not rounded to half precision: each of up to 32 terms a head differs by 2^-11 of it, and none is an eighth of the largest sum
    for name, g, w in zip(("dk", "dv"), got[3:], clean[3:]):
        assert torch.isfinite(g[behind]).all(), name
        assert ((g[behind].float() - w[behind].float()).abs() <= 2.0 ** -9 * (w[behind].float().abs() + w.float().abs().max() * 2.0 ** -3)).all(), name
    assert not torch.isfinite(got[4][50, 0, 5]) and not torch.isfinite(got[2][50, 0]).all()
    c.free()


@pytest.mark.parametrize("hq,hkv,hd", [(4, 2, 64), (7, 1, 128), (2, 2, 32)])
def test_tokens_that_weigh_nothing(sb, hq, hkv, hd):
    """Keys with an element of -inf where queries are positive: scores of -inf, weights of 0, dk and dv of 0; dq alone meets 0 times infinity."""
    import torch
    c = Call(sb, [50, 70, 33], hq, hkv, hd, "bfloat16", seed=37)
    c.q[:, :, 3] = c.q[:, :, 3].abs() + 1
    tokens = torch.tensor([1, 40, 51, 118, 152], device="cuda")
    c.k[tokens, :, 3] = -float("inf")
    c.forward()
    c.backward()
    weightless = [c.dk[tokens], c.dv[tokens]]
    for t in (*weightless, c.out, c.lse, c.dk, c.dv):
        assert torch.isfinite(t).all()
    assert not any(t.any() for t in weightless)
    q, k, v = c.host("q", "k", "v")
    half = HALF["bfloat16"]
    want, size = (ob.attention(q, k, x, c.lens, c.scale)[0] for x in (v, np.abs(v)))
    c.k[tokens, :, 3] = 0.0
    E = c.errors().T[:, :, None]
    close(c.host("out")[0], want, (half + 2 * E) * size + half * np.abs(want) * (1 + half), "out")
    c.free()


def test_rows_do_not_depend_on_other_sequences(sb):
    import torch
    c = Call(sb, [100, 333, 7, 64], 8, 2, 128, "bfloat16", seed=11)
    c.forward()
    c.backward()
    first = c.results()
    for cut, lens in ((slice(100, 433), [333]), (slice(433, 504), [7, 64])):
        d = Call(sb, lens, 8, 2, 128, "bfloat16", fused=False)
        for x in ("q", "k", "v", "dout"):
            getattr(d, x).copy_(getattr(c, x)[cut])
        d.forward()
        d.backward()
        for name, got, want in zip(("out", "lse", "dq", "dk", "dv"), d.results(), first):
            want = want[:, cut] if name == "lse" else want[cut]
            if name in ("dk", "dv"):                          # four heads' sums in another order: 2^-20 of the largest, then one rounding to 8 bits
                assert ((got.float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 2.0 ** -20 * want.float().abs().max()).all()
                assert (got == want).float().mean() >= 0.98
            else:
                assert torch.equal(got, want)
        d.free()
    c.free()


def test_many_short_sequences(sb):
    """More than one upload of the plan's items, sequences of one to three positions: the first of each is its own value."""
    import torch
    lens = [1 + i % 3 for i in range(1700)]
    c = Call(sb, lens, 4, 2, 32, "bfloat16", seed=41)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    check_forward(c)
    check_backward(c)
    first = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)[:-1]])).cuda()
    assert torch.equal(c.out[first], c.v[first].repeat_interleave(2, dim=1))
    c.free()


@pytest.mark.parametrize("which", ["q", "v", "dout", "dk"])
def test_rows_far_apart(sb, which):
    """Rows 2^22 elements apart, so that a matrix spans more than 2^31 of them: the bits of the same call on rows back to back."""
    import torch
    n = 530
    c = Call(sb, [n - 17, 17], 4, 2, 64, "bfloat16", fused=False, seed=43)
    c.forward()
    c.backward()
    want = c.results()
    near = getattr(c, which)
    whole = torch.empty(n << 22, dtype=near.dtype, device="cuda")
    far = whole.view(n, 1 << 22)[:, :near.shape[1] * 64].unflatten(1, (near.shape[1], 64))
    far.copy_(near)
    setattr(c, which, far)
    if which == "dk":
        far.zero_()
    c.forward()
    c.backward()
    assert all(torch.equal(a, b) for a, b in zip(c.results(), want))
    c.free()


def test_gradients_are_those_of_differences(sb):
    """d sum(dout . out) along a direction, from the oracle's outputs, against the kernels' gradients."""
    import torch
    c = Call(sb, [37, 90], 4, 2, 64, "float16", seed=13)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    x = dict(zip("qkv", c.host("q", "k", "v")))
    dout, = c.host("dout")
    rng = np.random.default_rng(1)
    for name, g in zip("qkv", c.host("dq", "dk", "dv")):
        d = rng.normal(size=g.shape)
        f = [(dout * ob.attention(*[x[m].astype(np.float64) + (s * 1e-5 * d if m == name else 0) for m in "qkv"], c.lens, c.scale)[0]).sum() for s in (1, -1)]
        slope = (f[0] - f[1]) / 2e-5
        assert abs(slope - (g.astype(np.float64) * d).sum()) <= 8 * HALF["float16"] * np.sqrt((g.astype(np.float64) ** 2 * d ** 2).sum()) + 1e-6 * abs(slope)
    c.free()


def test_long_sequence_against_sums_in_64_bits(sb):
    """6,000 positions: kernels' rows at the ends and between against the definition, gradients as a whole."""
    import torch
    c = Call(sb, [6000, 3], 4, 2, 128, "bfloat16", seed=17, sharp=1.3, dscale=0.01)
    c.forward()
    c.backward()
    L = 6000
    mask = torch.ones((L, L), dtype=torch.bool, device="cuda").tril_()
    for h in range(4):
        q, k, v, d = (t[:L, i].double() for t, i in ((c.q, h), (c.k, h // 2), (c.v, h // 2), (c.dout, h)))
        s = (q @ k.T * c.scale).masked_fill_(~mask, -np.inf)
        p = torch.softmax(s, 1)
        out = p @ v
        assert ((c.out[:L, h] - out).abs() <= (2.0 ** -8 + 1e-3) * (p @ v.abs()) + 2.0 ** -8 * out.abs()).all()
        assert ((c.lse[h, :L] - torch.logsumexp(s, 1)).abs() <= 2e-3).all()
        t = p * (d @ v.T - (d * out).sum(1, keepdim=True))
        w = p * (d.abs() @ v.abs().T + (d.abs() * out.abs()).sum(1, keepdim=True))
        dq = c.scale * t @ k
        assert ((c.dq[:L, h] - dq).abs() <= (2.0 ** -7 + 6e-3) * c.scale * (w @ k.abs()) + 2.0 ** -8 * dq.abs()).all()
        if h % 2 == 0:
            dk, dv, wk, wv = 0, 0, 0, 0
        dk, dv = dk + c.scale * t.T.contiguous() @ q, dv + p.T.contiguous() @ d
        wk, wv = wk + c.scale * w.T.contiguous() @ q.abs(), wv + p.T.contiguous() @ d.abs()
    assert ((c.dk[:L, 1] - dk).abs() <= (2.0 ** -7 + 6e-3) * wk + 2.0 ** -8 * dk.abs()).all()
    assert ((c.dv[:L, 1] - dv).abs() <= (2.0 ** -8 + 4e-3) * wv + 2.0 ** -8 * dv.abs()).all()
    c.free()


@pytest.mark.parametrize("hd", [64, 128])
def test_streams_and_graphs(sb, hd):
    """Two calls at once on two streams with one plan, then captured and replayed in turn, give what each gives alone."""
    import torch
    lens = [50, 0, 200, 129]
    works = [Call(sb, lens, 8, 4, hd, "bfloat16", seed=21), Call(sb, lens, 8, 4, hd, "bfloat16", fused=False, seed=22)]
    sb.spiral_attention_plan_free(works[1].plan)
    works[1].plan = works[0].plan
    alone = []
    for w in works:
        w.forward()
        w.backward()
        torch.cuda.synchronize()
        alone.append(w.results())

    def clear():
        for w in works:
            for t in (w.out, w.lse, w.dq, w.dk, w.dv):
                t.zero_()
        torch.cuda.synchronize()

    same = lambda: all(torch.equal(a, b) for w, r in zip(works, alone) for a, b in zip(w.results(), r))  # noqa: E731
    streams = [torch.cuda.Stream() for _ in works]
    clear()
    for w, st in zip(works, streams):
        with torch.cuda.stream(st):
            w.forward()
            w.backward()
    torch.cuda.synchronize()
    assert same()
    graphs = []
    for w, st in zip(works, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            w.forward()
            w.backward()
        graphs.append(g)
    for _ in range(3):
        clear()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        assert same()
    works[0].free()


def test_refusals(sb):
    """All of them before anything is enqueued: the addresses are made up."""
    import torch
    lib, mem = sb.load_library(), torch.zeros(4096, dtype=torch.uint8, device="cuda")
    lens, hq, hkv, hd = [3, 5], 4, 2, 32
    plan = sb.spiral_attention_plan_create(lens, hq, hkv, hd, mem)
    P = 1 << 30

    def forward(**change):
        a = dict(q=P, qs=256, k=P + 256, ks=256, v=P + 384, vs=256, t=1, c=0.2, o=2 * P, os=128, l=3 * P)
        a.update(change)
        return lib.spiral_attention_forward(plan, a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["t"], a["c"], a["o"], a["os"], a["l"], None)

    def backward(**change):
        a = dict(q=P, qs=256, k=P + 256, ks=256, v=P + 384, vs=256, t=1, c=0.2, o=2 * P, os=128, l=3 * P, d=4 * P, ds=128, dq=5 * P, dqs=256, dk=5 * P + 256, dks=256, dv=5 * P + 384, dvs=256, ws=6 * P, bytes=1 << 20)
        a.update(change)
        return lib.spiral_attention_backward(plan, a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["o"], a["os"], a["l"], a["d"], a["ds"], a["t"], a["c"], a["dq"], a["dqs"], a["dk"], a["dks"], a["dv"], a["dvs"],
                                             a["ws"], a["bytes"], None)

    both = [(dict(t=0), "type"), (dict(t=3), "type"), (dict(c=0.0), "scale"), (dict(c=-1.0), "scale"), (dict(c=float("nan")), "scale"), (dict(c=float("inf")), "scale")]
    both += [(dict([(x, None)]), "null") for x in "qkvol"] + [(dict([(x, P + 8)]), "misaligned") for x in "qkvo"] + [(dict(l=3 * P + 2), "misaligned"), (dict(qs=120), "stride"), (dict(ks=56), "stride"), (dict(vs=260), "stride"),
                                                                                                                       (dict(os=1 << 23), "stride")]
    for change, text in both + [(dict(o=P), "overlaps"), (dict(o=P + 512 - 16, os=256), "overlaps"), (dict(l=P), "overlaps"), (dict(l=2 * P), "overlaps"), (dict(o=P + 128, os=264), "overlaps")]:
        assert forward(**change) == sb.SPIRAL_ERR_INVALID_ARG and text in sb.spiral_last_error(), (change, sb.spiral_last_error())
    both += [(dict([(x, None)]), "null") for x in ("d", "dq", "dk", "dv")] + [(dict(d=4 * P + 8), "misaligned"), (dict(dqs=120), "stride"), (dict(dks=60), "stride"), (dict(dvs=0), "stride"), (dict(ws=None), "workspace"),
                                                                              (dict(ws=6 * P + 16), "workspace"), (dict(bytes=127), "workspace")]
    for change, text in both + [(dict(dq=P), "overlaps"), (dict(dk=P + 256), "overlaps"), (dict(dv=5 * P + 240), "overlaps"), (dict(dq=4 * P, dqs=128), "overlaps"), (dict(ws=3 * P), "overlaps"), (dict(dk=2 * P), "overlaps"),
                                (dict(dk=5 * P + 256, dks=264), "overlaps")]:
        assert backward(**change) == sb.SPIRAL_ERR_INVALID_ARG and text in sb.spiral_last_error(), (change, sb.spiral_last_error())
    q, k = torch.zeros(8, 4, 32, dtype=torch.bfloat16), torch.zeros(8, 2, 32, dtype=torch.bfloat16)
    for bad in (dict(dev_k=q), dict(dev_v=k.half()), dict(dev_q=q[:7]), dict(dev_out=q.transpose(0, 1)), dict(dev_lse=torch.zeros(31)), dict(dev_q=torch.zeros(8, 4, 64, dtype=torch.bfloat16)[:, :, ::2])):
        a = dict(plan=plan, dev_q=q, dev_k=k, dev_v=k, scale=0.2, dev_out=q.clone(), dev_lse=torch.zeros(4, 8), stream=0)
        a.update(bad)
        with pytest.raises(ValueError):
            sb.spiral_attention_forward(**a)
    sb.spiral_attention_plan_free(plan)
    with pytest.raises(ValueError):
        sb.spiral_attention_forward(plan, q, k, k, 0.2, q.clone(), torch.zeros(4, 8))
