"""spiral_adamw_* against the float64 oracle.

Bounds in units of eps = 2^-24: the scaled gradient is off by 3, m by 6 of its two parts, v by 10, the update (a root, a quotient, three
products) by 24, the parameter by that and 2 of itself; 16-bit parameters are rounded once more.  8-bit states: the value that a code
stands for is within half a step of the unrounded one (a positive root never 0: within the least code), relative errors of 1e-5 aside."""
import numpy as np
import pytest

from oracle import update as ou

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module")
def sb():
    import torch
    assert torch.cuda.is_available()
    from paper_2506_24119_amd import binding
    binding.load_library()
    return binding


class Guarded:
    """n elements behind `offset` others, with canaries on both sides."""

    def __init__(self, n, dtype, offset):
        import torch
        self.whole = torch.full((offset + n + 9,), 3.0, dtype=torch.float32, device="cuda").to(getattr(torch, dtype))
        self.t = self.whole[offset:offset + n]
        self.edges = torch.cat([self.whole[:offset], self.whole[offset + n:]]).float().cpu().numpy()
        self.at = (offset, n)

    def intact(self):
        import torch
        o, n = self.at
        return np.array_equal(torch.cat([self.whole[:o], self.whole[o + n:]]).float().cpu().numpy(), self.edges)

    def numpy(self):
        return self.t.float().cpu().numpy().astype(np.float64)


class Tensor:
    def __init__(self, sb, rng, n, param="bfloat16", grad="bfloat16", master=True, bits=32, decay=True, offset=0, fresh=False, wide=3.0):
        import torch
        self.n, self.bits, self.decay = n, bits, decay
        put = lambda a, dtype: self._put(a, dtype, offset)  # noqa: E731
        x = rng.normal(size=n).astype(np.float32) * 0.05
        self.param = put(x, param)
        self.master = put(x, "float32") if master and param != "float32" else None
        self.grad = put(self.new_grad(rng, wide), grad)
        blocks = -(-n // ou.BLOCK)
        m = rng.normal(size=n) * 10.0 ** rng.uniform(-wide, 0, size=n) * 0.01
        r = np.abs(rng.normal(size=n)) * 10.0 ** rng.uniform(-wide, 0, size=n) * 0.02
        if fresh:
            m, r = m * 0, r * 0
        if bits == 32:
            self.m, self.v = put(m, "float32"), put(r * r, "float32")
            self.ms = self.vs = None
        else:
            self.m, self.v = Guarded(n, "float8_e4m3fn", offset), Guarded(n, "float8_e4m3fn", offset)
            self.ms, self.vs = Guarded(blocks, "float32", offset), Guarded(blocks, "float32", offset)
            for code, scale, x in ((self.m, self.ms, m), (self.v, self.vs, r)):
                s, of = ou.block_scale(x)
                scale.t.copy_(torch.from_numpy(s))
                code.t.copy_(torch.from_numpy(np.divide(x, of, out=np.zeros_like(x), where=of > 0)).float().cuda().to(torch.float8_e4m3fn))
        self.rec = sb.spiral_adamw_tensor(self.param.t, self.grad.t, self.m.t, self.v.t, master=self.master.t if self.master else None,
                                          m_scale=self.ms.t if self.ms else None, v_scale=self.vs.t if self.vs else None, decay=decay)

    @staticmethod
    def _put(a, dtype, offset):
        import torch
        g = Guarded(len(a), dtype, offset)
        g.t.copy_(torch.from_numpy(np.asarray(a, dtype=np.float32)))
        return g

    def new_grad(self, rng, wide=3.0):
        g = rng.normal(size=self.n) * 10.0 ** rng.uniform(-wide, 0, size=self.n)
        g[rng.random(self.n) < 0.1] = 0.0
        return g.astype(np.float32)

    def guards(self):
        return [g for g in (self.param, self.master, self.grad, self.m, self.v, self.ms, self.vs) if g is not None]

    def values(self):
        import torch
        p = (self.master or self.param).numpy()
        if self.bits == 32:
            return {"p": p, "g": self.grad.numpy(), "m": self.m.numpy(), "v": self.v.numpy(), "decay": int(self.decay)}
        dec = lambda c, s: ou.decode_state(c.t.view(torch.uint8).cpu().numpy(), s.numpy())  # noqa: E731
        return {"p": p, "g": self.grad.numpy(), "m": dec(self.m, self.ms), "v": dec(self.v, self.vs) ** 2, "decay": int(self.decay)}


def build(sb, tensors):
    import torch
    recs = [t.rec for t in tensors]
    mem = torch.full((sb.spiral_adamw_bytes(recs),), 0xA5, dtype=torch.uint8, device="cuda")
    return sb.spiral_adamw_create(recs, mem), mem


def check_step(sb, opt, tensors, step, grad_scale=1.0, max_norm=0.0, want_norm=True, **hyper):
    import torch
    h = {**HYPER, **hyper}
    before = [t.values() for t in tensors]
    want, norm = ou.adamw(before, step=step, grad_scale=grad_scale, max_norm=max_norm, **h)
    dn = torch.full((3,), 4.0, device="cuda") if want_norm else None
    sb.spiral_adamw_step(opt, h["lr"], h["beta1"], h["beta2"], h["eps"], h["weight_decay"], step, grad_scale=grad_scale, max_norm=max_norm,
                         dev_norm=dn[1:2] if want_norm else None)
    torch.cuda.synchronize()
    if want_norm:
        assert dn[0].item() == dn[2].item() == 4.0 and abs(dn[1].item() - norm) <= 2 * EPS * norm
    b1, b2 = h["beta1"], h["beta2"]
    for t, b, w in zip(tensors, before, want):
        assert all(g.intact() for g in t.guards())
        e_m = 6 * EPS * (np.abs(b1 * b["m"]) + np.abs((1 - b1) * w["g"])) + 1e-37
        e_v = 10 * EPS * w["v"] + 1e-37
        p = (t.master or t.param).numpy()
        lost = h["lr"] / (1 - b1 ** step) * e_m / (np.sqrt(w["v"] / (1 - b2 ** step)) + h["eps"])
        tol = 24 * EPS * np.abs(w["update"]) + lost + 4 * EPS * np.abs(b["p"]) + 1e-37
        # a root of v in 32 bits near the least number has its absolute error
        tol += np.where(w["v"] < 1e-30, np.abs(w["update"]) * 1e-3 + h["lr"] * np.abs(w["m"]) / h["eps"] * 1e-6, 0.0)
        name = str(t.param.t.dtype)
        half = {"torch.float32": 0.0, "torch.bfloat16": 2.0 ** -8, "torch.float16": 2.0 ** -11}[name]
        if t.master is not None:
            assert (np.abs(p - w["p"]) <= tol).all(), np.abs((p - w["p"]) / tol).max()
            assert torch.equal(t.param.t, t.master.t.to(t.param.t.dtype))          # one rounding, to nearest even
        else:
            is16 = name == "torch.float16"
            # half's largest value is 65504, its last step 32: from 65520 on the nearest is infinite (an element with m but no v moves by lr m / eps)
            past = is16 & (np.abs(w["p"]) >= 65520 - tol) & (p == np.copysign(np.inf, w["p"]))
            with np.errstate(invalid="ignore"):
                near = np.abs(p - w["p"]) <= tol + half * np.abs(w["p"]) + (2.0 ** -25 if is16 else 0.0)
            assert (near | past).all()
        if t.bits == 32:
            assert (np.abs(t.m.numpy() - w["m"]) <= e_m).all() and (np.abs(t.v.numpy() - w["v"]) <= e_v).all()
            continue
        got = t.values()
        for key, scale, x in (("m", t.ms, w["m"]), ("v", t.vs, np.sqrt(w["v"]))):
            s, of = ou.block_scale(x)
            assert (np.abs(scale.numpy() - s) <= 1e-5 * s).all()
            y = got[key] if key == "m" else np.sqrt(got[key])
            off = ou.encode_off_by(x, of) * (1 + 1e-5) + 1e-5 * np.abs(x)
            err = np.abs(y - x)
            if key == "v":
                least = ou.E4M3_LEAST * of
                raised = (x > 0) & (x < least)
                assert (y[(x > 1e-5 * least) & (of > 0)] > 0).all()
                off = np.where(raised, least * (1 + 1e-5), off)
            else:
                off = off + e_m
            assert (err <= off).all(), (key, np.abs(err / np.maximum(off, 1e-300)).max())


SIZES = [1, 7, 255, 256, 257, 2047, 2048, 2049, 5000, 100003]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [0, 1])
def test_sizes_types_and_alignments(sb, bits, offset):
    rng = np.random.default_rng(bits + offset)
    kinds = [("bfloat16", "bfloat16", True), ("float32", "float32", False), ("float16", "float16", True), ("bfloat16", "float32", False), ("float16", "bfloat16", False),
             ("float32", "bfloat16", False)]
    tensors = [Tensor(sb, rng, n, *kinds[i % len(kinds)], bits=bits, decay=i % 3 != 0, offset=offset) for i, n in enumerate(SIZES)]
    opt, mem = build(sb, tensors)
    for step in (1, 2, 37):
        check_step(sb, opt, tensors, step, grad_scale=0.5, max_norm=0.0 if step == 2 else 1.0, want_norm=step != 2)
    sb.spiral_adamw_free(opt)


def test_states_of_both_kinds_in_one_step_from_nothing(sb):
    rng = np.random.default_rng(3)
    tensors = [Tensor(sb, rng, n, bits=8 if i % 2 else 32, fresh=True, offset=i % 3) for i, n in enumerate([300, 300, 4096, 4097, 65536, 70001])]
    opt, mem = build(sb, tensors)
    for step in range(1, 5):
        check_step(sb, opt, tensors, step, max_norm=100.0)
        for t in tensors:
            t.grad.t.copy_(t._put(t.new_grad(rng), "bfloat16", 0).t)
    sb.spiral_adamw_free(opt)


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_at_the_ends(sb, bits):
    """No gradient at all, gradients that square past 32 bits or to nothing, a lone one among zeros."""
    rng = np.random.default_rng(4)
    for fill in ("zero", "huge", "least", "lone"):
        t = Tensor(sb, rng, 1000, "float32", "float32", bits=bits, fresh=True)
        g = np.zeros(1000, np.float32)
        if fill == "huge":
            g[:] = rng.normal(size=1000) * 1e25
        if fill == "least":
            g[:] = rng.normal(size=1000) * 1e-12
        if fill == "lone":
            g[777] = 5.0
        t.grad.t.copy_(t._put(g, "float32", 0).t)
        opt, mem = build(sb, [t])
        check_step(sb, opt, [t], 1, max_norm=1.0)                      # huge: the norm is that of 64 bits, and the clipped step an ordinary one
        sb.spiral_adamw_free(opt)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_norm_that_is_not_finite_changes_nothing(sb, bad, bits):
    import torch
    rng = np.random.default_rng(5)
    tensors = [Tensor(sb, rng, n, bits=bits) for n in (900, 5000)]
    tensors[1].grad.t[4321] = bad
    opt, mem = build(sb, tensors)
    before = [[g.whole.clone().view(torch.uint8) for g in t.guards()] for t in tensors]
    norm = torch.zeros(1, device="cuda")
    for kw in (dict(max_norm=1.0, dev_norm=norm), dict(dev_norm=norm), dict(max_norm=1.0)):
        sb.spiral_adamw_step(opt, 1e-2, 0.9, 0.95, 1e-8, 0.1, 3, **kw)
        torch.cuda.synchronize()
        assert not np.isfinite(norm.item())
        assert all(torch.equal(g.whole.view(torch.uint8), b) for t, bs in zip(tensors, before) for g, b in zip(t.guards(), bs))
    tensors[1].grad.t[4321] = 0.5
    check_step(sb, opt, tensors, 3, max_norm=1.0)
    sb.spiral_adamw_free(opt)


def test_exchanged_gradients_and_replays(sb):
    """Two captured steps on the same object, replayed in turn with new gradients: every replay equals the step called by itself."""
    import torch
    rng = np.random.default_rng(6)
    mk = lambda: [Tensor(sb, np.random.default_rng(7), n, bits=b) for n, b in ((3000, 32), (777, 8), (20000, 8))]  # noqa: E731
    one, two = mk(), mk()
    o1, m1 = build(sb, one)
    o2, m2 = build(sb, two)
    other = [torch.zeros_like(t.grad.t) for t in two]
    sb.spiral_adamw_set_grads(o2, other)
    args = (1e-2, 0.9, 0.95, 1e-8, 0.1)
    n1, n2 = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs = []
    for step in (5, 6):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            sb.spiral_adamw_step(o2, *args, step, max_norm=1.0, dev_norm=n2)
        graphs.append((step, g))
    for r in range(4):
        step, g = graphs[r % 2]
        for t, o in zip(one, other):
            t.grad.t.copy_(t._put(t.new_grad(rng), "bfloat16", 0).t)
            o.copy_(t.grad.t)
        sb.spiral_adamw_step(o1, *args, step, max_norm=1.0, dev_norm=n1)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(n1, n2)
        for a, b in zip(one, two):
            for x, y in ((a.param, b.param), (a.master, b.master), (a.m, b.m), (a.v, b.v)):
                assert torch.equal(x.t.view(torch.uint8), y.t.view(torch.uint8))
    sb.spiral_adamw_free(o1); sb.spiral_adamw_free(o2)


def test_many_tensors(sb):
    """More tensors than one upload carries, most of them a few elements long."""
    rng = np.random.default_rng(8)
    tensors = [Tensor(sb, rng, int(n), "float32", "float32", bits=32, offset=0) for n in rng.integers(1, 40, 1500)]
    opt, mem = build(sb, tensors)
    check_step(sb, opt, tensors, 2, max_norm=0.5)
    sb.spiral_adamw_free(opt)


@pytest.mark.parametrize("bits", [32, 8])
def test_long_chunks(sb, bits):
    """From 2^23 elements on a workgroup takes 4,096 of a tensor at a time: tensors that end in and behind every run of them, each kind of
    parameter and gradient."""
    rng = np.random.default_rng(9)
    kinds = [("bfloat16", "bfloat16", True), ("float32", "float32", False), ("bfloat16", "float32", False), ("float16", "bfloat16", False)]
    sizes = [2_200_001, 4095, 4096, 4097, 2_150_400, 5121, 8191, 2_100_003, 300, 2_050_050]
    tensors = [Tensor(sb, rng, n, *kinds[i % 4], bits=bits, decay=i % 2 == 0, offset=i % 3) for i, n in enumerate(sizes)]
    assert sum(t.n for t in tensors) > 1 << 23
    opt, mem = build(sb, tensors)
    for step in (1, 9):
        check_step(sb, opt, tensors, step, max_norm=1.0)
    sb.spiral_adamw_free(opt)


def test_refusals_of_a_made_optimiser(sb):
    """What only an existing object can refuse: settings of a step, gradients that would be overwritten.  Nothing is enqueued by any of them."""
    import torch
    rng = np.random.default_rng(10)
    tensors = [Tensor(sb, rng, n, bits=b) for n, b in ((1000, 32), (600, 8))]
    opt, mem = build(sb, tensors)
    before = [[g.whole.clone().view(torch.uint8) for g in t.guards()] for t in tensors]
    ok = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.0, step=1)
    for bad in (dict(lr=-1.0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(eps=1e-31), dict(eps=float("inf")), dict(weight_decay=-1.0),
                dict(step=0), dict(grad_scale=float("inf")), dict(max_norm=-1.0), dict(max_norm=float("nan"))):
        with pytest.raises(sb.SpiralError) as e:
            sb.spiral_adamw_step(opt, **{**ok, **bad})
        assert e.value.code == sb.SPIRAL_ERR_INVALID_ARG, bad
    g0, g1 = tensors[0].grad.t, tensors[1].grad.t
    p16 = tensors[0].param.whole
    for grads in ([g0, tensors[0].param.t], [tensors[1].param.t, g1], [p16[2:1002], g1], [tensors[0].master.whole.view(torch.bfloat16)[5:1005], g1],
                  [g0, mem.view(torch.bfloat16)[-700:-100]]):
        with pytest.raises(sb.SpiralError) as e:
            sb.spiral_adamw_set_grads(opt, grads)
        assert "overlaps" in str(e.value)
    sb.spiral_adamw_set_grads(opt, [g0[:1000], g0[:600]])                  # two tensors may share a gradient: it is only read
    sb.spiral_adamw_set_grads(opt, [g0, g1])
    torch.cuda.synchronize()
    assert all(torch.equal(g.whole.view(torch.uint8), b) for t, bs in zip(tensors, before) for g, b in zip(t.guards(), bs))
    check_step(sb, opt, tensors, 1, max_norm=1.0)
    sb.spiral_adamw_free(opt)


def test_a_norm_inside_the_tables_buffers_is_refused(sb):
    import torch
    rng = np.random.default_rng(11)
    tensors = [Tensor(sb, rng, n, bits=b) for n, b in ((1000, 32), (600, 8))]
    opt, mem = build(sb, tensors)
    before = [[g.whole.clone().view(torch.uint8) for g in t.guards()] for t in tensors]
    t0, t1 = tensors
    for buf in (t0.param.t, t0.master.t, t0.m.t, t0.v.t, t0.grad.t, t1.grad.t, mem):
        words = buf.view(torch.uint8)
        at = -words.data_ptr() % 4
        for o in (at, at + (len(words) - at - 4) // 4 * 4):
            with pytest.raises(sb.SpiralError) as e:
                sb.spiral_adamw_step(opt, 1e-3, 0.9, 0.95, 1e-8, 0.0, 1, dev_norm=words[o:o + 4].view(torch.float32))
            assert e.value.code == sb.SPIRAL_ERR_INVALID_ARG and "overlaps" in str(e.value)
    grads = [t0.grad.t.clone(), t1.grad.t]
    sb.spiral_adamw_set_grads(opt, grads)                                   # the table's gradients are those that it has now
    with pytest.raises(sb.SpiralError):
        sb.spiral_adamw_step(opt, 1e-3, 0.9, 0.95, 1e-8, 0.0, 1, dev_norm=grads[0].view(torch.float32)[7:8])
    sb.spiral_adamw_set_grads(opt, [t0.grad.t, t1.grad.t])
    torch.cuda.synchronize()
    assert all(torch.equal(g.whole.view(torch.uint8), b) for t, bs in zip(tensors, before) for g, b in zip(t.guards(), bs))
    check_step(sb, opt, tensors, 1, max_norm=1.0)
    sb.spiral_adamw_free(opt)
