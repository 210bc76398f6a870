"""The learner's operators between the matrix products of a decoder block, forward and backward, as cases that can be timed and checked.

With `own` false every operator is computed in its plain form, elementary torch operations in 32 bits (64 for the angles of positions).  With
`own` true the same inputs go through the library's entry points.

Kinds:
  attention  causal attention with grouped heads over packed games of different lengths -> outputs and the log of each row's sum;
             with "backward" also the gradients of queries, keys and values, as one training step takes them
  norm       addition to the residual stream and root-mean-square norm -> sum, normed rows (16 or 32 bits, or codes of 8 bits under a scale a row);
             "backward": gradient of the sum and of the gain
  rope       norm of every q and k head (or none) and rotation by the rows' positions; "backward": gradients of the heads and of the gains

Widths, heads and lengths are those of the repository's geometries and workloads and their odd neighbours.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6
E4M3_MAX = 448.0


def listed():
    return [
        # the last turn of three short games: latency
        {"name": "attention one turn", "kind": "attention", "games": 3, "shortest": 5, "longest": 41, "q_heads": 16, "kv_heads": 8, "hd": 128, "dtype": "bf16",
         "fused": True, "backward": False},
        # the smallest decoder of the tests, one training step
        {"name": "attention tiny training", "kind": "attention", "games": 4, "shortest": 1, "longest": 67, "q_heads": 4, "kv_heads": 2, "hd": 32, "dtype": "fp16",
         "fused": True, "backward": True},
        # a scoring pass over a batch of ragged histories
        {"name": "attention scoring", "kind": "attention", "games": 24, "shortest": 256, "longest": 1024, "q_heads": 32, "kv_heads": 8, "hd": 128, "dtype": "bf16",
         "fused": True, "backward": False},
        # a micro-batch of games of the long workload, one training step
        {"name": "attention micro-batch", "kind": "attention", "games": 16, "shortest": 1024, "longest": 4096, "q_heads": 32, "kv_heads": 8, "hd": 128, "dtype": "bf16",
         "fused": True, "backward": True},
        # one very long history, groups of seven
        {"name": "attention long history", "kind": "attention", "games": 1, "shortest": 16001, "longest": 16001, "q_heads": 28, "kv_heads": 4, "hd": 128, "dtype": "bf16",
         "fused": False, "backward": True},
        # no grouped heads, narrow ones, odd lengths, half precision under a loss scale
        {"name": "attention narrow heads", "kind": "attention", "games": 37, "shortest": 3, "longest": 999, "q_heads": 12, "kv_heads": 12, "hd": 64, "dtype": "fp16",
         "fused": False, "backward": True},
        # the rows of a few sequences' last tokens
        {"name": "norm few rows", "kind": "norm", "rows": 5, "d": 2560, "dtype": "bf16", "residual": True, "out": "same", "backward": False},
        # a packed micro-batch whose next product takes 8 bits
        {"name": "norm 8 bits", "kind": "norm", "rows": 15271, "d": 2560, "dtype": "bf16", "residual": True, "out": "e4m3", "backward": False},
        # backward through the norm of the widest geometry, joined with the residual branch's gradient
        {"name": "norm gradient", "kind": "norm", "rows": 16384, "d": 3584, "dtype": "bf16", "residual": True, "out": "same", "backward": True},
        # a turn of one game, 32 bits
        {"name": "rope one turn", "kind": "rope", "rows": 33, "q_heads": 16, "kv_heads": 8, "hd": 128, "dtype": "fp32", "norm": True, "far": 4096, "backward": False},
        # the heads of a micro-batch, out of the fused projection
        {"name": "rope micro-batch", "kind": "rope", "rows": 15271, "q_heads": 32, "kv_heads": 8, "hd": 128, "dtype": "bf16", "norm": True, "far": 4096, "backward": False},
        # their gradient
        {"name": "rope gradient", "kind": "rope", "rows": 16384, "q_heads": 32, "kv_heads": 8, "hd": 128, "dtype": "bf16", "norm": True, "far": 40000, "backward": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "norm", "rope"])
    if kind == "attention":
        kv = rng.choice([1, 2, 4, 8])
        longest = _log_int(rng, 1, 8192)
        case = {"kind": "attention", "games": _log_int(rng, 1, 64), "shortest": rng.randint(0, longest - 1) if longest > 1 else 1, "longest": longest,
                "q_heads": kv * rng.choice([1, 2, 3, 4, 5, 7, 8]), "kv_heads": kv, "hd": rng.choice([32, 64, 128, 128]), "dtype": rng.choice(["bf16", "bf16", "fp16"]),
                "fused": rng.random() < 0.5, "backward": rng.random() < 0.6}
        while case["games"] > 1 and (_pairs(case) * case["q_heads"] * case["hd"] > 2e11 or sum(_lengths(case)) > 40000):
            case["games"] //= 2
        return case
    if kind == "norm":
        d = _log_int(rng, 64, 8192)
        return {"kind": "norm", "rows": _log_int(rng, 1, min(16384, 50_000_000 // d)), "d": d, "dtype": rng.choice(sorted(DTYPES)), "residual": rng.random() < 0.7,
                "out": rng.choice(["same", "same", "e4m3"]), "backward": rng.random() < 0.5}
    kv = rng.choice([1, 2, 4, 8])
    return {"kind": "rope", "rows": _log_int(rng, 1, 16384), "q_heads": kv * rng.randint(1, 5), "kv_heads": kv, "hd": rng.choice([32, 64, 128]),
            "dtype": rng.choice(sorted(DTYPES)), "norm": rng.random() < 0.6, "far": _log_int(rng, 1, 1_000_000), "backward": rng.random() < 0.5}


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """The games' lengths, between the shortest and the longest, in no order."""
    rng = random.Random(case["games"] * 7919 + case["longest"])
    lens = [rng.randint(case["shortest"], case["longest"]) for _ in range(case["games"])]
    lens[rng.randrange(len(lens))] = case["longest"]
    return lens


def _pairs(case):
    return sum(n * (n + 1) // 2 for n in _lengths(case))


def _heads(rows, counts, hd, dtype, fused):
    """One [rows, heads, hd] tensor for each count, beside each other in a row or apart."""
    if not fused:
        return [torch.empty((rows, c, hd), dtype=dtype, device=DEV) for c in counts]
    whole = torch.empty((rows, sum(counts), hd), dtype=dtype, device=DEV)
    return list(whole.split(counts, dim=1))


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(shape, scale=1.0):
        return torch.randn(shape, device=DEV, generator=g).mul_(scale)

    if case["kind"] == "attention":
        lens, hq, hkv, hd = _lengths(case), case["q_heads"], case["kv_heads"], case["hd"]
        n = sum(lens)
        q, k, v = _heads(n, [hq, hkv, hkv], hd, dtype, case["fused"])
        # heads as a norm leaves them, some sharper than others, and a first token of every game that draws attention
        q.copy_(normal((n, hq, hd)) * torch.empty((1, hq, 1), device=DEV).uniform_(0.7, 1.6, generator=g))
        k.copy_(normal((n, hkv, hd)))
        v.copy_(normal((n, hkv, hd)))
        starts = [0]
        for m in lens:
            starts.append(starts[-1] + m)
        for a, m in zip(starts, lens):
            if m:
                k[a] += (2.0 * q[a:a + m, ::hq // hkv].float().mean(0)).to(dtype)
        s = {"kind": "attention", "q": q, "k": k, "v": v, "lens": lens, "starts": starts, "scale": 1.0 / math.sqrt(hd), "backward": case["backward"],
             "out": torch.empty((n, hq, hd), dtype=dtype, device=DEV), "lse": torch.empty((hq, n), device=DEV)}
        if case["backward"]:
            s["dout"] = normal((n, hq, hd), 0.1 if case["dtype"] == "fp16" else 1e-3).to(dtype)
            s["dq"], s["dk"], s["dv"] = _heads(n, [hq, hkv, hkv], hd, dtype, case["fused"])
        if own:
            from paper_2506_24119_amd import binding as sb
            s["mem"] = torch.empty(sb.spiral_attention_plan_bytes(lens, hq, hkv, hd), dtype=torch.uint8, device=DEV)
            s["plan"] = sb.spiral_attention_plan_create(lens, hq, hkv, hd, s["mem"])
            if case["backward"]:
                s["ws"] = torch.empty(sb.spiral_attention_backward_workspace_bytes(s["plan"]), dtype=torch.uint8, device=DEV)
        return s
    if case["kind"] == "norm":
        n, d = case["rows"], case["d"]
        # a residual stream: a few wide channels, rows of different sizes
        wide = 1.0 + 9.0 * (torch.rand(d, device=DEV, generator=g) < 0.01)
        size = torch.empty((n, 1), device=DEV).uniform_(0.3, 3.0, generator=g)
        s = {"kind": "norm", "gain": 1.0 + normal(d, 0.1), "backward": case["backward"], "dtype": dtype, "out_dtype": torch.float8_e4m3fn if case["out"] == "e4m3" else dtype}
        if not case["backward"]:
            s["x"] = normal((n, d), 0.5).to(dtype)
            s["residual"] = (normal((n, d)) * wide * size).to(dtype) if case["residual"] else None
            s["sum"] = torch.empty((n, d), dtype=dtype, device=DEV) if case["residual"] else None
            s["out"] = torch.empty((n, d), dtype=s["out_dtype"], device=DEV)
            s["scale"] = torch.empty(n, device=DEV) if case["out"] == "e4m3" else None
            s["rstd"] = torch.empty(n, device=DEV)
            return s
        s["sum"] = (normal((n, d)) * wide * size).to(dtype)
        s["rstd"] = torch.rsqrt(s["sum"].float().square().mean(1) + EPS)
        s["dout"] = normal((n, d), 1e-3 if case["dtype"] != "fp16" else 0.1).to(dtype)
        s["dsum"] = normal((n, d), 1e-3 if case["dtype"] != "fp16" else 0.1).to(dtype) if case["residual"] else None
        s["dx"], s["dgain"] = torch.empty((n, d), dtype=dtype, device=DEV), torch.empty(d, device=DEV)
        if own:
            from paper_2506_24119_amd import binding as sb
            s["ws"] = torch.empty(sb.spiral_add_rmsnorm_backward_workspace_bytes(n, d), dtype=torch.uint8, device=DEV)
        return s
    n, hq, hkv, hd = case["rows"], case["q_heads"], case["kv_heads"], case["hd"]
    q, k, _ = _heads(n, [hq, hkv, hkv], hd, dtype, True)                 # out of the fused projection
    q.copy_(normal((n, hq, hd), 1.5))
    k.copy_(normal((n, hkv, hd), 1.5))
    gains = [1.0 + normal(hd, 0.1) for _ in range(2)] if case["norm"] else [None, None]
    first = torch.randint(0, case["far"], (1,), device=DEV, generator=g)
    s = {"kind": "rope", "q": q, "k": k, "gains": gains, "theta": 1e6 if case["norm"] else 1e4, "backward": case["backward"],
         "positions": ((first + torch.arange(n, device=DEV)) % case["far"]).int()}
    if not case["backward"]:
        s["out"] = [torch.empty((n, h, hd), dtype=dtype, device=DEV) for h in (hq, hkv)]
        return s
    size = 1e-3 if case["dtype"] != "fp16" else 0.1
    s["dout"] = [normal((n, h, hd), size).to(dtype) for h in (hq, hkv)]
    s["dq"], s["dk"], _ = _heads(n, [hq, hkv, hkv], hd, dtype, True)
    s["dgains"] = [torch.empty(hd, device=DEV) for _ in range(2)] if case["norm"] else [None, None]
    if own:
        from paper_2506_24119_amd import binding as sb
        s["ws"] = torch.empty(sb.spiral_norm_rope_backward_workspace_bytes(n, hq, hkv, hd), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ the operators
def run(s):
    if s["kind"] == "attention":
        return _run_attention(s)
    if s["kind"] == "norm":
        return _run_norm(s)
    return _run_rope(s)


def _run_attention(s):
    names = ("out", "lse") + (("dq", "dk", "dv") if s["backward"] else ())
    if own:
        from paper_2506_24119_amd import binding as sb
        sb.spiral_attention_forward(s["plan"], s["q"], s["k"], s["v"], s["scale"], s["out"], s["lse"])
        if s["backward"]:
            sb.spiral_attention_backward(s["plan"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["scale"], s["dq"], s["dk"], s["dv"], s["ws"])
        return {k: s[k] for k in names}
    hq, hkv = s["q"].shape[1], s["k"].shape[1]
    G, hd, scale = hq // hkv, s["q"].shape[2], s["scale"]
    for a, n in zip(s["starts"], s["lens"]):
        if not n:
            continue
        hidden = torch.ones((n, n), dtype=torch.bool, device=DEV).triu_(1)
        step = max(1, 2 ** 29 // (G * n * n))
        for h in range(0, hkv, step):
            kv = slice(h, min(hkv, h + step))
            qs = slice(h * G, kv.stop * G)
            heads = kv.stop - h
            grouped = lambda t: t[a:a + n, qs].float().view(n, heads, G, hd).permute(1, 2, 0, 3).reshape(heads, G * n, hd)  # noqa: E731
            back = lambda t: t.view(heads, G, n, hd).permute(2, 0, 1, 3).reshape(n, heads * G, hd)  # noqa: E731
            q, k, v = grouped(s["q"]), s["k"][a:a + n, kv].float().transpose(0, 1).contiguous(), s["v"][a:a + n, kv].float().transpose(0, 1).contiguous()
            p = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(scale)
            p.view(heads, G, n, n).masked_fill_(hidden, -math.inf)
            top = p.amax(2, keepdim=True)
            p.sub_(top).exp_()
            total = p.sum(2, keepdim=True)
            p.div_(total)
            out = torch.bmm(p, v)
            s["out"][a:a + n, qs] = back(out).to(s["out"].dtype)
            s["lse"][qs, a:a + n] = (top + torch.log(total)).view(heads * G, n)
            if not s["backward"]:
                continue
            dout = grouped(s["dout"])
            s["dv"][a:a + n, kv] = torch.bmm(p.transpose(1, 2), dout).transpose(0, 1).to(s["dv"].dtype)
            ds = torch.bmm(dout, v.transpose(1, 2).contiguous())
            ds.sub_((dout * out).sum(2, keepdim=True)).mul_(p).mul_(scale)
            del p
            s["dq"][a:a + n, qs] = back(torch.bmm(ds, k)).to(s["dq"].dtype)
            s["dk"][a:a + n, kv] = torch.bmm(ds.transpose(1, 2), q).transpose(0, 1).to(s["dk"].dtype)
            del ds
    return {k: s[k] for k in names}


def _run_norm(s):
    if own:
        from paper_2506_24119_amd import binding as sb
        if s["backward"]:
            sb.spiral_add_rmsnorm_backward(s["dout"], s["sum"], s["gain"], s["rstd"], s["dsum"], s["dx"], s["dgain"], s["ws"])
            return {"dx": s["dx"], "dgain": s["dgain"]}
        sb.spiral_add_rmsnorm(s["x"], s["residual"], s["gain"], EPS, s["out"], s["scale"], s["sum"], s["rstd"])
        return {k: s[k] for k in ("sum", "out", "scale", "rstd") if s[k] is not None}
    if s["backward"]:
        unit = s["sum"].float() * s["rstd"][:, None]
        dout = s["dout"].float()
        a = dout * s["gain"]
        dx = (a - unit * (a * unit).mean(1, keepdim=True)) * s["rstd"][:, None]
        if s["dsum"] is not None:
            dx = dx + s["dsum"].float()
        return {"dx": dx.to(s["dtype"]), "dgain": (dout * unit).sum(0)}
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    rstd = torch.rsqrt(h.square().mean(1) + EPS)
    y = h * rstd[:, None] * s["gain"]
    out = {} if s["residual"] is None else {"sum": h.to(s["dtype"])}
    if s["scale"] is None:
        return {**out, "out": y.to(s["dtype"]), "rstd": rstd}
    most = y.abs().amax(1)
    code = (y * torch.where(most > 0, E4M3_MAX / most, 0.0)[:, None]).to(torch.float8_e4m3fn)
    return {**out, "out": code, "scale": most / E4M3_MAX, "rstd": rstd}


def _angles(s, hd):
    j = torch.arange(hd // 2, device=DEV, dtype=torch.float64)
    a = s["positions"].double()[:, None] * torch.pow(s["theta"], -2.0 * j / hd)
    return torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]


def _run_rope(s):
    if own:
        from paper_2506_24119_amd import binding as sb
        if s["backward"]:
            sb.spiral_norm_rope_backward(s["q"], s["k"], s["dout"][0], s["dout"][1], s["gains"][0], s["gains"][1], EPS, s["theta"], s["positions"],
                                         s["dq"], s["dk"], s["dgains"][0], s["dgains"][1], s["ws"])
            return [t for t in (s["dq"], s["dk"], *s["dgains"]) if t is not None]
        sb.spiral_norm_rope(s["q"], s["k"], s["gains"][0], s["gains"][1], EPS, s["theta"], s["positions"], s["out"][0], s["out"][1])
        return s["out"]
    half = s["q"].shape[2] // 2
    cos, sin = _angles(s, 2 * half)
    outs, dgains = [], []
    for i, (x, gain) in enumerate(zip((s["q"], s["k"]), s["gains"])):
        n = x.float()
        if gain is not None:
            rstd = torch.rsqrt(n.square().mean(2, keepdim=True) + EPS)
            n = n * rstd
        if not s["backward"]:
            if gain is not None:
                n = n * gain
            lo, hi = n[..., :half], n[..., half:]
            outs.append(torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], 2).to(x.dtype))
            continue
        lo, hi = s["dout"][i].float().split(half, 2)
        d = torch.cat([lo * cos + hi * sin, hi * cos - lo * sin], 2)
        if gain is not None:
            dgains.append((d * n).sum((0, 1)))
            d = d * gain
            d = (d - n * (d * n).mean(2, keepdim=True)) * rstd
        outs.append(d.to(x.dtype))
    return outs + dgains


# ------------------------------------------------------------------------------------------------ what they cannot do without
def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "attention":
        n, hd, hq, hkv = sum(_lengths(case)), case["hd"], case["q_heads"], case["kv_heads"]
        per_row = size * hd * (2 * hq + 2 * hkv) + 4 * hq                          # q, k, v, out and the row sums
        if case["backward"]:
            per_row += size * hd * (2 * hq + 2 * hkv)                              # the output's gradient, and those of q, k, v
        return {"bytes": n * per_row, "flops": _pairs(case) * hq * hd * (14 if case["backward"] else 4)}
    if case["kind"] == "norm":
        n, d = case["rows"], case["d"]
        if case["backward"]:
            return {"bytes": n * d * size * (4 if case["residual"] else 3) + 4 * n + 8 * d, "flops": 10 * n * d}
        out = 1 if case["out"] == "e4m3" else size
        return {"bytes": n * (d * (size * (3 if case["residual"] else 1) + out) + 4 + (4 if case["out"] == "e4m3" else 0)) + 4 * d, "flops": 6 * n * d}
    n = case["rows"] * (case["q_heads"] + case["kv_heads"]) * case["hd"]
    if case["backward"]:
        return {"bytes": n * size * (3 if case["norm"] else 2) + 4 * case["rows"], "flops": 14 * n}
    return {"bytes": n * size * 2 + 4 * case["rows"], "flops": 8 * n}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attention":
        return _exact_attention(s)
    if case["kind"] == "norm":
        return _exact_norm(case, s)
    return _exact_rope(s)


def _exact_attention(s):
    """A query head at a time; gradients by reverse differentiation of the definition."""
    hq, hkv = s["q"].shape[1], s["k"].shape[1]
    wide = lambda t: torch.zeros(t.shape, dtype=torch.float64, device=DEV)  # noqa: E731
    res = {"out": wide(s["out"]), "lse": wide(s["lse"])}
    if s["backward"]:
        res.update(dq=wide(s["q"]), dk=wide(s["k"]), dv=wide(s["v"]))
    for a, n in zip(s["starts"], s["lens"]):
        if not n:
            continue
        rows = slice(a, a + n)
        sees = torch.arange(n, device=DEV)[:, None] >= torch.arange(n, device=DEV)[None, :]
        for h in range(hq):
            j = h // (hq // hkv)
            q, k, v = (t[rows, i].double().contiguous().requires_grad_(s["backward"]) for t, i in ((s["q"], h), (s["k"], j), (s["v"], j)))
            logits = torch.where(sees, s["scale"] * (q @ k.T), -math.inf)
            lse = torch.logsumexp(logits, 1)
            out = torch.exp(logits - lse[:, None]) @ v
            res["out"][rows, h], res["lse"][h, rows] = out.detach(), lse.detach()
            if s["backward"]:
                dq, dk, dv = torch.autograd.grad(out, (q, k, v), s["dout"][rows, h].double())
                res["dq"][rows, h] = dq
                res["dk"][rows, j] += dk
                res["dv"][rows, j] += dv
            del logits, out, lse
    return res


def _round_e4m3(x):
    """The nearest value of 4 exponent and 3 mantissa bits, ties to the even one, |x| <= 448."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _exact_norm(case, s):
    if case["backward"]:
        # the given 1 / rms takes part as it is: what follows from the definition with it held
        h, r, g, dy = s["sum"].double(), s["rstd"].double()[:, None], s["gain"].double(), s["dout"].double()
        along = torch.einsum("rd,rd->r", dy * g, h)[:, None]
        dx = r * g * dy - h * along * r ** 3 / h.shape[1]
        if s["dsum"] is not None:
            dx = dx + s["dsum"].double()
        return {"dx": dx, "dgain": torch.einsum("rd,rd->d", dy, h * r)}
    h = s["x"].double()
    out = {}
    if s["residual"] is not None:
        h = h + s["residual"].double()
        out["sum"] = h
    rms = torch.sqrt(torch.linalg.vector_norm(h, dim=1) ** 2 / h.shape[1] + EPS)
    y = s["gain"].double() * (h / rms[:, None])
    if s["scale"] is None:
        return {**out, "out": y, "rstd": 1 / rms}
    scale = torch.linalg.vector_norm(y, ord=math.inf, dim=1) / E4M3_MAX
    return {**out, "out": _round_e4m3(y / scale.clamp(min=1e-300)[:, None]), "scale": scale, "rstd": 1 / rms}


def _exact_rope(s):
    """Pairs as complex numbers, turned by multiplication; gradients by reverse differentiation."""
    hd = s["q"].shape[2]
    turn = torch.exp(-2.0 * math.log(s["theta"]) / hd * torch.arange(hd // 2, device=DEV, dtype=torch.float64))
    unit = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["positions"].double()[:, None] * turn)[:, None]
    outs, dgains = [], []
    for i, (x, gain) in enumerate(zip((s["q"], s["k"]), s["gains"])):
        x = x.double().requires_grad_(s["backward"])
        n = x
        if gain is not None:
            gain = gain.double().requires_grad_(s["backward"])
            n = gain * x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
        z = torch.complex(n[..., :hd // 2].contiguous(), n[..., hd // 2:].contiguous()) * unit
        y = torch.cat([z.real, z.imag], -1)
        if not s["backward"]:
            outs.append(y)
            continue
        grads = torch.autograd.grad(y, [x] if gain is None else [x, gain], s["dout"][i].double())
        outs.append(grads[0])
        dgains += grads[1:]
    return outs + dgains
