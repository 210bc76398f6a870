"""The operators that close one update of the policy, as cases that can be timed and checked: the draw that also says how
probable the drawn token was, the gradient of the clipped objective, and the optimiser's step on the weights that the decoder reads.

With `own` false every operator is computed in its plain form, elementary torch operations in 32 bits (64 for the draw, whose
tokens follow from sums that come close to a border).  With `own` true the same inputs go through the library's entry points.

Kinds:
  draw      one token a row from [batch, vocab] logits and one given uniform number a row, under the row's own temperature, top-k, top-p
            and min-p -> tokens and their log-probabilities under what they were drawn from
  gradient  log-probabilities of given tokens and the gradient of the clipped (or plain) policy objective in the logits
  adamw     one AdamW step, gradients clipped to a global norm, over the tensors of a decoder: 16-bit matrices with 32-bit
            masters and 32-bit gains, states in 32 or in 8 bits

Vocabularies, batches and widths are those of the repository's geometries and their odd neighbours.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BLOCK = 256                       # elements that share a scale of 8-bit states
E4M3_MAX, E4M3_MIN = 448.0, 2.0 ** -9
BETA1, BETA2, EPS = 0.9, 0.95, 1e-8


def listed():
    return [
        # an evaluation of a few games with a small vocabulary: the smallest call, all settings mixed
        {"name": "draw few rows", "kind": "draw", "batch": 5, "vocab": 2039, "dtype": "fp32", "pad": 0, "cuts": "mixed"},
        # the actor's step: 128 games, temperature 1, nothing cut
        {"name": "draw actor", "kind": "draw", "batch": 128, "vocab": 151936, "dtype": "fp32", "pad": 0, "cuts": "none"},
        # the evaluation setting (temperature 0.6, top-p 0.95) on the whole batch
        {"name": "draw evaluation", "kind": "draw", "batch": 128, "vocab": 151936, "dtype": "fp32", "pad": 0, "cuts": "top-p"},
        # requests of several users in one batch, each with its own cuts, on 16-bit logits with padded rows
        {"name": "draw mixed requests", "kind": "draw", "batch": 61, "vocab": 152064, "dtype": "bf16", "pad": 24, "cuts": "mixed"},
        # the last few tokens of a batch of small games, an odd vocabulary
        {"name": "gradient few rows", "kind": "gradient", "rows": 9, "vocab": 8209, "dtype": "fp32", "pad": 0, "clip": 0.2, "temperature": 1.0, "masked": 0.2},
        # the paper's objective without the ratio, logits in 32 bits, one game's turn
        {"name": "gradient one turn", "kind": "gradient", "rows": 333, "vocab": 151936, "dtype": "fp32", "pad": 0, "clip": -1.0, "temperature": 1.0, "masked": 0.0},
        # a micro-batch of games: 16-bit logits, prompt and observation tokens masked, the clipped ratio
        {"name": "gradient micro-batch", "kind": "gradient", "rows": 4096, "vocab": 151936, "dtype": "bf16", "pad": 0, "clip": 0.2, "temperature": 1.0, "masked": 0.25},
        # the smallest decoder of the tests: launches and latency
        {"name": "adamw small", "kind": "adamw", "d": 256, "q": 1024, "kv": 256, "ffn": 512, "layers": 2, "vocab": 2048, "bits": 32},
        # layers of the 4B shape, one GPU's share
        {"name": "adamw layers", "kind": "adamw", "d": 2560, "q": 4096, "kv": 1024, "ffn": 9728, "layers": 3, "vocab": 0, "bits": 32},
        # the same with states in 8 bits
        {"name": "adamw layers 8 bits", "kind": "adamw", "d": 2560, "q": 4096, "kv": 1024, "ffn": 9728, "layers": 3, "vocab": 0, "bits": 8},
        # many layers of odd widths with an embedding: tensors that end inside every tile
        {"name": "adamw odd 8 bits", "kind": "adamw", "d": 893, "q": 897, "kv": 131, "ffn": 2431, "layers": 11, "vocab": 10007, "bits": 8},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["draw", "gradient", "adamw"])
    if kind == "draw":
        return {"kind": "draw", "batch": _log_int(rng, 1, 128), "vocab": _log_int(rng, 500, 152064), "dtype": rng.choice(sorted(DTYPES)),
                "pad": rng.choice([0, 0, 1, 8, 37]), "cuts": rng.choice(["none", "top-p", "top-k", "min-p", "mixed"])}
    if kind == "gradient":
        vocab = _log_int(rng, 500, 152064)
        return {"kind": "gradient", "rows": _log_int(rng, 1, min(4096, 300_000_000 // vocab)), "vocab": vocab, "dtype": rng.choice(sorted(DTYPES)),
                "pad": rng.choice([0, 0, 1, 8, 37]), "clip": rng.choice([-1.0, 0.2, 0.2]), "temperature": rng.choice([1.0, 1.0, 0.7]),
                "masked": rng.choice([0.0, 0.3, 0.7])}
    d = _log_int(rng, 64, 2560)
    return {"kind": "adamw", "d": d, "q": _log_int(rng, 64, 4096), "kv": _log_int(rng, 32, 1024), "ffn": _log_int(rng, 100, 9728),
            "layers": rng.randint(1, 3), "vocab": rng.choice([0, _log_int(rng, 300, 20000)]), "bits": rng.choice([8, 32])}


# ------------------------------------------------------------------------------------------------ inputs
def _settings(case, rng):
    """Temperature, top-k, top-p and min-p of every row, as a batch of requests has them."""
    B, V = case["batch"], case["vocab"]
    T, k, p, mp = np.ones(B, np.float32), np.zeros(B, np.int32), np.ones(B, np.float32), np.zeros(B, np.float32)
    for i in range(B):
        cuts = rng.choice(["none", "top-p", "top-k", "min-p", "all", "greedy"]) if case["cuts"] == "mixed" else case["cuts"]
        if cuts == "greedy":
            T[i] = 0.0
        elif cuts != "none":
            T[i] = 0.6 if case["cuts"] == "top-p" else rng.choice([0.6, 0.8, 1.0, 1.3])
        if cuts in ("top-k", "all"):
            k[i] = rng.choice([1, 20, 50, 200, max(1, V // 3)])
        if cuts in ("top-p", "all"):
            p[i] = 0.95 if case["cuts"] == "top-p" else rng.choice([0.5, 0.8, 0.9, 0.95, 0.99])
        if cuts in ("min-p", "all"):
            mp[i] = rng.choice([0.02, 0.05, 0.1])
    return T, k, p, mp


def _rows(n, V, pad, dtype):
    return torch.empty((n, V + pad), dtype=dtype, device=DEV)[:, :V]


def _sections(case):
    """Elements of every 16-bit matrix and of every 32-bit gain."""
    d, q, kv, f = case["d"], case["q"], case["kv"], case["ffn"]
    matrices = [q * d, kv * d, kv * d, d * q, f * d, f * d, d * f] * case["layers"] + ([case["vocab"] * d] if case["vocab"] else [])
    return matrices, [d, d] * case["layers"] + [d]


def _padded(n):
    return -(-n // BLOCK) * BLOCK


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = random.Random(seed)
    if case["kind"] == "draw":
        B, V = case["batch"], case["vocab"]
        # rows from nearly flat to sharp, a few entries well above the rest, some entries that are masked out
        width = torch.empty((B, 1), device=DEV).uniform_(0.8, 3.0, generator=g)
        x = torch.randn((B, V), device=DEV, generator=g) * width
        lift = torch.randint(0, V, (B, 6), device=DEV, generator=g)
        x.scatter_add_(1, lift, torch.empty((B, 6), device=DEV).uniform_(0.0, 9.0, generator=g))
        out = torch.rand((B, V), device=DEV, generator=g) < 0.01
        logits = _rows(B, V, case["pad"], DTYPES[case["dtype"]])
        logits.copy_(x.masked_fill(out, -math.inf))
        T, k, p, mp = _settings(case, rng)
        s = {"kind": "draw", "logits": logits, "u": torch.rand(B, device=DEV, generator=g), "host": (T, k, p, mp),
             "dev": [torch.from_numpy(a).to(DEV) for a in (T, k, p, mp)],
             "tokens": torch.empty(B, dtype=torch.int32, device=DEV), "logp": torch.empty(B, device=DEV)}
        if own:
            from paper_2506_24119_amd import binding as sb
            s["ws"] = torch.empty(sb.spiral_sample_uniform_workspace_bytes(B, V), dtype=torch.uint8, device=DEV)
        return s
    if case["kind"] == "gradient":
        n, V = case["rows"], case["vocab"]
        targets = torch.randint(0, V, (n,), device=DEV, generator=g, dtype=torch.int32)
        logits = _rows(n, V, case["pad"], DTYPES[case["dtype"]])
        noise = torch.randn((n, V), device=DEV, generator=g).mul_(2.0)
        noise.scatter_add_(1, targets[:, None].long(), torch.empty((n, 1), device=DEV).uniform_(4.0, 14.0, generator=g))
        logits.copy_(noise)
        del noise
        # the policy that drew the tokens was a little different
        logp = torch.cat([torch.log_softmax(c.float() / case["temperature"], -1).gather(1, t[:, None].long())[:, 0]
                          for c, t in zip(logits.split(512), targets.split(512))])
        old = logp + 0.15 * torch.randn(n, device=DEV, generator=g)
        masked = torch.rand(n, device=DEV, generator=g) < case["masked"]
        dropped = torch.rand(n, device=DEV, generator=g) < 0.1 * (case["masked"] > 0)
        s = {"kind": "gradient", "logits": logits, "targets": targets.masked_fill(dropped, -1), "old": old if case["clip"] >= 0 else None,
             "adv": torch.randn(n, device=DEV, generator=g), "mask": (~masked).int(), "clip": case["clip"], "T": case["temperature"],
             "scale": 1.0 / n, "logp": torch.empty(n, device=DEV), "grad": _rows(n, V, 0, DTYPES[case["dtype"]])}
        if own:
            from paper_2506_24119_amd import binding as sb
            s["ws"] = torch.empty(sb.spiral_policy_gradient_workspace_bytes(n, V), dtype=torch.uint8, device=DEV)
        return s
    mats, gains = _sections(case)
    sizes = mats + gains
    starts = np.concatenate([[0], np.cumsum([_padded(n) for n in sizes])]).tolist()
    split, total = starts[len(mats)], starts[-1]
    real = torch.zeros(total, dtype=torch.bool, device=DEV)
    for a, n in zip(starts, sizes):
        real[a:a + n] = True

    def normal(scale):
        return torch.randn(total, device=DEV, generator=g).mul_(scale).masked_fill_(~real, 0.0)

    master = normal(0.02)
    grad = normal(1e-3)
    m = normal(3e-4)
    v = normal(1e-3).square_().mul_(torch.rand(total, device=DEV, generator=g).mul_(0.9).add_(0.1))
    s = {"kind": "adamw", "master": master, "param": master[:split].to(torch.bfloat16), "grad16": grad[:split].to(torch.bfloat16),
         "grad32": grad[split:].clone(), "bits": case["bits"], "norm": torch.zeros(1, device=DEV),
         "lr": 1e-3, "wd": 0.01, "step": rng.randint(1, 300), "max_norm": 1.0, "grad_scale": 0.5,
         # matrices decay, gains do not
         "decay": torch.tensor([1.0] * len(mats) + [0.0] * len(gains), device=DEV),
         "spans": torch.tensor([_padded(n) for n in sizes], device=DEV), "total": total}
    del grad
    if case["bits"] == 8:
        s["m"], s["m_scale"] = _to_8bit(m, False)
        s["v"], s["v_scale"] = _to_8bit(v.sqrt_(), True)
    else:
        s["m"], s["v"] = m, v
    if own:
        from paper_2506_24119_amd import binding as sb
        recs = []
        for i, (a, n) in enumerate(zip(starts, sizes)):
            is_mat = i < len(mats)
            scales = {}
            if case["bits"] == 8:
                b = slice(a // BLOCK, (a + _padded(n)) // BLOCK)
                scales = {"m_scale": s["m_scale"][b], "v_scale": s["v_scale"][b]}
            e = slice(a, a + n)
            recs.append(sb.spiral_adamw_tensor(s["param"][e] if is_mat else master[e], s["grad16"][e] if is_mat else s["grad32"][a - split:a - split + n],
                                               s["m"][e], s["v"][e], master=master[e] if is_mat else None, decay=is_mat, **scales))
        s["mem"] = torch.empty(sb.spiral_adamw_bytes(recs), dtype=torch.uint8, device=DEV)
        s["opt"] = sb.spiral_adamw_create(recs, s["mem"])
    return s


# ------------------------------------------------------------------------------------------------ the operators
def run(s):
    if s["kind"] == "draw":
        return _run_draw(s)
    if s["kind"] == "gradient":
        return _run_gradient(s)
    return _run_adamw(s)


def _run_draw(s):
    if own:
        from paper_2506_24119_amd import binding as sb
        T, k, p, mp = s["host"]
        sb.spiral_sample_uniform(s["logits"], T, k, p, mp, s["u"], s["ws"], s["tokens"], s["logp"])
        return {"tokens": s["tokens"], "logp": s["logp"]}
    T, k, p, mp = (a[:, None] for a in s["dev"])
    lg = s["logits"].double()
    lg = torch.where(lg == lg, lg, -math.inf)
    V = lg.shape[1]
    top = lg.amax(1, keepdim=True)
    greedy = T == 0
    x = torch.where(lg == top, 0.0, (lg - top) / torch.where(greedy, 1.0, T.double()))
    w = torch.where(greedy, (lg == top).double(), torch.exp(x))
    down, order = lg.sort(dim=1, descending=True)
    kth = torch.where((k > 0) & (k < V), down.gather(1, (k.clamp(1, V) - 1).long()), -math.inf)
    c = torch.where(down >= kth, w.gather(1, order), 0.0).cumsum(1)
    at = (c < p.double() * c[:, -1:]).sum(1, keepdim=True).clamp(max=V - 1)
    tau = torch.where(p < 1, down.gather(1, at), -math.inf)
    keep = (lg >= kth) & (lg >= tau) & (w >= mp.double())
    c = torch.where(keep, w, 0.0).cumsum(1)
    u = torch.where(greedy, 0.0, s["u"].double()[:, None])
    tok = (c <= u * c[:, -1:]).sum(1, keepdim=True).clamp(max=V - 1)
    logp = torch.where(greedy, 0.0, x.gather(1, tok) - torch.log(c[:, -1:]))
    none = top == -math.inf
    return {"tokens": torch.where(none, 0, tok)[:, 0].int(), "logp": torch.where(none, -math.inf, logp)[:, 0].float()}


def _run_gradient(s):
    if own:
        from paper_2506_24119_amd import binding as sb
        sb.spiral_policy_gradient(s["logits"], s["targets"], s["old"], s["adv"], s["mask"], s["T"], max(s["clip"], 0.0), s["scale"], s["logp"],
                                  s["grad"], s["ws"])
        return {"logp": s["logp"], "grad": s["grad"]}
    z = s["logits"].float() / s["T"]
    live = ((s["mask"] != 0) & (s["targets"] >= 0))[:, None]
    y = s["targets"].clamp(min=0).long()[:, None]
    e = torch.exp(z - z.amax(1, keepdim=True))
    total = e.sum(1, keepdim=True)
    logp = z.gather(1, y) - z.amax(1, keepdim=True) - torch.log(total)
    A = s["adv"][:, None]
    slope = A
    if s["old"] is not None:
        r = torch.exp(logp - s["old"][:, None])
        slope = torch.where(r * A <= r.clamp(1 - s["clip"], 1 + s["clip"]) * A, r * A, 0.0)
    slope = torch.where(live, slope * (s["scale"] / s["T"]), 0.0)
    grad = e.mul_(slope / total)
    grad.scatter_add_(1, y, -slope)
    return {"logp": torch.where(live, logp, 0.0)[:, 0], "grad": grad.to(s["logits"].dtype)}


def _to_8bit(x, positive):
    """Codes and the scales of their blocks; positive values never become 0."""
    blocks = x.view(-1, BLOCK)
    most = blocks.abs().amax(1, keepdim=True)
    inv = torch.where(most > 1e-30, E4M3_MAX / most, 0.0)
    code = (blocks * inv).to(torch.float8_e4m3fn)
    if positive:
        code = torch.where((blocks > 0) & (inv > 0) & (code.float() == 0), torch.full_like(blocks, E4M3_MIN), code.float()).to(torch.float8_e4m3fn)
    return code.view(-1), torch.where(most > 1e-30, most / E4M3_MAX, 0.0)[:, 0].contiguous()


def _run_adamw(s):
    if own:
        from paper_2506_24119_amd import binding as sb
        sb.spiral_adamw_step(s["opt"], s["lr"], BETA1, BETA2, EPS, s["wd"], s["step"], grad_scale=s["grad_scale"], max_norm=s["max_norm"], dev_norm=s["norm"])
    else:
        g = torch.cat([s["grad16"].float(), s["grad32"]]).mul_(s["grad_scale"])
        s["norm"].copy_(g.double().square().sum().sqrt())
        g.mul_(torch.clamp(s["max_norm"] / s["norm"], max=1.0))
        wide = s["bits"] == 32
        m = s["m"] if wide else (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = s["v"] if wide else (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1).square()
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g.square()
        decay = torch.repeat_interleave(s["decay"], s["spans"], output_size=s["total"])
        root = torch.sqrt(v / (1 - BETA2 ** s["step"])) + EPS
        s["master"].mul_(1 - s["lr"] * s["wd"] * decay).sub_(s["lr"] * (m / (1 - BETA1 ** s["step"])) / root)
        s["param"].copy_(s["master"][:s["param"].numel()])
        if wide:
            s["m"].copy_(m)
            s["v"].copy_(v)
        else:
            s["m"], s["m_scale"] = _to_8bit(m, False)
            s["v"], s["v_scale"] = _to_8bit(v.sqrt(), True)
    return {k: s[k] for k in ("param", "master", "m", "v", "m_scale", "v_scale", "norm") if k in s}


# ------------------------------------------------------------------------------------------------ what they cannot do without
def work(case):
    if case["kind"] == "draw":
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": case["batch"] * (case["vocab"] * size + 4 + 8), "flops": 4 * case["batch"] * case["vocab"]}
    if case["kind"] == "gradient":
        size = 4 if case["dtype"] == "fp32" else 2
        live = (1 - case["masked"]) * (0.9 if case["masked"] > 0 else 1.0)
        return {"bytes": case["rows"] * case["vocab"] * size * (1 + live) + 20 * case["rows"], "flops": 8 * case["rows"] * case["vocab"]}
    mats, gains = _sections(case)
    state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK        # both moments, read and written
    return {"bytes": sum(mats) * (2 + 8 + 2 + state) + sum(gains) * (4 + 8 + state), "flops": 20 * (sum(mats) + sum(gains))}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "draw":
        return _exact_draw(case, s)
    if case["kind"] == "gradient":
        return _exact_gradient(case, s)
    return _exact_adamw(s)


def _exact_draw(case, s):
    """Row by row on the host: the k-th largest by partition, the nucleus over groups of equal logits."""
    logits, us = s["logits"].float().cpu().numpy().astype(np.float64), s["u"].cpu().numpy().astype(np.float64)
    tokens, logps = np.zeros(len(us), np.int32), np.zeros(len(us))
    for i, row in enumerate(logits):
        T, k, p, mp = (float(a[i]) for a in s["host"])
        if T == 0:
            tokens[i] = int(np.argmax(row))
            continue
        floor = -np.inf
        if 0 < k < row.size:
            floor = np.partition(row, row.size - int(k))[row.size - int(k)]
        if p < 1:
            values, counts = np.unique(row[row >= floor], return_counts=True)
            mass = (counts * np.exp((values - values[-1]) / T))[::-1].cumsum()
            floor = values[::-1][int(np.argmax(mass >= p * mass[-1]))]
        weight = np.exp((row - row.max()) / T)
        kept = np.flatnonzero((row >= floor) & (weight >= mp))
        run_sum = weight[kept].cumsum()
        tokens[i] = kept[np.searchsorted(run_sum, us[i] * run_sum[-1], side="right")]
        logps[i] = (row[tokens[i]] - row.max()) / T - np.log(run_sum[-1])
    return {"tokens": tokens, "logp": logps}


def _exact_gradient(case, s):
    """d(-scale J)/d logits by the chain rule through log_softmax, a few rows at a time."""
    n, V = case["rows"], case["vocab"]
    grad, logps = torch.zeros((n, V), dtype=torch.float64, device=DEV), torch.zeros(n, dtype=torch.float64, device=DEV)
    for a in range(0, n, 256):
        rows = torch.arange(a, min(n, a + 256), device=DEV)
        rows = rows[(s["mask"][rows] > 0) & (s["targets"][rows] >= 0)]
        if not len(rows):
            continue
        ls = torch.log_softmax(s["logits"][rows].double() / s["T"], -1)
        y = s["targets"][rows].long()
        lp = ls[torch.arange(len(rows), device=DEV), y]
        A = s["adv"][rows].double()
        if s["old"] is None:
            d = A
        else:
            ratio = torch.exp(lp - s["old"][rows].double())
            inside = torch.where(A > 0, ratio <= 1 + s["clip"], ratio >= 1 - s["clip"])
            d = A * ratio * inside
        hot = torch.nn.functional.one_hot(y, V).to(torch.float64)
        grad[rows] = -s["scale"] / s["T"] * d[:, None] * (hot - ls.exp())
        logps[rows] = lp
    return {"logp": logps, "grad": grad}


def _round_e4m3(x):
    """The nearest value of 4 exponent and 3 mantissa bits, ties to the even one, |x| <= 448."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _exact_adamw(s):
    """From the recurrence of the method, 8-bit states decoded and encoded as they are defined."""
    b1, b2, eps, t = BETA1, BETA2, EPS, s["step"]
    g = torch.cat([s["grad16"].double(), s["grad32"].double()]) * s["grad_scale"]
    norm = torch.linalg.vector_norm(g)
    if norm > s["max_norm"]:
        g = g * (s["max_norm"] / norm)
    blocks = lambda a: a.view(-1, BLOCK)  # noqa: E731
    if s["bits"] == 8:
        m = (blocks(s["m"].double()) * s["m_scale"].double()[:, None]).view(-1)
        v = (blocks(s["v"].double()) * s["v_scale"].double()[:, None]).view(-1) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m = m + (1 - b1) * (g - m)
    v = v + (1 - b2) * (g * g - v)
    wd = torch.repeat_interleave(s["decay"].double(), s["spans"]) * s["wd"]
    p = s["master"].double()
    p = p - s["lr"] * wd * p - s["lr"] * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)) ** 0.5 + eps)
    out = {"param": p[:s["param"].numel()], "master": p, "norm": norm[None]}
    if s["bits"] == 32:
        return {**out, "m": m, "v": v}
    for name, x in (("m", m), ("v", v ** 0.5)):
        scale = blocks(x).abs().amax(1) / E4M3_MAX
        code = _round_e4m3(blocks(x) / scale.clamp(min=1e-300)[:, None])
        if name == "v":
            code = torch.where((blocks(x) > 0) & (code == 0), E4M3_MIN, code)
        out[name], out[name + "_scale"] = code.view(-1), scale
    return out
