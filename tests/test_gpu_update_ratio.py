"""Which log-probability is the old one of the objective's ratio: the draw's for rows without a cut at the objective's temperature, a scoring call's for all others.

Bounds: a log-probability of spiral_policy_gradient is off by R = eps (8 max|z| + 2 |logp| + V / 256 + 64), eps = 2^-24 (tests/test_gpu_policy_gradient.py), one of the draw by a rounding."""
import numpy as np
import pytest

from oracle import update as ou

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


@pytest.mark.parametrize("V,dtype", [(151936, "float32"), (2048, "float32"), (50257, "bfloat16")])
def test_ratios_of_an_unchanged_policy_are_one(V, dtype):
    import torch
    from paper_2506_24119_amd import binding as sb
    rng = np.random.default_rng(V)
    B, T, clip = 24, 0.8, 0.2
    rows = torch.from_numpy((rng.normal(size=(B, V)) * 2.5).astype(np.float32)).cuda().to(getattr(torch, dtype))
    k, p, mp = np.zeros(B, np.int32), np.ones(B, np.float32), np.zeros(B, np.float32)
    k[8:12], p[12:16], mp[16:20] = 40, 0.9, 0.05
    k[20:], p[20:] = 300, 0.95
    u = torch.from_numpy(rng.random(B).astype(np.float32)).cuda()
    ws = torch.empty(sb.spiral_sample_uniform_workspace_bytes(B, V), dtype=torch.uint8, device="cuda")
    tok, drawn = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, device="cuda")
    sb.spiral_sample_uniform(rows, T, k, p, mp, u, ws, tok, drawn)
    adv = torch.from_numpy(rng.normal(size=B).astype(np.float32)).cuda()
    gws = torch.empty(sb.spiral_policy_gradient_workspace_bytes(B, V), dtype=torch.uint8, device="cuda")
    old, plain = torch.empty(B, device="cuda"), torch.empty_like(rows)
    sb.spiral_policy_gradient(rows, tok, None, adv, None, T, clip, 1.0, old, plain, gws)
    logp, grad = torch.empty(B, device="cuda"), torch.empty_like(rows)
    sb.spiral_policy_gradient(rows, tok, old, adv, None, T, clip, 1.0, logp, grad, gws)
    J = torch.zeros(2, dtype=torch.float64, device="cuda")
    sb.spiral_policy_objective(logp, old, adv, None, B, clip, J)
    torch.cuda.synchronize()
    # old and new from the same call: ratios of exactly 1, nothing clipped, the plain gradient
    assert torch.equal(old, logp) and torch.equal(plain, grad)
    assert abs(J[0].item() - adv.double().sum().item()) <= 1e-12 * B
    x, t = rows.float().cpu().numpy(), tok.cpu().numpy()
    lp, d = old.double().cpu().numpy(), drawn.double().cpu().numpy()
    R = EPS * (8 * np.abs(x).max(axis=1) / T + 4 * np.abs(lp) + V / 256 + 64)
    assert (np.abs(d - lp)[:8] <= R[:8]).all()                             # without a cut the draw's is the same
    for i in range(8, B):                                                  # with one it is larger by the kept mass
        w, _ = ou.weights_of(x[i], T)
        _, of_kept, slack = ou.draw_row(x[i], float(u[i]), T, int(k[i]), float(p[i]), float(mp[i]))
        if slack < 1e-9:
            continue
        kept = np.exp(np.log(w[t[i]]) - np.log(w.sum()) - of_kept)         # of the whole mass
        assert kept < 0.999 and abs((d[i] - lp[i]) + np.log(kept)) <= R[i], (i, kept)
