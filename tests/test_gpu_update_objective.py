"""Values of the objective from the gradient's log-probabilities, where targets are dropped without the mask's knowledge and where there are no old ones."""
import numpy as np
import pytest

from oracle import scoring as osc
from oracle import update as ou

pytestmark = pytest.mark.gpu


def test_values_where_targets_are_dropped_and_without_old_ones():
    import torch
    from paper_2506_24119_amd import binding as sb
    rng = np.random.default_rng(15)
    n, V, clip = 200, 700, 0.2
    x = (rng.normal(size=(n, V)) * 2).astype(np.float32)
    y = rng.integers(0, V, n).astype(np.int32)
    adv = rng.normal(size=n).astype(np.float32)
    mask = (rng.random(n) < 0.8).astype(np.int32) * rng.integers(1, 5, n).astype(np.int32)
    y[::7] = -1                                                        # dropped, with either mask
    mask[[0, 7, 14]], adv[[0, 7, 14]] = 1, -2.0
    lp64 = ou.objective(x, y, None, adv, mask, 1.0, 0)[1]
    old = (lp64 + 0.3 * rng.normal(size=n)).astype(np.float32)
    old[[0, 7, 14]] = -9.0
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    rows, logp, grad = dev(x), torch.empty(n, device="cuda"), torch.empty(n, V, device="cuda")
    ws = torch.empty(sb.spiral_policy_gradient_workspace_bytes(n, V), dtype=torch.uint8, device="cuda")
    sb.spiral_policy_gradient(rows, dev(y), dev(old), dev(adv), dev(mask), 1.0, clip, 1.0, logp, grad, ws)
    out = torch.zeros(2, dtype=torch.float64, device="cuda")
    value = lambda o, m: (sb.spiral_policy_objective(logp, o, dev(adv), m, n, clip, out), out.cpu().numpy().copy())[1]  # noqa: E731
    eps = float(np.float32(clip))
    # 200 log-probabilities, each off by at most 2^-24 (8 max|z| + 2 |logp| + V / 256 + 64) < 1.2e-5, ratios of e^1.5 at most
    tol = 200 * 1.2e-5 * 5 * np.abs(adv).max()
    J = ou.objective(x, y, old, adv, mask, 1.0, eps)[0]
    assert abs(value(dev(old), dev(mask * (y >= 0)))[0] - J) <= tol
    # the mask alone: dropped rows come in with a logp of 0, e^9 A each for those of a negative advantage
    lp = logp.cpu().numpy()
    extra = (y < 0) & (mask != 0)
    more = osc.clipped_surrogate(lp[extra], old[extra], adv[extra], np.ones(extra.sum()), eps)
    assert more < -3 * 2 * np.exp(9.0) + 1000
    assert abs(value(dev(old), dev(mask))[0] - J - more) <= tol + 1e-9 * abs(more)
    # without old ones: the gradient's own in their place, and the sum beside
    plain = ou.objective(x, y, None, adv, mask, 1.0, 0)[0]
    assert abs(value(logp, dev(mask))[1] - plain) <= tol
    assert abs(value(logp, dev(mask * (y >= 0)))[1] - plain) <= tol


def test_an_undefined_log_probability_shows_in_the_plain_sum():
    import torch
    from paper_2506_24119_amd import binding as sb
    lp = torch.tensor([-1.0, float("nan"), -2.0], device="cuda")
    old, adv = torch.tensor([-1.0, -1.0, -2.0], device="cuda"), torch.ones(3, device="cuda")
    out = torch.zeros(2, dtype=torch.float64, device="cuda")
    sb.spiral_policy_objective(lp, old, adv, None, 3, 0.2, out)
    assert torch.isnan(out[1]).item()
