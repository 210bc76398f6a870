"""spiral_policy_gradient where scale / temperature passes 32 bits, with the bounds of tests/test_gpu_policy_gradient.py."""
import numpy as np
import pytest

from test_gpu_policy_gradient import matrix, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [50, 70000])
@pytest.mark.parametrize("T,scale", [(1e-30, 1e9), (1e-20, 1e30)])
def test_a_scale_over_the_temperature_that_passes_32_bits(T, scale, V):
    """1e39 and 1e50 times a slope of nothing is nothing, and times a small one what it is.  All logits are equal, so the softmax is 1 / V at any temperature."""
    from paper_2506_24119_amd import binding as sb
    n = 5
    whole, rows = matrix(n, V, "float32", 0, 0)
    rows.fill_(2.0)
    y = np.array([0, 1, 2, 3, V - 1], np.int32)
    lp0 = -np.log(V)
    old = np.array([lp0, lp0 - 2.0, lp0 + 2.0, lp0, lp0], np.float32)             # ratios 1, e^2 and e^-2 (clipped both), 1, 1
    unit = scale / T
    adv = np.array([0.0, 3.0, -3.0, 1e12 / unit, -1e30 / unit], np.float32)
    _, grad = matrix(n, V, "float32", 0, 0)
    lp = run(sb, rows, y, old, adv, None, T, 0.2, scale, grad)
    g = grad.cpu().numpy().astype(np.float64)
    assert np.abs(lp - lp0).max() <= 2.0 ** -24 * (2 * abs(lp0) + V / 256 + 64)
    assert (g[:3] == 0).all()
    for i in (3, 4):
        slope = float(np.float32(scale)) / float(np.float32(T)) * float(adv[i])
        want = np.full(V, slope / V)
        want[y[i]] -= slope
        R = 2.0 ** -24 * (2 * abs(lp0) + V / 256 + 64 + 2 * abs(lp0))             # of the ratio and of the softmax, as in the other tests
        if adv[i] < 2e-38 and adv[i] > -2e-38:
            R += 2.0 ** -150 / abs(float(adv[i]))                                 # an advantage of few bits
        assert (np.abs(g[i] - want) <= 3 * R * (np.abs(want) + abs(slope) / V)).all(), np.abs(g[i] / want - 1).max()
