"""Weight decay of the sizes that a policy is trained with, lr * weight_decay from 1e-8 to 1e-6 of the parameter a step, which is of the order of a
parameter's last bit or below it.

One step: the new parameter is the exact one rounded once (half a step of fp32, taken at whichever of the two is larger), but for the update's own 30 eps, eps = 2^-24
(as tests/test_gpu_adamw.py counts them: 24, and 6 of the first moment), and 4 eps of the decay.
In the mean: sum p (p - p' - update) / sum p^2 is lr weight_decay, but for the roundings.  Those do not average out: the first step's updates are all of one size, so that
within a power of two the part that is rounded off moves with p alone.  (Taken for independent, with a deviation of 3.5e-8 p each, 200,000 of them would leave 1.4e-10; the exact
results rounded to fp32 by the host are off by up to 7.5e-10.)  So the estimate is compared with that of the exact results rounded once.  The two differ where the exact
one lies so near to the middle of two numbers that its own bound reaches over it, and there by one step: the sum of p times that step over those elements is what is allowed."""
import numpy as np
import pytest

from oracle import update as ou

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
B1, B2, ADAM_EPS = 0.9, 0.95, 1e-8


def step(n, lr, wd, bits, master, gradient, seed):
    """(p, p', what the step's own definition gives from the given state in 64 bits)"""
    import torch
    from paper_2506_24119_amd import binding as sb
    rng = np.random.default_rng(seed)
    dev = lambda a, t=torch.float32: torch.from_numpy(np.asarray(a, np.float32)).cuda().to(t)  # noqa: E731
    p = dev(rng.normal(size=n) * 0.05)
    g = dev(rng.normal(size=n) * (1e-3 if gradient else 0.0))
    state = torch.float32 if bits == 32 else torch.float8_e4m3fn
    m, v = (torch.zeros(n, device="cuda").to(state) for _ in range(2))
    scales = {} if bits == 32 else {k: torch.zeros(-(-n // sb.SPIRAL_ADAMW_BLOCK), device="cuda") for k in ("m_scale", "v_scale")}
    half = p.bfloat16() if master else None
    rec = sb.spiral_adamw_tensor(half if master else p, g, m, v, master=p if master else None, **scales)
    mem = torch.empty(sb.spiral_adamw_bytes([rec]), dtype=torch.uint8, device="cuda")
    opt = sb.spiral_adamw_create([rec], mem)
    before = {"p": p.double().cpu().numpy(), "g": g.double().cpu().numpy(), "m": np.zeros(n), "v": np.zeros(n), "decay": 1}
    sb.spiral_adamw_step(opt, lr, B1, B2, ADAM_EPS, wd, 1)
    torch.cuda.synchronize()
    sb.spiral_adamw_free(opt)
    if master:
        assert torch.equal(half, p.bfloat16())
    return before["p"], p.double().cpu().numpy(), ou.adamw([before], lr, B1, B2, ADAM_EPS, wd, 1)[0][0]


SETTINGS = [(1e-6, 0.01), (1e-6, 0.1), (2e-6, 0.1), (1e-6, 0.7), (3e-5, 0.01), (1e-2, 0.1)]


@pytest.mark.parametrize("lr,wd", SETTINGS)
@pytest.mark.parametrize("bits,master", [(32, False), (32, True), (8, True)])
@pytest.mark.parametrize("gradient", [True, False])
def test_the_parameter_is_rounded_once(lr, wd, bits, master, gradient):
    p, got, want = step(9001, lr, wd, bits, master, gradient, seed=int(wd * 100) + bits)
    ulp = np.spacing(np.maximum(np.abs(got), np.abs(want["p"])).astype(np.float32)).astype(np.float64)
    bound = ulp / 2 + 30 * EPS * np.abs(want["update"]) + 4 * EPS * lr * wd * np.abs(p)
    assert (np.abs(got - want["p"]) <= bound).all(), (np.abs(got - want["p"]) / bound).max()


@pytest.mark.parametrize("lr,wd", SETTINGS[:4])
@pytest.mark.parametrize("bits", [32, 8])
def test_decay_in_the_mean(lr, wd, bits):
    n = 200_000
    p, got, want = step(n, lr, wd, bits, False, True, seed=5 + bits)
    estimate = lambda new: (p * (p - new - want["update"])).sum() / (p * p).sum()  # noqa: E731
    once = want["p"].astype(np.float32)
    ulp = np.spacing(np.abs(once)).astype(np.float64)
    # distance from the nearest middle of two numbers; below a power of two the steps are half as long, which the minimum with a quarter step covers
    off = np.abs(want["p"] - once.astype(np.float64))
    near = np.minimum(np.abs(ulp / 2 - off), np.abs(ulp / 4 - off)) <= 30 * EPS * np.abs(want["update"]) + 4 * EPS * lr * wd * np.abs(p)
    allowed = (np.abs(p) * ulp)[near].sum() / (p * p).sum()
    assert abs(estimate(got) - estimate(once.astype(np.float64))) <= allowed, (estimate(got), estimate(once.astype(np.float64)), allowed)
    assert allowed <= 0.05 * lr * wd                                   # and that is little beside the decay itself


def test_an_infinite_parameter_stays():
    """fp16 without a master: what has once passed its largest value is infinite, not undefined, from then on."""
    import torch
    from paper_2506_24119_amd import binding as sb
    p = torch.full((300,), 2.0, dtype=torch.float16, device="cuda")
    p[7], p[8], p[9] = float("inf"), float("-inf"), float("nan")
    g, m, v = torch.ones(300, device="cuda"), torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    rec = sb.spiral_adamw_tensor(p, g, m, v)
    mem = torch.empty(sb.spiral_adamw_bytes([rec]), dtype=torch.uint8, device="cuda")
    opt = sb.spiral_adamw_create([rec], mem)
    for wd in (0.0, 0.1):
        sb.spiral_adamw_step(opt, 1e-2, B1, B2, ADAM_EPS, wd, 1)
        torch.cuda.synchronize()
        assert p[7].item() == float("inf") and p[8].item() == float("-inf") and torch.isnan(p[9]).item()
        assert torch.isfinite(p[10:]).all()
    sb.spiral_adamw_free(opt)
