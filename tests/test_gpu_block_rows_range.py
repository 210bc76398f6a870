"""spiral_add_rmsnorm where 32 bits do not tell: 8-bit codes and scales of rows whose products of sums and gains leave their range or their normal numbers, codes of sums that
they do not hold, outputs whose products of sum and gain, or of 1 / rms and gain, they do not.

Bounds, u = 2^-24: 1 / rms is off by u (d / 128 + 16), a scale by four roundings more and its own, an output by that and half a step of its type."""
import numpy as np
import pytest

from test_gpu_block_rows import HALF, LEAST, U, sb  # noqa: F401  (sb: the fixture)

pytestmark = pytest.mark.gpu


def some(dtype, n, d, size, seed):
    """[n, d] of random signs and three binary orders of magnitude below `size`, a hundredth of them up to 20 orders."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rand = lambda: torch.rand((n, d), device="cuda", generator=g, dtype=torch.float64)  # noqa: E731
    x = size * torch.exp2(-3 * rand() - torch.where(rand() < 0.01, 20 * rand(), 0)) * torch.where(rand() < 0.5, -1.0, 1.0)
    return x.to(getattr(torch, dtype))


# the largest products: below 2^-119.2 (448 over it passes 32 bits), 2^-117 (smaller ones are subnormal where they have codes), 2^-145 (all are), 2^133 (past 32 bits)
SIZES = [("float32", 2.0 ** -119.5, 1.0, 1e-14), ("bfloat16", 2.0 ** -119.5, 1.0, 1e-14), ("float16", 2.0 ** -22, 2.0 ** -98, 1e-14), ("float32", 2.0 ** -117, 1.0, 1e-14), ("bfloat16", 2.0 ** -117, 1.0, 1e-14),
         ("float32", 2.0 ** -60, 2.0 ** -85, 0.0), ("bfloat16", 2.0 ** -60, 2.0 ** -85, 0.0), ("float32", 2.0 ** 50, 2.0 ** 83, 1e-6), ("bfloat16", 2.0 ** 50, 2.0 ** 83, 1e-6)]


def exact(x, gain, eps):
    """(sum times gain, 1 / rms) in 64 bits"""
    h = x.double()
    return h * gain.double(), 1 / (h.square().mean(1, keepdim=True) + float(np.float32(eps))).sqrt()


def gain_of(d, size):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    return (size * (0.7 + 0.3 * torch.rand(d, device="cuda", generator=g, dtype=torch.float64))).float()


@pytest.mark.parametrize("n,d", [(6, 100), (3, 2560), (5, 20000), (2100, 130), (2049, 2560), (7, 5)])
@pytest.mark.parametrize("dtype,size,gain_size,eps", SIZES)
def test_codes_of_products_far_from_one(sb, n, d, dtype, size, gain_size, eps):  # noqa: F811
    """Beside rows of ordinary size, which keep theirs."""
    import torch
    x = some(dtype, n, d, size, n + d)
    gain = gain_of(d, gain_size)
    ordinary = torch.arange(n, device="cuda") % 3 == 1
    if gain_size == 1.0:                                      # (a gain far from 1 is every row's)
        x[ordinary] = some(dtype, n, d, 1.0, 3)[ordinary]
    out, scale = torch.full((n, d), 1.0, device="cuda").to(torch.float8_e4m3fn), torch.full((n,), 5.0, device="cuda")
    sb.spiral_add_rmsnorm(x, None, gain, eps, out, scale)
    p, rstd = exact(x, gain, eps)
    most = p.abs().amax(1, keepdim=True)
    assert (most * rstd > 1.01e-30).all() and (most * rstd < 3e38).all()
    v = p * (448.0 / most)
    step = torch.exp2(torch.clamp(torch.frexp(v)[1] - 1, min=-6).double() - 3)
    assert torch.equal(out.double(), torch.round(v / step) * step)
    want = (most * rstd / 448)[:, 0]
    assert ((scale.double() - want).abs() <= U * (d / 128 + 21) * want + LEAST["float32"]).all()


@pytest.mark.parametrize("n,d", [(4000, 2560), (700, 8200), (40, 20001), (2100, 4090), (300000, 5)])
@pytest.mark.parametrize("dtype,apart", [("float32", 0), ("float32", 12), ("bfloat16", 17), ("float16", 16)])
@pytest.mark.parametrize("place", ["apart", "over x", "over residual", "none"])
def test_codes_of_sums_that_32_bits_do_not_hold(sb, n, d, dtype, apart, place):  # noqa: F811
    """Sums of more than 24 bits, x `apart` orders of magnitude below the residual stream: every code that of the 64-bit quotient, of sums in 64 bits where their parts are of 32
    and in 32 where they are of 16, wherever the sum goes."""
    import torch
    x, res = some(dtype, n, d, 4.0 * 2.0 ** -apart, n), some(dtype, n, d, 4.0, d)
    gain = gain_of(d, 1.0)
    p = (x.double() + res.double() if dtype == "float32" else (x.float() + res.float()).double()) * gain.double()
    total = (x.float() + res.float()).to(x.dtype)
    out, scale = torch.empty((n, d), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(n, device="cuda")
    into = {"apart": torch.empty_like(x), "over x": x, "over residual": res, "none": None}[place]
    sb.spiral_add_rmsnorm(x, res, gain, 1e-6, out, scale, into)
    v = p * (448.0 / p.abs().amax(1, keepdim=True))
    step = torch.exp2(torch.clamp(torch.frexp(v)[1] - 1, min=-6).double() - 3)
    assert torch.equal(out.double(), torch.round(v / step) * step)
    assert into is None or torch.equal(into, total)


@pytest.mark.parametrize("n,d", [(6, 100), (3, 2560), (5, 40000), (2100, 130), (7, 5)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size,gain_size", [(2.0 ** 50, 2.0 ** 83), (2.0 ** -60, 2.0 ** -80)])
def test_outputs_whose_products_leave_32_bits(sb, n, d, dtype, size, gain_size):  # noqa: F811
    """gain rstd sum is in range, gain sum alone is not."""
    import torch
    x, gain = some(dtype, n, d, size, 5), gain_of(d, gain_size)
    out = torch.zeros_like(x)
    sb.spiral_add_rmsnorm(x, None, gain, 0.0, out)
    p, rstd = exact(x, gain, 0.0)
    want = p * rstd
    assert torch.isfinite(want.to(out.dtype)).all()
    half = HALF[dtype]
    assert ((out.double() - want).abs() <= (half + U * (d / 128 + 24)) * want.abs() * (1 + half) + LEAST[dtype]).all()


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("size,gain_size", [(2.0 ** -60, 2.0 ** 83), (2.0 ** 55, 2.0 ** -85)])
def test_heads_whose_gain_over_rms_leaves_32_bits(sb, hd, dtype, size, gain_size):  # noqa: F811
    """At position 0 a head's output is its norm."""
    import torch
    x, gain = some(dtype, 50, 5 * hd, size, hd).unflatten(1, (5, hd)), gain_of(hd, gain_size)
    out = torch.zeros_like(x)
    sb.spiral_norm_rope(x[:, :4], x[:, 4:], gain, gain, 0.0, 1e4, torch.zeros(50, dtype=torch.int32, device="cuda"), out[:, :4], out[:, 4:])
    want = x.double() * gain.double() / x.double().square().mean(2, keepdim=True).sqrt()
    assert torch.isfinite(want.to(out.dtype)).all()
    half = HALF[dtype]
    assert ((out.double() - want).abs() <= (half + U * (hd / 32 + 32)) * want.abs() * (1 + half) + LEAST[dtype]).all()
