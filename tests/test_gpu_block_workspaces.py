"""spiral_add_rmsnorm_backward on more rows than parts, of widths that registers do not hold: the gain's sums, and nothing written behind the workspace.

Bounds are those of the other tests of rows."""
import numpy as np
import pytest

from oracle import block as ob
from test_gpu_block_rows import U, host, matrix, sb  # noqa: F401  (sb: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("n,d", [(300, 12289), (1000, 7), (300, 12288), (300, 8200), (1000, 8)])
def test_workspace_of_the_gains_sums(sb, dtype, n, d):  # noqa: F811
    import torch
    rng = np.random.default_rng(n + d)
    _, dy = matrix(n, d, dtype, 1, 0, rng.normal(size=(n, d)) * 0.1)
    _, total = matrix(n, d, dtype, 0, 0, rng.normal(size=(n, d)))
    gain = torch.from_numpy((1 + 0.3 * rng.normal(size=d)).astype(np.float32)).cuda()
    rstd = torch.from_numpy((1 / np.sqrt((host(total) ** 2).mean(1) + 1e-5)).astype(np.float32)).cuda()
    need = sb.spiral_add_rmsnorm_backward_workspace_bytes(n, d)
    room = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    dx, dg = torch.empty_like(total), torch.empty(d, device="cuda")
    sb.spiral_add_rmsnorm_backward(dy, total, gain, rstd, None, dx, dg, room[:need])
    torch.cuda.synchronize()
    assert (room[need:] == 0xA5).all()
    _, want = ob.add_rmsnorm_grad(host(dy), host(total), host(gain), host(rstd))
    size = (np.abs(host(dy)) * np.abs(host(total)) * host(rstd)[:, None]).sum(0)
    assert (np.abs(host(dg) - want) <= U * (n / 8 + 64) * size).all()
