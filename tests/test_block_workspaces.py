"""What the learner's operators between matrix products ask for as a workspace, on the host: no more than the parts that a call of any type writes."""
import pytest

from paper_2506_24119_amd import binding as sb


@pytest.mark.parametrize("n,d,parts", [(1, 7, 1), (5000, 7, 128), (128, 5, 128), (127, 1, 127), (5000, 8, 512), (5000, 12288, 512), (300, 12288, 300), (5000, 12289, 128), (100, 12289, 100),
                                       (1 << 20, 1 << 24, 128), (16384, 3584, 512)])
def test_norm_gradient(n, d, parts):
    assert sb.spiral_add_rmsnorm_backward_workspace_bytes(n, d) == parts * d * 4


@pytest.mark.parametrize("d", [7, 12289, 20000])
def test_norm_gradient_refuses_less(d):
    lib, P = sb.load_library(), 1 << 40
    need = sb.spiral_add_rmsnorm_backward_workspace_bytes(5000, d)
    assert lib.spiral_add_rmsnorm_backward(P, d, 2 * P, d, 3 * P, 4 * P, None, 0, 1, 5000, d, 5 * P, d, 6 * P, 7 * P, need - 1, None) == sb.SPIRAL_ERR_INVALID_ARG
    assert "workspace" in sb.spiral_last_error()
