"""Host-only guard on the rows' kernels: every form that the launches name is built, and the norm's has the waves a SIMD that its registers were chosen for."""
import re

from test_block_resources import resources


def test_forms_and_their_registers(tmp_path):
    found = resources(tmp_path, "kernels_block.hip")
    of = lambda kernel: {k: v for k, v in found.items() if kernel in k}  # noqa: E731
    # types x 16 or 8 bits out x one or four waves x eights a lane (4 of fp32, 8 of the others) x past the caches' order or not
    assert len(of("15add_norm_kernel")) == (4 + 8 + 8) * 2 * 2 * 2, sorted(found)
    assert len(of("16norm_grad_kernel")) == (4 + 6 + 6) * 2 * 2
    assert len(of("16norm_rope_kernel")) == 3 * 3 * 2 * 2
    for name in ("add_norm_long_kernel", "norm_grad_long_kernel", "gain_part_kernel"):
        assert len(of(name)) == 3, name
    assert len(of("add_parts_kernel")) == 1
    for name, (vgprs, spills) in of("15add_norm_kernel").items():
        eights = int(re.search(r"Li[14]ELi(\d)E", name).group(1))
        assert vgprs <= (128 if eights <= 2 else 168 if eights <= 5 else 256) and spills == 0, (name, vgprs, spills)
    # two workgroups of four waves a compute unit
    for name, (vgprs, spills) in {**of("16norm_grad_kernel"), **of("16norm_rope_kernel")}.items():
        assert vgprs <= 256 and spills == 0, (name, vgprs, spills)
    # add_parts_kernel: 1,024 threads
    assert all(vgprs <= 128 for vgprs, _ in of("add_parts_kernel").values())
