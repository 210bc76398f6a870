"""Settings of an AdamW step that 32 bits cannot hold are refused: elements without a gradient would become undefined (infinite times nothing)."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [dict(lr=1e39), dict(lr=1e38, step=1), dict(lr=1e20, weight_decay=1e19), dict(lr=1.0, weight_decay=1e300), dict(lr=1e300, weight_decay=1e300)])
def test_settings_past_32_bits_are_refused(bad):
    import torch
    from paper_2506_24119_amd import binding as sb
    p, g, m, v = torch.ones(300, device="cuda"), torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    rec = sb.spiral_adamw_tensor(p, g, m, v)
    mem = torch.empty(sb.spiral_adamw_bytes([rec]), dtype=torch.uint8, device="cuda")
    opt = sb.spiral_adamw_create([rec], mem)
    ok = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.0, step=1)
    with pytest.raises(sb.SpiralError) as e:
        sb.spiral_adamw_step(opt, **{**ok, **bad})
    assert e.value.code == sb.SPIRAL_ERR_INVALID_ARG and "32 bits" in str(e.value)
    torch.cuda.synchronize()
    assert (p == 1).all() and (m == 0).all() and (v == 0).all()
    sb.spiral_adamw_step(opt, **{**ok, "lr": 1e37, "step": 100})                 # as large as they may be: no gradient, no change
    torch.cuda.synchronize()
    assert (p == 1).all()
    sb.spiral_adamw_free(opt)
