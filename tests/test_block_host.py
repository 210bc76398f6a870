"""What the learner's operators between matrix products refuse, on the host: every call here is turned down before anything is enqueued (the
addresses are made up)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2506_24119_amd import binding as sb

P = 1 << 20                      # an aligned address that nothing dereferences
INVALID, SHAPE = sb.SPIRAL_ERR_INVALID_ARG, sb.SPIRAL_ERR_SHAPE


@pytest.fixture(scope="module")
def lib():
    return sb.load_library()


def refused(rc, code, text):
    assert rc == code, (rc, sb.spiral_last_error())
    assert text in sb.spiral_last_error(), sb.spiral_last_error()


def ints(a):
    a = np.asarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(C.POINTER(C.c_int32))


# ------------------------------------------------------------------------------------------------ attention
def create(lib, lens=(5, 0, 7), hq=4, hkv=2, hd=64, mem=P, nbytes=1 << 30, B=None):
    keep, p = (None, None) if lens is None else ints(lens)
    out = C.c_void_p(1)
    rc = lib.spiral_attention_plan_create(p, len(lens or ()) if B is None else B, hq, hkv, hd, mem, nbytes, None, C.byref(out))
    assert rc == 0 or not out.value
    return rc


@pytest.mark.parametrize("change,code,text", [
    (dict(lens=None, B=3), INVALID, "no sequences"), (dict(B=0), INVALID, "no sequences"), (dict(lens=(5, -1)), INVALID, "length -1 of sequence 1"), (dict(lens=(0, 0)), INVALID, "0 rows"),
    (dict(lens=(1 << 30, 1 << 30)), INVALID, "2147483648 rows"), (dict(hd=16), SHAPE, "head_dim 16"), (dict(hd=256), SHAPE, "head_dim"), (dict(hq=5), SHAPE, "5 query heads"), (dict(hkv=0), SHAPE, "0 kv heads"),
    (dict(hq=0), SHAPE, "0 query heads"), (dict(hq=2048), SHAPE, "2048"), (dict(mem=None), INVALID, "memory"), (dict(mem=P + 128), INVALID, "memory"), (dict(nbytes=0), INVALID, "memory")])
def test_plan_refuses(lib, change, code, text):
    refused(create(lib, **change), code, text)
    if "mem" not in change and "nbytes" not in change and "lens" in change and change["lens"]:
        assert sb.spiral_attention_plan_bytes(change["lens"], 4, 2, 64) == 0


def test_plans_null(lib):
    _, p = ints([3])
    assert lib.spiral_attention_plan_create(p, 1, 2, 1, 64, P, 1 << 20, None, None) == INVALID
    assert lib.spiral_attention_backward_workspace_bytes(None) == 0
    lib.spiral_attention_plan_free(None)
    refused(lib.spiral_attention_forward(None, P, 64, P, 64, P, 64, 1, 1.0, P, 64, P, None), sb.SPIRAL_ERR_NOT_LOADED, "null plan")
    refused(lib.spiral_attention_backward(None, P, 64, P, 64, P, 64, P, 64, P, P, 64, 1, 1.0, P, 64, P, 64, P, 64, P, 1 << 20, None), sb.SPIRAL_ERR_NOT_LOADED, "null plan")
    for call in (sb.spiral_attention_backward_workspace_bytes, lambda p: sb.spiral_attention_forward(p, None, None, None, 1.0, None, None)):
        with pytest.raises(ValueError):
            call(12345)


# ------------------------------------------------------------------------------------------------ addition and RMSNorm
def norm(lib, **change):
    a = dict(x=P, xs=100, r=2 * P, rs=100, g=3 * P, dtype=1, n=8, d=100, eps=1e-6, out=4 * P, od=1, os=100, sc=None, sum=5 * P, ss=100, rstd=6 * P)
    a.update(change)
    return lib.spiral_add_rmsnorm(a["x"], a["xs"], a["r"], a["rs"], a["g"], a["dtype"], a["n"], a["d"], a["eps"], a["out"], a["od"], a["os"], a["sc"], a["sum"], a["ss"], a["rstd"], None)


@pytest.mark.parametrize("change,text", [
    (dict(x=None), "null"), (dict(g=None), "null"), (dict(out=None), "null"), (dict(n=0), "n_rows"), (dict(n=1 << 31), "n_rows"), (dict(d=0), "d=0"), (dict(d=(1 << 24) + 1), "d="),
    (dict(dtype=3, od=3), "type"), (dict(dtype=-1, od=-1), "type"), (dict(od=0), "type"), (dict(od=2), "type"), (dict(od=3), "scales"), (dict(sc=P), "scales"), (dict(xs=99), "stride"),
    (dict(rs=99), "stride"), (dict(os=99), "stride"), (dict(ss=99), "stride"), (dict(x=P + 1), "misaligned"), (dict(r=P + 1), "misaligned"), (dict(g=P + 2), "misaligned"),
    (dict(out=P + 1), "misaligned"), (dict(sum=P + 1), "misaligned"), (dict(rstd=P + 2), "misaligned"), (dict(eps=-1e-6), "eps"), (dict(eps=math.nan), "eps"), (dict(eps=1.5), "eps"),
    (dict(out=P), "overlaps"), (dict(out=2 * P + 1598), "overlaps"), (dict(out=3 * P + 398), "overlaps"), (dict(out=5 * P), "overlaps"), (dict(sum=P, ss=101), "overlaps"), (dict(sum=P + 2), "overlaps"),
    (dict(rstd=P + 4), "overlaps"), (dict(rstd=3 * P), "overlaps"), (dict(od=3, sc=6 * P), "overlaps"), (dict(od=3, sc=4 * P + 16), "overlaps"), (dict(xs=300, os=300, out=P + 198), "overlaps")])
def test_norm_refuses(lib, change, text):
    refused(norm(lib, **change), INVALID, text)


def norm_grad(lib, **change):
    a = dict(dy=P, dys=100, h=2 * P, hs=100, g=3 * P, rstd=4 * P, ds=5 * P, dss=100, dtype=1, n=8, d=100, dx=6 * P, dxs=100, dg=7 * P, ws=8 * P, bytes=1 << 30)
    a.update(change)
    return lib.spiral_add_rmsnorm_backward(a["dy"], a["dys"], a["h"], a["hs"], a["g"], a["rstd"], a["ds"], a["dss"], a["dtype"], a["n"], a["d"], a["dx"], a["dxs"], a["dg"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("change,text", [
    (dict(dy=None), "null"), (dict(h=None), "null"), (dict(g=None), "null"), (dict(rstd=None), "null"), (dict(dx=None), "null"), (dict(n=0), "n_rows"), (dict(d=0), "d=0"), (dict(dtype=3), "type"),
    (dict(dys=99), "stride"), (dict(hs=99), "stride"), (dict(dss=99), "stride"), (dict(dxs=99), "stride"), (dict(dy=P + 1), "misaligned"), (dict(dg=7 * P + 2), "misaligned"), (dict(rstd=4 * P + 1), "misaligned"),
    (dict(ws=None), "workspace"), (dict(ws=8 * P + 64), "workspace"), (dict(bytes=3), "workspace"), (dict(dx=2 * P), "overlaps"), (dict(dx=P, dxs=104), "overlaps"), (dict(dx=5 * P + 2), "overlaps"),
    (dict(dg=3 * P), "overlaps"), (dict(dg=4 * P), "overlaps"), (dict(ws=P), "overlaps"), (dict(dx=P, ds=P, dss=104), "overlaps"), (dict(dg=6 * P + 1596), "overlaps")])
def test_norm_gradient_refuses(lib, change, text):
    refused(norm_grad(lib, **change), INVALID, text)


# ------------------------------------------------------------------------------------------------ norm and rotation
def rope(lib, **change):
    a = dict(q=P, qs=384, k=P + 512, ks=384, gq=2 * P, gk=2 * P, dtype=1, n=8, hq=4, hk=2, hd=64, eps=1e-6, theta=1e6, pos=3 * P, oq=4 * P, oqs=256, ok=5 * P, oks=128)
    a.update(change)
    return lib.spiral_norm_rope(a["q"], a["qs"], a["k"], a["ks"], a["gq"], a["gk"], a["dtype"], a["n"], a["hq"], a["hk"], a["hd"], a["eps"], a["theta"], a["pos"], a["oq"], a["oqs"], a["ok"], a["oks"], None)


COMMON = [(dict(pos=None), INVALID, "positions"), (dict(pos=3 * P + 2), INVALID, "positions"), (dict(n=0), INVALID, "n_rows"), (dict(n=1 << 31), INVALID, "n_rows"), (dict(hd=48), SHAPE, "head_dim 48"), (dict(hq=0), SHAPE, "0 query"),
          (dict(hk=0), SHAPE, "0 kv"), (dict(hq=1025), SHAPE, "1025"), (dict(dtype=3), INVALID, "type"), (dict(eps=-1.0), INVALID, "eps"), (dict(eps=math.nan), INVALID, "eps"), (dict(theta=0.5), INVALID, "theta"),
          (dict(theta=math.inf), INVALID, "theta"), (dict(theta=math.nan), INVALID, "theta")]


@pytest.mark.parametrize("change,code,text", COMMON + [(c, INVALID, t) for c, t in (
    (dict(q=None), "null"), (dict(k=None), "null"), (dict(oq=None), "null"), (dict(ok=None), "null"), (dict(qs=255), "stride"), (dict(ks=127), "stride"), (dict(oqs=255), "stride"), (dict(oks=127), "stride"),
    (dict(q=P + 1), "misaligned"), (dict(ok=5 * P + 1), "misaligned"), (dict(gq=2 * P + 2), "misaligned"), (dict(oq=P), "overlaps"), (dict(oq=P + 2, oqs=384), "overlaps"), (dict(ok=P + 510, oks=384), "overlaps"),
    (dict(oq=5 * P, oqs=384, ok=5 * P + 510, oks=384), "overlaps"), (dict(oq=3 * P), "overlaps"), (dict(ok=2 * P), "overlaps"), (dict(oq=P, oqs=384, q=P + 2), "overlaps"))])
def test_rope_refuses(lib, change, code, text):
    refused(rope(lib, **change), code, text)


def rope_grad(lib, **change):
    a = dict(q=P, qs=384, k=P + 512, ks=384, gq=2 * P, gk=2 * P, dtype=1, n=8, hq=4, hk=2, hd=64, eps=1e-6, theta=1e6, pos=3 * P, dyq=4 * P, dyqs=256, dyk=5 * P, dyks=128, dq=6 * P, dqs=384, dk=6 * P + 512, dks=384,
             dgq=7 * P, dgk=7 * P + 256, ws=8 * P, bytes=1 << 30)
    a.update(change)
    return lib.spiral_norm_rope_backward(a["q"], a["qs"], a["k"], a["ks"], a["dyq"], a["dyqs"], a["dyk"], a["dyks"], a["gq"], a["gk"], a["dtype"], a["n"], a["hq"], a["hk"], a["hd"], a["eps"], a["theta"], a["pos"],
                                         a["dq"], a["dqs"], a["dk"], a["dks"], a["dgq"], a["dgk"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("change,code,text", COMMON + [(c, INVALID, t) for c, t in (
    (dict(q=None), "null"), (dict(k=None), "null"), (dict(dyq=None), "null"), (dict(dyk=None), "null"), (dict(dq=None), "null"), (dict(dk=None), "null"), (dict(gq=None), "not there"), (dict(gk=None), "not there"),
    (dict(qs=255), "stride"), (dict(dyqs=255), "stride"), (dict(dyks=127), "stride"), (dict(dqs=255), "stride"), (dict(dks=127), "stride"), (dict(dyq=4 * P + 1), "misaligned"), (dict(dgq=7 * P + 2), "misaligned"),
    (dict(ws=None), "workspace"), (dict(ws=8 * P + 8), "workspace"), (dict(bytes=16), "workspace"), (dict(dq=P), "overlaps"), (dict(dq=4 * P), "overlaps"), (dict(dgk=7 * P + 252), "overlaps"), (dict(dgq=2 * P), "overlaps"),
    (dict(ws=4 * P), "overlaps"), (dict(dk=6 * P + 510), "overlaps"))])
def test_rope_gradient_refuses(lib, change, code, text):
    refused(rope_grad(lib, **change), code, text)


def test_sizes_of_workspaces():
    assert sb.spiral_add_rmsnorm_backward_workspace_bytes(0, 10) == 0 and sb.spiral_add_rmsnorm_backward_workspace_bytes(10, 0) == 0 and sb.spiral_add_rmsnorm_backward_workspace_bytes(1, 1) > 0
    assert sb.spiral_norm_rope_backward_workspace_bytes(0, 1, 1, 64) == 0 and sb.spiral_norm_rope_backward_workspace_bytes(1, 1, 1, 48) == 0 and sb.spiral_norm_rope_backward_workspace_bytes(1, 1, 1, 64) > 0
    assert sb.spiral_attention_plan_bytes([], 1, 1, 64) == 0 and sb.spiral_attention_plan_bytes([3, 0], 2, 1, 64) > 0


def test_binding_checks_what_it_marshals():
    import torch
    x, g, v = torch.zeros(4, 10), torch.zeros(10), torch.zeros(4)
    for bad in (dict(dev_x=x.t()[:, ::2]), dict(dev_x=x[0]), dict(dev_residual=x.half()), dict(dev_residual=x[:3]), dict(dev_gain=v), dict(dev_gain=g.half()), dict(dev_out=x.half()), dict(dev_sum=x[:, :9]),
                dict(dev_rstd=g), dict(dev_out=x[:3])):
        a = dict(dev_x=x, dev_residual=x, dev_gain=g, eps=1e-6, dev_out=x.clone(), stream=0)
        a.update(bad)
        with pytest.raises(ValueError):
            sb.spiral_add_rmsnorm(**a)
    with pytest.raises(TypeError):
        sb.spiral_add_rmsnorm(x.double(), None, g, 1e-6, x.double(), stream=0)
    for bad in (dict(dev_dout=x.half()), dict(dev_dsum=x[:, :9]), dict(dev_dx=x[:3]), dict(dev_rstd=g), dict(dev_gain=v), dict(dev_dgain=v)):
        a = dict(dev_dout=x, dev_sum=x, dev_gain=g, dev_rstd=v, dev_dsum=None, dev_dx=x.clone(), dev_dgain=g.clone(), dev_workspace=None, stream=0)
        a.update(bad)
        with pytest.raises(ValueError):
            sb.spiral_add_rmsnorm_backward(**a)
    q, k, h, pos = torch.zeros(4, 3, 32), torch.zeros(4, 1, 32), torch.zeros(32), torch.zeros(4, dtype=torch.int32)
    for bad in (dict(dev_k=k.half()), dict(dev_k=torch.zeros(4, 1, 64)), dict(dev_out_q=q.transpose(0, 1)), dict(dev_out_k=q), dict(dev_gain_q=v), dict(dev_positions=pos.long()), dict(dev_positions=pos[:3]),
                dict(dev_q=torch.zeros(4, 6, 32)[:, ::2]), dict(dev_q=torch.zeros(4, 3, 64)[:, :, ::2])):
        a = dict(dev_q=q, dev_k=k, dev_gain_q=h, dev_gain_k=h, eps=1e-6, theta=1e4, dev_positions=pos, dev_out_q=q.clone(), dev_out_k=k.clone(), stream=0)
        a.update(bad)
        with pytest.raises(ValueError):
            sb.spiral_norm_rope(**a)
    for bad in (dict(dev_q=k), dict(dev_dout_k=k.half()), dict(dev_dq=k), dict(dev_dgain_q=v)):
        a = dict(dev_q=q, dev_k=k, dev_dout_q=q, dev_dout_k=k, dev_gain_q=h, dev_gain_k=h, eps=1e-6, theta=1e4, dev_positions=pos, dev_dq=q.clone(), dev_dk=k.clone(), dev_dgain_q=h.clone(), dev_dgain_k=h.clone(),
                 dev_workspace=None, stream=0)
        a.update(bad)
        with pytest.raises(ValueError):
            sb.spiral_norm_rope_backward(**a)
