"""What the entry points of a policy update refuse, on the host: every call here is turned down before anything is enqueued (the addresses
are made up)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2506_24119_amd import binding as sb

P = 1 << 20                      # an aligned address that nothing dereferences


@pytest.fixture(scope="module")
def lib():
    return sb.load_library()


def refused(rc, code, text):
    assert rc == code, rc
    assert text in sb.spiral_last_error(), sb.spiral_last_error()


def draw(lib, **change):
    a = dict(logits=P, dtype=0, stride=100, B=4, V=100, T=None, k=None, p=None, mp=None, u=P, ws=P, bytes=1 << 40, out=P, logp=P)
    a.update(change)
    keep = []

    def host(x, t):
        if x is None:
            return None
        keep.append(np.asarray(x, dtype=t))
        return keep[-1].ctypes.data
    return lib.spiral_sample_uniform(a["logits"], a["dtype"], a["stride"], a["B"], a["V"], host(a["T"], np.float32), host(a["k"], np.int32),
                                     host(a["p"], np.float32), host(a["mp"], np.float32), a["u"], a["ws"], a["bytes"], a["out"], a["logp"], None)


@pytest.mark.parametrize("change,text", [
    (dict(logits=None), "null"), (dict(u=None), "null"), (dict(out=None), "null"), (dict(B=0), "bad B"), (dict(B=1025), "bad B"),
    (dict(V=0), "V=0"), (dict(dtype=3), "type"), (dict(dtype=-1), "type"), (dict(stride=99), "stride"), (dict(logits=P + 2), "misaligned"),
    (dict(logits=P + 1, dtype=1), "misaligned"), (dict(u=P + 2), "misaligned"), (dict(out=P + 1), "misaligned"), (dict(logp=P + 2), "misaligned"),
    (dict(ws=None), "workspace"), (dict(ws=P + 64), "workspace"), (dict(bytes=0), "workspace"),
    (dict(T=[1, -1, 1, 1]), "temperature of row 1"), (dict(T=[1, 1, 1, math.inf]), "temperature of row 3"), (dict(T=[math.nan] * 4), "temperature"),
    (dict(p=[1, 1, 0, 1]), "top_p of row 2"), (dict(p=[1.5] * 4), "top_p"), (dict(p=[math.nan] * 4), "top_p"),
    (dict(mp=[0, -0.1, 0, 0]), "min_p of row 1"), (dict(mp=[1.1] * 4), "min_p"), (dict(mp=[math.nan] * 4), "min_p")])
def test_draw_refuses(lib, change, text):
    refused(draw(lib, **change), sb.SPIRAL_ERR_INVALID_ARG, text)


def test_sizes_of_workspaces(lib):
    assert sb.spiral_sample_uniform_workspace_bytes(0, 10) == 0 and sb.spiral_sample_uniform_workspace_bytes(1025, 10) == 0
    assert sb.spiral_sample_uniform_workspace_bytes(1, 0) == 0 and sb.spiral_sample_uniform_workspace_bytes(1024, 151936) > 0
    assert sb.spiral_policy_gradient_workspace_bytes(0, 10) == 0 and sb.spiral_policy_gradient_workspace_bytes(1 << 31, 10) == 0
    assert sb.spiral_policy_gradient_workspace_bytes(5, 0) == 0 and sb.spiral_policy_gradient_workspace_bytes(5, 10) > 0
    assert lib.spiral_adamw_bytes(0) == 0 and lib.spiral_adamw_bytes(-1) == 0 and lib.spiral_adamw_bytes(1) > 0


def grad(lib, **change):
    a = dict(logits=P, dtype=1, ls=100, n=8, V=100, t=P, old=P, adv=P, mask=P, T=1.0, clip=0.2, scale=1.0, logp=P, grad=2 * P, gs=100, ws=P, bytes=1 << 40)
    a.update(change)
    return lib.spiral_policy_gradient(a["logits"], a["dtype"], a["ls"], a["n"], a["V"], a["t"], a["old"], a["adv"], a["mask"], a["T"], a["clip"], a["scale"],
                                      a["logp"], a["grad"], a["gs"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("change,text", [
    (dict(logits=None), "null"), (dict(t=None), "null"), (dict(adv=None), "null"), (dict(logp=None), "null"), (dict(grad=None), "null"),
    (dict(n=0), "n_rows"), (dict(n=1 << 31), "n_rows"), (dict(V=0), "V=0"), (dict(dtype=3), "type"), (dict(ls=99), "stride"), (dict(gs=99), "stride"),
    (dict(logits=P + 1), "misaligned"), (dict(grad=2 * P + 1), "misaligned"), (dict(t=P + 2), "misaligned"), (dict(old=P + 2), "misaligned"),
    (dict(T=0.0), "temperature"), (dict(T=math.inf), "temperature"), (dict(T=math.nan), "temperature"), (dict(clip=-0.1), "clip"),
    (dict(clip=math.nan), "clip"), (dict(scale=math.inf), "scale"), (dict(grad=P, gs=101), "overlaps"), (dict(grad=P + 2), "overlaps"),
    (dict(grad=P + 1598), "overlaps"), (dict(grad=P - 1598), "overlaps"), (dict(ws=None), "workspace"), (dict(ws=P + 8), "workspace"), (dict(bytes=0), "workspace")])
def test_gradient_refuses(lib, change, text):
    refused(grad(lib, **change), sb.SPIRAL_ERR_INVALID_ARG, text)


def record(i=0, **change):
    base = (1 << 30) + (i << 24)
    r = dict(dev_param=base, dev_grad=base + (1 << 16), dev_master=base + (2 << 16), dev_m=base + (3 << 16), dev_v=base + (4 << 16),
             dev_m_scale=None, dev_v_scale=None, n=1000, param_dtype=1, grad_dtype=1, state_dtype=0, decay=1)
    r.update(change)
    return sb.spiral_adamw_tensor_t(**r)


def create(lib, recs, mem=P, nbytes=1 << 20):
    arr = (sb.spiral_adamw_tensor_t * max(1, len(recs)))(*recs)
    out = C.c_void_p(1)
    rc = lib.spiral_adamw_create(arr, len(recs), mem, nbytes, None, C.byref(out))
    assert rc == 0 or not out.value
    return rc


B0 = 1 << 30


@pytest.mark.parametrize("change,text", [
    (dict(param_dtype=3), "unknown type"), (dict(grad_dtype=7), "unknown type"), (dict(state_dtype=1), "unknown type"), (dict(n=0), "0 elements"), (dict(n=-5), "elements"),
    (dict(dev_param=None), "null"), (dict(dev_grad=None), "null"), (dict(dev_m=None), "null"), (dict(dev_v=None), "null"),
    (dict(param_dtype=0), "no master"), (dict(dev_m_scale=P), "scales"), (dict(state_dtype=3), "scales"), (dict(state_dtype=3, dev_m_scale=P), "scales"),
    (dict(decay=2), "decay"), (dict(dev_param=B0 + 1), "misaligned"), (dict(dev_grad=B0 + 65537), "misaligned"), (dict(dev_master=B0 + 131074), "misaligned"),
    (dict(dev_m=B0 + 196610), "misaligned"), (dict(dev_v=B0 + 196608), "overlaps"), (dict(dev_v=B0 + 196608 + 3996), "overlaps"),
    (dict(dev_grad=B0 + 1998), "overlaps"), (dict(dev_master=B0), "overlaps"), (dict(dev_m=P), "overlaps")])
def test_adamw_refuses_tables(lib, change, text):
    refused(create(lib, [record(1), record(0, **change)]), sb.SPIRAL_ERR_INVALID_ARG, text)


def test_adamw_refuses_tensors_that_share_memory_and_bad_memory(lib):
    refused(create(lib, [record(), record()]), sb.SPIRAL_ERR_INVALID_ARG, "overlaps")                       # a tied weight given twice
    refused(create(lib, [record(), record(1, dev_param=B0 + 1024)]), sb.SPIRAL_ERR_INVALID_ARG, "overlaps")
    refused(create(lib, []), sb.SPIRAL_ERR_INVALID_ARG, "no tensors")
    for mem, nbytes in ((None, 1 << 20), (P + 8, 1 << 20), (P, 64)):
        refused(create(lib, [record()], mem, nbytes), sb.SPIRAL_ERR_INVALID_ARG, "memory")
    assert lib.spiral_adamw_create(None, 1, P, 1 << 20, None, C.byref(C.c_void_p())) == sb.SPIRAL_ERR_INVALID_ARG
    assert lib.spiral_adamw_create((sb.spiral_adamw_tensor_t * 1)(record()), 1, P, 1 << 20, None, None) == sb.SPIRAL_ERR_INVALID_ARG


def test_adamw_null_objects(lib):
    assert lib.spiral_adamw_step(None, 1e-3, 0.9, 0.95, 1e-8, 0.0, 1, 1.0, 0.0, None, None) == sb.SPIRAL_ERR_NOT_LOADED
    assert lib.spiral_adamw_set_grads(None, None, None) == sb.SPIRAL_ERR_NOT_LOADED
    lib.spiral_adamw_free(None)


def test_binding_checks_what_it_marshals():
    import torch
    lg, i, f = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    for bad in (dict(dev_logits=lg.t()), dict(dev_logits=lg[:, ::2]), dict(dev_logits=lg[0]), dict(dev_uniform=f[:3]), dict(dev_uniform=i),
                dict(dev_out_tokens=f), dict(dev_out_logp=torch.zeros(4, dtype=torch.float64)), dict(top_k=[1, 2]), dict(temperature=np.ones((4, 1)))):
        a = dict(dev_logits=lg, temperature=None, top_k=None, top_p=None, min_p=None, dev_uniform=f, dev_workspace=None, dev_out_tokens=i, dev_out_logp=f, stream=0)
        a.update(bad)
        with pytest.raises(ValueError):
            sb.spiral_sample_uniform(**a)
    with pytest.raises(TypeError):
        sb.spiral_sample_uniform(lg.double(), None, None, None, None, f, None, i, stream=0)
    for bad in (dict(dev_grad=lg.half()), dict(dev_grad=torch.zeros(4, 9)), dict(dev_targets=f), dict(dev_mask=torch.zeros(4, dtype=torch.bool)), dict(dev_advantage=torch.zeros(5))):
        a = dict(dev_logits=lg, dev_targets=i, dev_logp_old=None, dev_advantage=f, dev_mask=None, temperature=1.0, clip_eps=0.2, scale=1.0, dev_logp=f,
                 dev_grad=lg.clone(), dev_workspace=None, stream=0)
        a.update(bad)
        with pytest.raises(ValueError):
            sb.spiral_policy_gradient(**a)
    n = torch.zeros(300)
    for bad in (dict(grad=n[:299]), dict(m=n[:299]), dict(v=torch.zeros(300, dtype=torch.bfloat16)), dict(m_scale=torch.zeros(3)), dict(param=torch.zeros(600)[::2]),
                dict(master=torch.zeros(300, dtype=torch.float16))):
        a = dict(param=n, grad=n, m=n, v=n)
        a.update(bad)
        with pytest.raises(ValueError):
            sb.spiral_adamw_tensor(**a)


def test_rows_of_the_gradient_are_cut_where_there_are_few_long_ones(lib):
    """The lines of the rule: 96 rows, 16,384 vectors of 16 bytes to a row, slices of 1,024 of them at least."""
    slices = lib["_ZN6spiral18policy_grad_slicesExii"]
    slices.restype, slices.argtypes = C.c_int, [C.c_longlong, C.c_int, C.c_int]
    FP32, BF16, FP16 = sb.SPIRAL_DTYPE_FP32, sb.SPIRAL_DTYPE_BF16, sb.SPIRAL_DTYPE_FP16
    assert slices(1, 65536, FP32) == 16 and slices(1, 65532, FP32) == 1 and slices(1, 131072, BF16) == 16 and slices(1, 131071, FP16) == 1
    assert slices(96, 151936, BF16) == 10 and slices(97, 151936, BF16) == 1 and slices(5, 8209, FP32) == 1
    for n in (1, 7, 96):
        for V in (65536, 151936, 1 << 20, (1 << 31) - 1):
            k = slices(n, V, FP32)
            assert 2 <= k <= max(2, 1024 // n) and V // 4 // k >= 1024
            assert sb.spiral_policy_gradient_workspace_bytes(n, V) >= n * k * 8 + n * 4


@pytest.mark.parametrize("T", [0.0, 1e-31, 1e-39])
def test_gradient_refuses_temperatures_whose_inverse_is_infinite(lib, T):
    refused(grad(lib, T=T), sb.SPIRAL_ERR_INVALID_ARG, "temperature")


Q = 1 << 31                      # far from P


@pytest.mark.parametrize("change", [
    dict(logp=P), dict(logp=P + 12), dict(u=P + (1 << 8) - 12, logp=P + (1 << 8)), dict(out=Q, logp=Q + 12), dict(out=Q + 1596, logp=None), dict(logits=P, u=Q, out=P + 1596, logp=None),
    dict(ws=P), dict(ws=Q), dict(out=2 * Q + 252), dict(logp=2 * Q)])
def test_draw_refuses_outputs_that_are_read(lib, change):
    a = dict(logits=Q, u=P, out=P + 4096, logp=P + 8192, ws=2 * Q)
    a.update(change)
    refused(draw(lib, **a), sb.SPIRAL_ERR_INVALID_ARG, "overlaps")


@pytest.mark.parametrize("change", [
    dict(logp=P), dict(t=Q, logp=Q), dict(adv=Q, logp=Q + 28), dict(mask=Q, logp=Q + 16), dict(logp=2 * Q + 1500), dict(old=2 * Q), dict(t=2 * Q + 1596), dict(logits=2 * Q, logp=2 * Q + 4),
    dict(ws=P), dict(ws=Q, logp=Q), dict(ws=2 * Q), dict(ws=2 * Q + 1536), dict(logits=3 * Q, ws=3 * Q + 256), dict(logp=3 * Q + 100, logits=3 * Q)])
def test_gradient_refuses_outputs_that_are_read(lib, change):
    a = dict(logits=3 * Q + 4096, t=P, old=P, adv=P, mask=P, logp=P + 4096, grad=2 * Q, ws=4 * Q)
    a.update(change)
    refused(grad(lib, **a), sb.SPIRAL_ERR_INVALID_ARG, "overlaps")
