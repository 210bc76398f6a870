"""A training step of a decoder block with the library's operators as they follow each other - norm, projections, head norm and rotation, attention,
residual branches, head, the objective's gradient and all the way back - against a float64 model differentiated by torch, and its log-probabilities
against those that the library's own decoder gives the same tokens."""
import numpy as np
import pytest

from paper_2506_24119_amd import inputs as si

pytestmark = pytest.mark.gpu

# Every tensor that is stored in bf16 is off by at most 2^-8 of each element, 2^-9 on average; a value of the forward pass has at most 12 such tensors behind it, a
# gradient as many more, each rounding adds to the relative 2-norm of the error at most its own 2^-8 (the block's products of random matrices do not amplify it).
FORWARD, GRADIENT = 12 * 2.0 ** -8, 24 * 2.0 ** -8


def close(got, want, bound, what):
    got, want = got.double(), want.double()
    assert torch_norm(got - want) <= bound * torch_norm(want), (what, (torch_norm(got - want) / torch_norm(want)).item())


def torch_norm(t):
    import torch
    return torch.linalg.vector_norm(t)


@pytest.mark.parametrize("hq,hkv,hd,qk_norm", [(8, 2, 64, True), (4, 4, 32, False), (7, 1, 128, True)])
def test_a_training_step_of_a_block(hq, hkv, hd, qk_norm):
    import torch
    from paper_2506_24119_amd import binding as sb
    g = si.ModelGeometry("block", 1, 256, hq, hkv, hd, 512, 2048, 1e6, qk_norm=qk_norm)
    w = sb.weights_to_device(si.make_weights(g, seed=5))
    lw = w["layers"][0]
    lens = [37, 1, 130, 64]
    prompts = [p[:n] for p, n in zip(si.make_prompts(g.vocab, 4, 130, 130, seed=6), lens)]
    n, d = sum(lens), g.d_model
    gen = torch.Generator(device="cuda").manual_seed(7)
    # matrices of a trained size, so that every branch carries weight
    for name in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down"):
        lw[name].copy_((torch.randn(lw[name].shape, device="cuda", generator=gen) / lw[name].shape[1] ** 0.5).bfloat16())
    Wq, Wk, Wv, Wo, Wg, Wu, Wd = (lw[x] for x in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down"))
    g1, g2, g3 = lw["attn_norm"], lw["mlp_norm"], w["final_norm"]
    gq, gk = (lw["q_norm"], lw["k_norm"]) if qk_norm else (None, None)
    for t in (g1, g2, g3, gq, gk):
        if t is not None:
            t.copy_(1 + 0.2 * torch.randn(t.shape, device="cuda", generator=gen))
    tokens = torch.from_numpy(np.concatenate(prompts).astype(np.int64)).cuda()
    targets = torch.cat([torch.cat([t[1:], t.new_full((1,), -1)]) for t in tokens.split(lens)]).int()
    positions = torch.cat([torch.arange(m, device="cuda", dtype=torch.int32) for m in lens])
    adv = torch.randn(n, device="cuda", generator=gen)
    eps, scale = g.rms_eps, 1.0 / hd ** 0.5
    new = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731

    # ---- forward
    x0 = w["embed"][tokens].contiguous()
    W = torch.cat([Wq, Wk, Wv])
    n1, r1 = new(n, d), new(n, dtype=torch.float32)
    sb.spiral_add_rmsnorm(x0, None, g1, eps, n1, None, None, r1)
    qkv = (n1 @ W.t()).unflatten(1, (hq + 2 * hkv, hd))
    q, k, v = qkv.split([hq, hkv, hkv], dim=1)
    qr, kr = new(n, hq, hd), new(n, hkv, hd)
    sb.spiral_norm_rope(q, k, gq, gk, eps, g.rope_theta, positions, qr, kr)
    mem = new(sb.spiral_attention_plan_bytes(lens, hq, hkv, hd), dtype=torch.uint8)
    plan = sb.spiral_attention_plan_create(lens, hq, hkv, hd, mem)
    o, lse = new(n, hq, hd), new(hq, n, dtype=torch.float32)
    sb.spiral_attention_forward(plan, qr, kr, v, scale, o, lse)
    y = o.flatten(1) @ Wo.t()
    s1, n2, r2 = new(n, d), new(n, d), new(n, dtype=torch.float32)
    sb.spiral_add_rmsnorm(y, x0, g2, eps, n2, None, s1, r2)
    gate, up = n2 @ Wg.t(), n2 @ Wu.t()
    act = (torch.nn.functional.silu(gate.float()) * up.float()).bfloat16()
    z = act @ Wd.t()
    s2, n3, r3 = new(n, d), new(n, d), new(n, dtype=torch.float32)
    sb.spiral_add_rmsnorm(z, s1, g3, eps, n3, None, s2, r3)
    logits = n3.float() @ w["lm_head"].float().t()
    logp, dlogits = new(n, dtype=torch.float32), torch.empty_like(logits)
    gws = new(sb.spiral_policy_gradient_workspace_bytes(n, g.vocab), dtype=torch.uint8)
    sb.spiral_policy_gradient(logits, targets, None, adv, None, 1.0, 0.0, 1.0, logp, dlogits, gws)

    # ---- backward
    dl = dlogits.bfloat16()
    grads = {"lm_head": dl.t() @ n3}
    nws = new(sb.spiral_add_rmsnorm_backward_workspace_bytes(n, d), dtype=torch.uint8)
    ds2, dg3 = new(n, d), new(d, dtype=torch.float32)
    sb.spiral_add_rmsnorm_backward(dl @ w["lm_head"], s2, g3, r3, None, ds2, dg3, nws)
    grads.update(final_norm=dg3, w_down=ds2.t() @ act)
    dact = (ds2 @ Wd).float()
    sig = torch.sigmoid(gate.float())
    dgate = (dact * up.float() * sig * (1 + gate.float() * (1 - sig))).bfloat16()
    dup = (dact * gate.float() * sig).bfloat16()
    grads.update(w_gate=dgate.t() @ n2, w_up=dup.t() @ n2)
    ds1, dg2 = new(n, d), new(d, dtype=torch.float32)
    sb.spiral_add_rmsnorm_backward((dgate.float() @ Wg.float() + dup.float() @ Wu.float()).bfloat16(), s1, g2, r2, ds2, ds1, dg2, nws)
    grads.update(mlp_norm=dg2, wo=ds1.t() @ o.flatten(1))
    dqkv = new(n, hq + 2 * hkv, hd)
    dq, dk, dv = dqkv.split([hq, hkv, hkv], dim=1)
    aws = new(sb.spiral_attention_backward_workspace_bytes(plan), dtype=torch.uint8)
    sb.spiral_attention_backward(plan, qr, kr, v, o, lse, (ds1 @ Wo).unflatten(1, (hq, hd)), scale, dq, dk, dv, aws)
    dgq, dgk = (new(hd, dtype=torch.float32), new(hd, dtype=torch.float32)) if qk_norm else (None, None)
    rws = new(sb.spiral_norm_rope_backward_workspace_bytes(n, hq, hkv, hd), dtype=torch.uint8)
    sb.spiral_norm_rope_backward(q, k, dq, dk, gq, gk, eps, g.rope_theta, positions, dq, dk, dgq, dgk, rws)          # in place in the fused gradient
    dqkv = dqkv.flatten(1)
    grads["wqkv"] = dqkv.t() @ n1
    dx0, dg1 = new(n, d), new(d, dtype=torch.float32)
    sb.spiral_add_rmsnorm_backward(dqkv @ W, x0, g1, r1, ds1, dx0, dg1, nws)
    grads.update(attn_norm=dg1, x0=dx0)
    if qk_norm:
        grads.update(q_norm=dgq, k_norm=dgk)
    torch.cuda.synchronize()

    # ---- the same in 64 bits
    leaf = {"x0": x0, "wqkv": W, "wo": Wo, "w_gate": Wg, "w_up": Wu, "w_down": Wd, "lm_head": w["lm_head"], "attn_norm": g1, "mlp_norm": g2, "final_norm": g3}
    if qk_norm:
        leaf.update(q_norm=gq, k_norm=gk)
    L = {name: t.detach().double().clone().requires_grad_() for name, t in leaf.items()}
    rms = lambda t, gain: t * torch.rsqrt((t * t).mean(-1, keepdim=True) + eps) * gain  # noqa: E731
    angle = positions.double()[:, None] * g.rope_theta ** (-2.0 * torch.arange(hd // 2, device="cuda", dtype=torch.float64) / hd)
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    turn = lambda t: torch.cat([t[..., :hd // 2] * c - t[..., hd // 2:] * s, t[..., hd // 2:] * c + t[..., :hd // 2] * s], -1)  # noqa: E731
    h = (rms(L["x0"], L["attn_norm"]) @ L["wqkv"].T).unflatten(1, (hq + 2 * hkv, hd))
    Q, K, V = h.split([hq, hkv, hkv], dim=1)
    if qk_norm:
        Q, K = rms(Q, L["q_norm"]), rms(K, L["k_norm"])
    Q, K = turn(Q), turn(K)
    outs = []
    for a, m in zip(np.cumsum([0] + lens[:-1]), lens):
        row = []
        mask = torch.ones((m, m), dtype=torch.bool, device="cuda").tril()
        for i in range(hq):
            j = i // (hq // hkv)
            p = torch.softmax((Q[a:a + m, i] @ K[a:a + m, j].T * scale).masked_fill(~mask, -np.inf), 1)
            row.append(p @ V[a:a + m, j])
        outs.append(torch.stack(row, 1))
    S1 = L["x0"] + torch.cat(outs).flatten(1) @ L["wo"].T
    N2 = rms(S1, L["mlp_norm"])
    S2 = S1 + (torch.nn.functional.silu(N2 @ L["w_gate"].T) * (N2 @ L["w_up"].T)) @ L["w_down"].T
    LG = rms(S2, L["final_norm"]) @ L["lm_head"].T
    live = targets >= 0
    LP = torch.log_softmax(LG, 1).gather(1, targets.clamp(min=0).long()[:, None])[:, 0]
    loss = -(adv.double() * LP)[live].sum()
    want = dict(zip(L, torch.autograd.grad(loss, list(L.values()))))
    close(logits, LG.detach(), FORWARD, "logits")
    for name, t in want.items():
        close(grads[name], t, GRADIENT, name)

    # ---- the library's decoder on the same weights gives the same tokens the same log-probabilities
    sess = sb.Session(g, w, 64, 4, 16, 256, 192)
    ids = np.arange(4, dtype=np.int32)
    scored = new(n, dtype=torch.float32)
    sb.spiral_score(sess.model, sess.pool, ids, lens, tokens.int(), targets, sess.ws, scored)
    torch.cuda.synchronize()
    spread = LG.detach().std().item()
    assert ((scored - logp).abs()[live].max().item() <= 8 * FORWARD * spread) and (scored[~live] == 0).all()
    sess.close()
    sb.spiral_attention_plan_free(plan)
