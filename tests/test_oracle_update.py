"""The update oracle against closed forms, differences and the library optimiser, on the CPU."""
import numpy as np
import pytest
import torch

from oracle import update as ou


def test_draw_of_hand_worked_rows():
    row = np.log(np.array([1.0, 2.0, 3.0, 4.0]))              # probabilities .1 .2 .3 .4
    for u, tok in ((0.0, 0), (0.05, 0), (0.11, 1), (0.29, 1), (0.31, 2), (0.59, 2), (0.61, 3), (0.999, 3), (1.5, 3), (-1.0, 0), (np.nan, 0)):
        t, lp, _ = ou.draw_row(row, u)
        assert t == tok and abs(lp - np.log((tok + 1) / 10)) < 1e-12
    assert ou.draw_row(row, 0.0, top_k=2)[0] == 2             # 3 and 4 are kept: .43 .57
    assert abs(ou.draw_row(row, 0.5, top_k=2)[1] - np.log(4 / 7)) < 1e-12
    assert ou.draw_row(row, 0.0, top_p=0.6)[0] == 2 and ou.draw_row(row, 0.0, top_p=0.8)[0] == 1
    assert ou.draw_row(row, 0.0, min_p=0.6)[0] == 2 and ou.draw_row(row, 0.0, min_p=1.0)[0] == 3
    assert ou.draw_row(row, 0.9, temperature=0.0)[:2] == (3, 0.0)
    assert ou.draw_row(np.full(3, -np.inf), 0.5)[:2] == (0, -np.inf)
    assert ou.draw_row(np.array([np.nan, 1.0, np.inf, np.inf]), 0.7)[0] == 3
    flat = np.zeros(8)
    assert ou.draw_row(flat, 0.99, top_k=2)[0] == 7           # equal logits stay together


def test_top_p_groups_agree_with_a_walk():
    rng = np.random.default_rng(0)
    for V in (5, 50, 400):
        row = np.round(rng.normal(size=V) * 3) / 2
        w = np.exp(row - row.max())
        for p in (0.3, 0.9):
            order = np.argsort(-row, kind="stable")
            c = w[order].cumsum()
            tau = row[order][int(np.argmax(c >= float(np.float32(p)) * c[-1]))]
            kept = np.flatnonzero(row >= tau)
            assert ou.draw_row(row, 0.0, top_p=p)[0] == kept[0] and ou.draw_row(row, 0.9999999, top_p=p)[0] == kept[-1]


@pytest.mark.parametrize("with_old", [True, False])
def test_policy_gradient_agrees_with_differences(with_old):
    rng = np.random.default_rng(1)
    n, V, T, scale = 6, 11, 0.7, 0.3
    z = rng.normal(size=(n, V)) * 2
    y, A, mask = rng.integers(0, V, n), rng.normal(size=n), np.array([1, 1, 0, 1, 1, 1])
    y[4] = -1
    old = ou.objective(z, y, None, A, None, T, 0.0)[1] + rng.normal(size=n) * 0.4 if with_old else None
    _, grad, _, _ = ou.policy_gradient(z, y, old, A, mask, T, 0.2, scale)
    h = 1e-6
    for t in range(n):
        for v in range(V):
            up, down = z.copy(), z.copy()
            up[t, v] += h
            down[t, v] -= h
            d = (ou.objective(up, y, old, A, mask, T, 0.2)[0] - ou.objective(down, y, old, A, mask, T, 0.2)[0]) / (2 * h)
            assert abs(-scale * d - grad[t, v]) < 1e-8
    assert (grad[2] == 0).all() and (grad[4] == 0).all()


def test_adamw_agrees_with_the_library_optimiser():
    rng = np.random.default_rng(2)
    p = [torch.nn.Parameter(torch.from_numpy(rng.normal(size=s))) for s in (7, 300)]
    opt = torch.optim.AdamW(p, lr=0.01, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    state = [{"p": q.detach().numpy().copy(), "m": np.zeros(q.numel()), "v": np.zeros(q.numel()), "decay": 1} for q in p]
    for step in range(1, 6):
        for q, s in zip(p, state):
            s["g"] = rng.normal(size=q.numel()) * 3
            q.grad = torch.from_numpy(s["g"].copy()) * 0.5
        total = torch.nn.utils.clip_grad_norm_(p, 1.0)
        opt.step()
        out, norm = ou.adamw(state, 0.01, 0.9, 0.95, 1e-8, 0.1, step, grad_scale=0.5, max_norm=1.0)
        assert abs(norm - total.item()) < 1e-12 * norm
        for s, o, q in zip(state, out, p):
            s.update(p=o["p"], m=o["m"], v=o["v"])
            assert np.abs(o["p"] - q.detach().numpy()).max() < 2e-8          # its clip divides by the norm + 1e-6


def test_e4m3_values_are_torchs():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    got = ou.e4m3_value(codes.numpy())
    assert np.array_equal(np.isnan(want), np.isnan(got)) and np.array_equal(want[~np.isnan(want)], got[~np.isnan(got)])
    x = np.linspace(-448, 448, 4001)
    v = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert (np.abs(v - x) <= ou.encode_off_by(x, np.ones_like(x)) * (1 + 1e-12)).all()
