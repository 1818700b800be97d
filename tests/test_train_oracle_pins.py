"""Pins of oracle/train_oracle.py: against torch's double-precision autograd, against differences, and against torch's 8-bit type."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as R


def _scan_torch(z, c0, lens, direction):
    T, B, n = z.shape[0], z.shape[1], z.shape[2] // 3
    c, y = c0, [None] * T
    for t in (range(T) if direction > 0 else range(T - 1, -1, -1)):
        ok = (t < lens)[:, None]
        f = torch.sigmoid(z[t, :, :n])
        new = f * c + (1 - f) * torch.tanh(z[t, :, n:2 * n])
        c = torch.where(ok, new, c)
        y[t] = torch.where(ok, torch.sigmoid(z[t, :, 2 * n:]) * new, torch.zeros_like(new))
    return torch.stack(y), c


@pytest.mark.parametrize("direction", [1, -1])
def test_gated_scan_is_autograds(direction):
    rng = np.random.default_rng(3)
    T, B, n = 7, 5, 4
    lens = np.array([7, 0, 1, 4, 6])
    leaf = lambda *s: torch.tensor(rng.standard_normal(s), requires_grad=True)
    z, c0 = leaf(T, B, 3 * n), leaf(B, n)
    dy, dcT = rng.standard_normal((T, B, n)), rng.standard_normal((B, n))
    y, cT = _scan_torch(z, c0, torch.tensor(lens), direction)
    ((y * torch.tensor(dy)).sum() + (cT * torch.tensor(dcT)).sum()).backward()
    yo, co, _ = R.gated_scan_fwd(z.detach().numpy(), c0.detach().numpy(), lens, direction)
    dz, dc0, db = R.gated_scan_bwd(z.detach().numpy(), dy, c0.detach().numpy(), lens, dcT, direction)
    for a, b in ((yo, y), (co, cT)):
        np.testing.assert_allclose(a, b.detach().numpy(), atol=1e-13)
    np.testing.assert_allclose(dz, z.grad.numpy(), atol=1e-13)
    np.testing.assert_allclose(dc0, c0.grad.numpy(), atol=1e-13)
    np.testing.assert_allclose(db, z.grad.sum((0, 1)).numpy(), atol=1e-12)


def test_gated_scan_gradient_by_differences():
    rng = np.random.default_rng(4)
    z, dy, lens = rng.standard_normal((5, 2, 6)), rng.standard_normal((5, 2, 2)), np.array([5, 3])
    dz = R.gated_scan_bwd(z, dy, None, lens)[0]
    value = lambda q: (R.gated_scan_fwd(q, None, lens)[0] * dy).sum()
    for at in [(0, 0, 0), (2, 1, 3), (4, 0, 5), (4, 1, 1), (1, 0, 2)]:
        d = np.zeros_like(z)
        d[at] = 1e-5
        assert abs((value(z + d) - value(z - d)) / 2e-5 - dz[at]) < 1e-9


def test_label_score_is_autograds():
    rng = np.random.default_rng(5)
    T, B, V = 3, 4, 9
    lens, label = np.array([3, 1, 0, 2]), rng.integers(0, V, (T, B))
    label[0, 0] = -1
    x = torch.tensor(rng.standard_normal((T, B, V)) * 2, requires_grad=True)
    wl, we = rng.standard_normal((T, B)), rng.standard_normal((T, B))
    q = torch.log_softmax(x, -1)
    ok = torch.arange(T)[:, None] < torch.tensor(lens)
    logp = q.gather(2, torch.tensor(label).clamp(min=0)[:, :, None])[:, :, 0] * ok * torch.tensor(label >= 0)
    ent = -(q.exp() * q).sum(-1) * ok
    ((logp * torch.tensor(wl)).sum() + (ent * torch.tensor(we)).sum()).backward()
    f = R.label_score_fwd(x.detach().numpy(), label, lens, top=4)
    np.testing.assert_allclose(f["logp"], logp.detach().numpy(), atol=1e-13)
    np.testing.assert_allclose(f["entropy"], ent.detach().numpy(), atol=1e-13)
    np.testing.assert_allclose(R.label_score_bwd(x.detach().numpy(), label, wl, we, lens), x.grad.numpy(), atol=1e-13)
    best = q.detach().topk(4, -1)
    np.testing.assert_allclose(f["top_logp"][ok.numpy()], best.values.numpy()[ok.numpy()], atol=1e-13)
    assert np.array_equal(f["top_label"][ok.numpy()], best.indices.numpy()[ok.numpy()])


def test_label_score_of_rows_with_little_left():
    inf = np.inf
    x = np.array([[[-inf, -inf, -inf], [1.0, -inf, 1.0], [0.0, np.nan, 1.0], [0.0, inf, 1.0]]])
    f = R.label_score_fwd(x, np.array([[0, 1, 0, 1]]), top=3)
    assert f["lse"][0, 0] == -inf and f["logp"][0, 0] == -inf and f["entropy"][0, 0] == 0
    assert f["logp"][0, 1] == -inf and abs(f["entropy"][0, 1] - np.log(2)) < 1e-15
    assert f["top_label"][0, 1].tolist() == [0, 2, 0] and f["top_logp"][0, 1, 2] == -inf
    assert np.isnan(f["logp"][0, 2:]).all() and (f["top_logp"][0, 2:] == -inf).all()
    d = R.label_score_bwd(x, np.array([[0, 2, 0, -1]]), np.ones((1, 4)), np.zeros((1, 4)))
    assert (d[0, 0] == 0).all() and np.allclose(d[0, 1], [-0.5, 0, 0.5]) and np.isnan(d[0, 2]).all() and (d[0, 3] == 0).all()


def test_8_bit_values_are_torchs():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes, R.values8())
    x = np.random.default_rng(6).uniform(-448, 448, 20000).astype(np.float32)
    x = np.concatenate([x, x * 1e-3, x * 1e-5, codes[1:] * 1.0, (codes[1:] + codes[:-1]) / 2]).astype(np.float32)
    assert np.array_equal(R.to8(x), torch.tensor(x).to(torch.float8_e4m3fn).double().numpy())


def test_adamw_is_torchs():
    rng = np.random.default_rng(7)
    w, grads = rng.standard_normal(50), rng.standard_normal((4, 50))
    p = torch.tensor(w, requires_grad=True)
    opt = torch.optim.AdamW([p], lr=3e-2, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    m, v = np.zeros(50), np.zeros(50)
    for k, g in enumerate(grads):
        p.grad = torch.tensor(g)
        opt.step()
        w, m, v = R.adamw(w, g, m, v, k + 1, 3e-2, 0.8, 0.95, 1e-6, 0.1)
    np.testing.assert_allclose(w, p.detach().numpy(), atol=1e-13)
    norm, scale = R.grad_norm(list(grads), 2.0)
    assert abs(norm - np.sqrt((grads ** 2).sum())) < 1e-12 and abs(scale - 2.0 / norm) < 1e-15
