"""A training step as a user runs it: an LSTM layer, a gated scan above it, the output layer, label scores, the gradients of all of them, the clipped
AdamW step - against the same network in double precision (torch autograd on the CPU), two steps in a row, float storage.

Tolerance: 1e-4 of a gradient's largest magnitude against double precision, the tolerance of the products and of the layers; the update is compared with
the formula applied to the gradients that the GPU gave, since a first step's size does not depend on a gradient's, only on its sign."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import train_oracle as R
from tests.gpu_util import check, host

T, B, NI, N, V = 23, 5, 12, 20, 37
LENS = [23, 1, 0, 17, 9]


def _network(P, x, lens, labels, weight):
    """The loss in double precision."""
    n = N
    h, c = torch.zeros(B, n, dtype=torch.float64), torch.zeros(B, n, dtype=torch.float64)
    s, loss = torch.zeros(B, n, dtype=torch.float64), 0.0
    for t in range(T):
        ok = (t < lens)[:, None]
        z = x[t] @ P["Wx"] + h @ P["Wh"] + P["b"]
        i, f, g, o = z.chunk(4, 1)
        c2 = torch.sigmoid(f) * c + torch.sigmoid(i) * torch.tanh(g)
        h2 = torch.sigmoid(o) * torch.tanh(c2)
        c, h = torch.where(ok, c2, c), torch.where(ok, h2, h)
        zf, zg, zo = (h2 @ P["Ws"] + P["bs"]).chunk(3, 1)
        s2 = torch.sigmoid(zf) * s + torch.sigmoid(-zf) * torch.tanh(zg)
        s = torch.where(ok, s2, s)
        q = torch.log_softmax((torch.sigmoid(zo) * s2) @ P["Wo"].T + P["bo"], 1)
        ent = -(q.exp() * q).sum(1)
        each = weight * q[torch.arange(B), labels[t]] + 0.1 * weight * ent
        loss = loss + torch.where(ok[:, 0], each, torch.zeros_like(each)).sum()
    return loss


def _gradients(Bn, P, x, lens, labels, weight):
    """The same loss's gradient through the library."""
    f = Bn.forward(x, P["Wx"], P["Wh"], P["b"], None, None, lens, bidirectional=False)
    y1 = f["y"]
    z = Bn.gemm(y1.view(T * B, N), P["Ws"], a_kcontig=True, b_kcontig=False, M=T * B, N=3 * N, K=N, bias=P["bs"]).view(T, B, 3 * N)
    s = Bn.gated_scan_fwd(z, None, lens)
    y2 = s["y"].view(T * B, N)
    logits = Bn.gemm(y2, P["Wo"], a_kcontig=True, b_kcontig=True, M=T * B, N=V, K=N, bias=P["bo"]).view(T, B, V)
    score = Bn.label_score_fwd(logits, labels, lens)
    w = torch.full((T, B), weight, device="cuda")
    loss = (score["logp"] * w + 0.1 * w * score["entropy"]).double().sum()
    d = Bn.label_score_bwd(score, logits, labels, w, 0.1 * w, lens, out=logits).view(T * B, V)
    ones = torch.ones(T * B, 1, device="cuda")
    G = dict(Wo=Bn.gemm(d, y2, a_kcontig=False, b_kcontig=False, M=V, N=N, K=T * B),
             bo=Bn.gemm(ones, d, a_kcontig=False, b_kcontig=False, M=1, N=V, K=T * B).view(V))
    dy2 = Bn.gemm(d, P["Wo"], a_kcontig=True, b_kcontig=False, M=T * B, N=N, K=V).view(T, B, N)
    g = Bn.gated_scan_bwd(s, z, dy2, lens)
    dz = g["dz"].view(T * B, 3 * N)
    G["Ws"] = Bn.gemm(y1.view(T * B, N), dz, a_kcontig=False, b_kcontig=False, M=N, N=3 * N, K=T * B, lens=lens, Bt=B, T=T)
    G["bs"] = g["db"]
    dy1 = Bn.gemm(dz, P["Ws"], a_kcontig=True, b_kcontig=True, M=T * B, N=N, K=3 * N).view(T, B, N)
    b = Bn.backward(f, x, P["Wx"], P["Wh"], None, None, lens, dy1, want_dx=False, want_dstate=False)
    G["Wx"], G["Wh"], G["b"] = b["dW_x"], b["dW_h"], b["db"]
    assert not Bn.sync_status(f["workspace"])
    return loss, G


@pytest.mark.parametrize("bits", [32, 8])
def test_two_training_steps(bits):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1805_05225_amd import binding as Bn
    rng = np.random.default_rng(31)
    rnd = lambda *s: torch.from_numpy(rng.uniform(-.3, .3, s).astype(np.float32))
    shapes = dict(Wx=(NI, 4 * N), Wh=(N, 4 * N), b=(4 * N,), Ws=(N, 3 * N), bs=(3 * N,), Wo=(V, N), bo=(V,))
    P = {k: rnd(*s).cuda() for k, s in shapes.items()}
    x = torch.from_numpy(rng.standard_normal((T, B, NI)).astype(np.float32))
    lens, labels = torch.tensor(LENS, dtype=torch.int32), torch.from_numpy(rng.integers(0, V, (T, B)).astype(np.int32))
    weight, names = -1.0 / sum(LENS), list(shapes)
    state = Bn.adamw_state([P[k] for k in names], bits)
    decay = [0.0 if k.startswith("b") else 0.02 for k in names]
    for step in (1, 2):
        D = {k: P[k].double().cpu().requires_grad_() for k in names}
        ref = _network(D, x.double(), lens, labels.long(), weight)
        ref.backward()
        loss, G = _gradients(Bn, P, x.cuda(), lens.cuda(), labels.cuda(), weight)
        print("  training step %d, %d bits: loss %.6f" % (step, bits, loss.item()), flush=True)
        assert abs(loss.item() - ref.item()) < 1e-5 * abs(ref.item())
        for k in names:
            check(k, G[k], D[k].grad.numpy(), 1e-4)
        before, grads = {k: host(P[k]).reshape(-1) for k in names}, {k: host(G[k]).reshape(-1) for k in names}
        mv = []
        for i, k in enumerate(names):
            m, v = (state[q][i].double().cpu().numpy().reshape(-1) for q in ("m", "v"))
            if bits == 8:
                m = m * R.spread(host(state["m_scale"][i]), m.size)
                v = (v * R.spread(host(state["v_scale"][i]), v.size)) ** 2
            mv.append((m, v))
        norm = Bn.grad_norm([G[k] for k in names], 0.05)
        Bn.adamw_step([P[k] for k in names], [G[k] for k in names], lr=1e-2, step=step, weight_decay=decay, grad_scale=norm[1:], **state)
        total, clip = R.grad_norm(list(grads.values()), 0.05)
        assert abs(norm[0].item() - total) < 1e-6 * total and abs(norm[1].item() - clip) < 1e-6 and clip < 1
        for i, k in enumerate(names):
            want, _, _ = R.adamw(before[k], grads[k], *mv[i], step, 1e-2, decay=decay[i], scale=float(np.float32(norm[1].item())))
            assert np.abs(host(P[k]).reshape(-1) - want).max() < 2e-6, k            # 2^-24 of a weight of 0.3, and 16 roundings of a step of 0.01
