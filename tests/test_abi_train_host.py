"""Host-side tests of the scan's, the label scores' and the update's entry points: every argument error is reported before the HIP runtime is touched."""
import ctypes

import torch

from paper_1805_05225_amd import binding as Bn

P = 0x10000  # an aligned fake device pointer: validation must fail before anything dereferences it
L = Bn.lib
U = lambda: ctypes.byref(ctypes.c_uint64(0))
GPU = torch.cuda.is_available()


def _value(f, *a):
    r = ctypes.c_uint64(0)
    assert f(*a, ctypes.byref(r)) == 0
    return r.value


def test_gated_scan_arguments():
    for gone in range(3):
        assert L.lstm_gated_scan_query(4, 2, 8, *[None if i == gone else U() for i in range(3)]) == -1
    assert Bn.gated_scan_query(1, 768, 1000)[1] == 0 and Bn.gated_scan_query(40000, 1, 64)[1] > 0 and Bn.gated_scan_query(4, 2, 8)[2] > 0
    for T, B, n in ((-1, 2, 8), (4, -1, 8), (4, 2, 0), (4, 70000, 8), (1 << 20, 1 << 15, 8), (4, 1 << 15, 1 << 15), ((1 << 30) + 1, 1, 1), (2 ** 31 - 1, 1, 1), (4, 1, (1 << 27) + 1)):
        assert L.lstm_gated_scan_query(T, B, n, U(), U(), U()) == -2
    base = dict(dt=1, dir=1, T=4, B=2, n=8, z=P, ldz=24, c0=None, lens=None, y=P, ldy=8, cT=None, res=P, rb=1 << 20, ws=P, wb=1 << 20)
    fwd = lambda **o: L.lstm_gated_scan_fwd(*[{**base, **o}[k] for k in base], None)
    base_b = dict(dt=1, dir=1, T=4, B=2, n=8, z=P, ldz=24, lens=None, res=P, rb=1 << 20, dy=P, lddy=8, dcT=None, dz=P, lddz=24, dc0=None, db=None, ws=P, wb=1 << 20)
    bwd = lambda **o: L.lstm_gated_scan_bwd(*[{**base_b, **o}[k] for k in base_b], None)
    assert [fwd(**{k: None}) for k in ("z", "y")] == [-1] * 2 and fwd(T=40000, ws=None) == -1 and [bwd(**{k: None}) for k in ("z", "res", "dy", "dz", "ws")] == [-1] * 5
    for f in (fwd, bwd):
        assert f(T=-1) == -2 and f(B=-1) == -2 and f(n=0) == -2 and f(ldz=23) == -2 and f(dir=0) == -3 and f(dir=2) == -3 and f(dt=2) == -4
        assert f(z=P + 1) == -5 and f(dt=0, z=P + 2) == -5 and f(lens=P + 2) == -5 and f(res=P + 2) == -5
        assert f(rb=1) == -6 and f(T=40000, rb=1 << 30, wb=1) == -6
    assert fwd(ldy=7) == -2 and bwd(lddy=7) == -2 and bwd(lddz=23) == -2 and fwd(c0=P + 2) == -5 and fwd(cT=P + 1) == -5 and bwd(db=P + 2) == -5
    assert fwd(B=0) == 0 and bwd(B=0) == 0
    if not GPU:
        assert fwd() == -7 and bwd() == -7 and fwd(res=None, rb=0) == -7


def test_label_score_arguments():
    q = L.lstm_label_score_query
    assert _value(q, 1, 12, 100000, 5) > 0 and _value(q, 1, 12, 20000, 5) == 0 and _value(q, 80, 64, 20000, 0) == 0 and q(1, 2, 10, 0, None) == -1
    assert q(-1, 2, 10, 0, U()) == -2 and q(1, -2, 10, 0, U()) == -2 and q(1, 2, 0, 0, U()) == -2 and q(1, 2, 10, -1, U()) == -2 and q(1 << 16, 1 << 16, 10, 0, U()) == -2
    assert q(1, 2, 10, 17, U()) == -4 and q(1, 2, (1 << 26) + 1, 0, U()) == -4
    base = dict(dt=0, T=1, B=2, V=10, x=P, ld=10, label=P, lens=None, logp=P, ent=P, lse=P, top=2, tp=P, tl=P, ws=P, wb=1 << 20)
    fwd = lambda **o: L.lstm_label_score_fwd(*[{**base, **o}[k] for k in base], None)
    base_b = dict(dt=0, T=1, B=2, V=10, x=P, ld=10, label=P, lens=None, lse=P, ent=P, dl=P, de=P, dx=P + 4096, ldd=10)
    bwd = lambda **o: L.lstm_label_score_bwd(*[{**base_b, **o}[k] for k in base_b], None)
    assert [fwd(**{k: None}) for k in ("x", "label", "tp", "tl")] == [-1] * 4 and fwd(V=100000, ld=100000, ws=None) == -1 and [bwd(**{k: None}) for k in ("x", "label", "lse", "ent", "dx")] == [-1] * 5
    for f in (fwd, bwd):
        assert f(T=-1) == -2 and f(B=-1) == -2 and f(V=0) == -2 and f(ld=9) == -2 and f(dt=2) == -4 and f(V=(1 << 26) + 1) == -4
        assert f(x=P + 2) == -5 and f(lse=P + 4) == -5 and f(lens=P + 1) == -5 and f(T=0) == 0 and f(B=0) == 0
    assert fwd(top=17) == -4 and fwd(top=-1) == -2 and fwd(V=100000, ld=100000, wb=8) == -6 and bwd(ldd=9) == -2 and bwd(dx=P, ldd=11) == -4 and bwd(de=P + 1) == -5
    if not GPU:
        assert fwd() == -7 and bwd() == -7 and fwd(top=0, tp=None, tl=None, label=None, logp=None) == -7 and bwd(dl=None, label=None, dx=P) == -7


def _items(count=2, **over):
    a = (Bn.AdamwItem * max(count, 1))()
    for it in a:
        it.param = it.grad = it.m = it.v = it.m_scale = it.v_scale = P
        it.count = 100
    for k, v in over.items():
        setattr(a[max(count, 1) - 1], k, v)
    return a


def test_update_arguments():
    q = L.lstm_grad_norm_query
    assert _value(q, 2, _items()) > 0 and q(2, _items(), None) == -1 and q(2, None, U()) == -1 and q(-1, _items(), U()) == -2
    norm = lambda items=None, count=2, mx=1.0, out=P, ws=P, wb=1 << 20: L.lstm_grad_norm(count, items or _items(), mx, out, ws, wb, None)
    assert norm(out=None) == -1 and norm(ws=None) == -1 and norm(_items(grad=None)) == -1
    assert norm(mx=0.0) == -2 and norm(mx=float("nan")) == -2 and norm(mx=-1.0) == -2 and norm(count=-1) == -2
    assert norm(_items(grad_dtype=2)) == -4 and norm(_items(grad=P + 2)) == -5 and norm(out=P + 2) == -5 and norm(wb=8) == -6
    bad = _items()
    bad[1].count = -1
    assert norm(bad) == -2 and norm(count=0, wb=8) == -6

    def step(items=None, count=2, **o):
        d = Bn.AdamwDesc(1e-3, 0.9, 0.999, 1e-8, 1, 0, None, None, None)
        for k, v in o.items():
            setattr(d, k, v)
        return L.lstm_adamw_step(ctypes.byref(d), count, items if items is not None else _items(), None)

    assert L.lstm_adamw_step(None, 2, _items(), None) == -1
    assert [step(_items(**{k: None})) for k in ("param", "grad", "m", "v")] == [-1] * 4
    assert step(_items(m_scale=None), state_dtype=1) == -1 and step(_items(v_scale=None), state_dtype=1) == -1
    assert step(count=-1) == -2 and step(step=0) == -2 and step(lr=-1.0) == -2 and step(lr=float("nan")) == -2 and step(beta1=1.0) == -2
    assert step(beta2=-0.1) == -2 and step(eps=-1.0) == -2 and step(eps=float("inf")) == -2 and step(_items(weight_decay=-1.0)) == -2
    assert step(state_dtype=2) == -4 and step(_items(param_dtype=2)) == -4 and step(_items(grad_dtype=-1)) == -4 and step(_items(reserved=1)) == -4
    assert step(_items(master=P)) == -4                           # a master of a float parameter
    assert step(_items(param=P + 2)) == -5 and step(_items(m=P + 1)) == -5 and step(_items(m_scale=P + 1), state_dtype=1) == -5
    assert step(lr_dev=P + 1) == -5 and step(grad_scale=P + 2) == -5
    if not GPU:
        assert step() == -7 and step(_items(m=P + 1), state_dtype=1) == -7 and step(lr=-1.0, lr_dev=P) == -7 and norm() == -7
