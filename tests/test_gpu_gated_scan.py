"""GPU parity of the gated linear recurrence (lstm_gated_scan_fwd / _bwd through the binding) against oracle/train_oracle.py.

Tolerances.  A gate is off by at most (|z| + 8) 2^-24 of min(f, 1 - f): the rounding of the exponent's argument, and a few roundings of
exp2, reciprocal and products.  A state's recurrence adds one rounding of 2^-24 |c| per frame and forgets it at the rate 1 - f: with |z_f| <= 7
(1 - f >= 2^-10) an error stays below (2^10 + |z| + 8) 2^-24 = 6.3e-5 of the largest state.  So 1e-4 of the largest magnitude holds for float
results, the tolerance of the layers; a bfloat16 result is off by half a step, 2^-8 of itself, more.  db sums N values that are each
off by that much: 1e-4 of the sum of the magnitudes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import train_oracle as R
from tests.gpu_util import dev, host, tdtype

Bn = None


@pytest.fixture(scope="module", autouse=True)
def _binding():
    global Bn
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1805_05225_amd import binding
    Bn = binding
    yield


def _near(name, got, ref, dt, scale=None):
    got = host(got)
    assert got.shape == ref.shape and np.isfinite(got).all(), name
    tol = 1e-4 * (np.abs(ref).max() if scale is None else scale) + (2.0 ** -8 * np.abs(ref) if dt == "bf16" else 0) + 1e-30
    assert (np.abs(got - ref) <= tol).all(), (name, float((np.abs(got - ref) / tol).max()))


def _inputs(T, B, n, dt, seed, lens):
    rng = np.random.default_rng(seed)
    rnd = lambda a: torch.from_numpy(a.astype(np.float32)).to(tdtype(dt)).float().numpy()
    z = rng.standard_normal((T, B, 3 * n))
    z[:, :, :n] = np.clip(z[:, :, :n] * 1.5 + 2, -7, 7)
    if lens == "ragged":
        lens = rng.integers(0, T + 1, B)
        lens[0] = T
        if B > 2:
            lens[1], lens[2] = 0, 1
    f32 = lambda *s: rng.standard_normal(s).astype(np.float32)
    return rnd(z), rnd(rng.standard_normal((T, B, n))), f32(B, n), f32(B, n), None if lens is None else np.asarray(lens, dtype=np.int32)


def _compare(T, B, n, dt, direction, lens, seed=0, state=True):
    z, dy, c0, dcT, L = _inputs(T, B, n, dt, seed, lens)
    print("  scan T=%d B=%d n=%d %s direction %d" % (T, B, n, dt, direction), flush=True)
    if not state:
        c0 = dcT = None
    yo, co, _ = R.gated_scan_fwd(z, c0, L, direction)
    dzo, dco, dbo = R.gated_scan_bwd(z, dy, c0, L, dcT, direction)
    if L is not None:                                            # whatever padded frames hold must not reach a result
        pad = np.arange(T)[:, None] >= L[None, :]
        z, dy = np.where(pad[:, :, None], np.nan, z), np.where(pad[:, :, None], np.nan, dy)
    zt, dyt = dev(z, dt), dev(dy, dt)
    f = Bn.gated_scan_fwd(zt, dev(c0), dev(L), direction=direction)
    g = Bn.gated_scan_bwd(f, zt, dyt, dev(L), dev(dcT))
    torch.cuda.synchronize()
    _near("y", f["y"], yo, dt)
    _near("cT", f["cT"], co, "f32")
    _near("dz", g["dz"], dzo, dt)
    _near("dc0", g["dc0"], dco, "f32", max(np.abs(dco).max(initial=0), np.abs(dy[np.isfinite(dy)]).max(initial=0)))
    _near("db", g["db"], dbo, "f32", np.abs(dzo).sum((0, 1)) + 1e-12)
    inf = Bn.gated_scan_fwd(zt, dev(c0), dev(L), direction=direction, save=False)
    assert torch.equal(inf["y"], f["y"]) and torch.equal(inf["cT"], f["cT"]) and inf["reserve"] is None


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("direction", [1, -1])
@pytest.mark.parametrize("T,B,n", [(1, 1, 1), (1, 37, 130), (2, 3, 64), (15, 2, 5), (16, 4, 128), (17, 5, 66), (33, 3, 7), (129, 4, 200), (130, 2, 1000),
                                   (257, 9, 33)])
def test_scan_shapes(T, B, n, dt, direction):
    _compare(T, B, n, dt, direction, "ragged", seed=T + n)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,n,direction", [(3000, 1, 96, 1), (5001, 1, 130, -1), (2049, 2, 258, 1), (1030, 3, 64, -1), (16500, 1, 130, -1)])
def test_scan_long(T, B, n, direction, dt):
    _compare(T, B, n, dt, direction, None, seed=7)
    _compare(T, B, n, dt, direction, "ragged", seed=8)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,n,direction", [(129, 140, 70, 1), (600, 300, 66, -1), (1500, 130, 20, 1)])
def test_scan_of_many_rows(T, B, n, direction, dt):
    _compare(T, B, n, dt, direction, "ragged", seed=17)
    _compare(T, B, n, dt, direction, None, seed=18, state=False)


def test_scan_without_state_and_with_odd_lengths():
    _compare(40, 4, 70, "bf16", 1, [-3, 0, 40, 99], state=False)         # lengths are clamped to [0, T]
    _compare(40, 4, 70, "f32", -1, None, state=False)


def test_scan_of_nothing():
    """T = 0: the state passes through; B = 0: no rows, db = 0."""
    c0, dcT = torch.randn(3, 8, device="cuda"), torch.randn(3, 8, device="cuda")
    z = torch.empty(0, 3, 24, device="cuda")
    f = Bn.gated_scan_fwd(z, c0)
    g = Bn.gated_scan_bwd(f, z, torch.empty(0, 3, 8, device="cuda"), None, dcT)
    assert torch.equal(f["cT"], c0) and torch.equal(g["dc0"], dcT) and not g["db"].any() and g["db"].numel() == 24
    z = torch.empty(5, 0, 24, device="cuda")
    f = Bn.gated_scan_fwd(z)
    g = Bn.gated_scan_bwd(f, z, torch.empty(5, 0, 8, device="cuda"))
    assert g["dz"].shape == (5, 0, 24) and not g["db"].any()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("shift,extra", [(0, 2), (1, 0), (1, 3), (2, 6)])
def test_scan_rows_at_any_element(dt, shift, extra):
    """z, dy, y and dz as parts of wider rows: what lies between the rows stays as it was."""
    T, B, n = 21, 3, 34
    z, dy, c0, dcT, L = _inputs(T, B, n, dt, 5, "ragged")

    def wide(a, F):
        full = torch.full((T, B, F + extra + shift), 7.0, dtype=tdtype(dt), device="cuda")
        view = full[:, :, shift:shift + F]
        if a is not None:
            view.copy_(dev(a, dt))
        return full, view

    (_, zt), (_, dyt), (yw, yt), (dzw, dzt) = wide(z, 3 * n), wide(dy, n), wide(None, n), wide(None, 3 * n)
    f = Bn.gated_scan_fwd(zt, dev(c0), dev(L), out=yt)
    g = Bn.gated_scan_bwd(f, zt, dyt, dev(L), dev(dcT), out=dzt)
    p = Bn.gated_scan_fwd(dev(z, dt), dev(c0), dev(L))
    q = Bn.gated_scan_bwd(p, dev(z, dt), dev(dy, dt), dev(L), dev(dcT))
    assert f["y"].data_ptr() == yt.data_ptr() and torch.equal(yt, p["y"]) and torch.equal(dzt, q["dz"])
    assert torch.equal(f["cT"], p["cT"]) and torch.equal(g["dc0"], q["dc0"])
    _near("db", g["db"], host(q["db"]), "f32")
    for full, F in ((yw, n), (dzw, 3 * n)):
        assert (full[:, :, :shift] == 7).all() and (full[:, :, shift + F:] == 7).all()


def test_scan_two_directions_side_by_side():
    """Both directions into the halves of one output, as a bidirectional layer's."""
    T, B, n = 30, 4, 48
    z0, _, _, _, L = _inputs(T, B, n, "bf16", 1, "ragged")
    z1 = _inputs(T, B, n, "bf16", 2, None)[0]
    y = torch.empty(T, B, 2 * n, dtype=torch.bfloat16, device="cuda")
    Bn.gated_scan_fwd(dev(z0, "bf16"), None, dev(L), direction=1, out=y[:, :, :n])
    Bn.gated_scan_fwd(dev(z1, "bf16"), None, dev(L), direction=-1, out=y[:, :, n:])
    ref = np.concatenate([R.gated_scan_fwd(z0, None, L, 1)[0], R.gated_scan_fwd(z1, None, L, -1)[0]], axis=2)
    _near("y", y, ref, "bf16")


@pytest.mark.parametrize("T,B,n", [(1, 96, 200), (50, 2, 64), (4000, 1, 64), (300, 140, 40)])
def test_scan_carries_its_state_in_place(T, B, n):
    """cT = c0: the state of a text that arrives in pieces, one array; pieces give what the whole gives."""
    z = _inputs(2 * T, B, n, "f32", 9, None)[0]
    zt, state = dev(z, "f32"), torch.zeros(B, n, device="cuda")
    y = torch.empty(2 * T, B, n, device="cuda")
    ws = torch.empty(Bn.gated_scan_query(T, B, n)[1] + 1, dtype=torch.uint8, device="cuda")
    for k in range(2):
        part, out = zt[k * T:(k + 1) * T], y[k * T:(k + 1) * T]
        rc = Bn.lib.lstm_gated_scan_fwd(0, 1, T, B, n, part.data_ptr(), 3 * n, state.data_ptr(), None, out.data_ptr(), n, state.data_ptr(), None, 0,
                                        ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
        assert rc == 0
    yo, co, _ = R.gated_scan_fwd(z)
    _near("y", y, yo, "f32")
    _near("cT", state, co, "f32")


def test_scan_saturated_gates_and_large_values():
    """Gates of 0 and 1 to the last bit, infinities among the pre-activations (sigmoid and tanh have limits there), a NaN that stays in its unit."""
    T, B, n = 20, 1, 64
    z = np.random.default_rng(3).standard_normal((T, B, 3 * n)).astype(np.float32) * 3
    z[3, 0, :8], z[4, 0, :8], z[5, 0, 8:16], z[6, 0, n:n + 8] = 200, -200, np.inf, -np.inf
    z[7, 0, 2 * n:2 * n + 8] = -np.inf
    dy = np.ones((T, B, n), dtype=np.float32)
    yo, co, _ = R.gated_scan_fwd(z)
    dzo, _, _ = R.gated_scan_bwd(z, dy)
    zt = dev(z, "f32")
    f = Bn.gated_scan_fwd(zt)
    g = Bn.gated_scan_bwd(f, zt, dev(dy, "f32"))
    _near("y", f["y"], yo, "f32")
    _near("dz", g["dz"], dzo, "f32")
    z[2, 0, n + 5] = np.nan
    h = Bn.gated_scan_fwd(dev(z, "f32"))["y"]
    assert torch.isnan(h[2:, 0, 5]).all() and torch.isfinite(h[:2, 0, 5]).all()
    other = [i for i in range(n) if i != 5]
    assert torch.equal(h[:, 0, other], f["y"][:, 0, other])


@pytest.mark.parametrize("size", [1e-1, 1e-3, 1e-6])
def test_scan_keeps_the_digits_of_small_values(size):
    """States of positive candidates of one size, in float storage: no sum cancels, so every state keeps its digits.  A gate is off by (|z_f| + 8) 2^-24 of itself (and
    of 1 - f), |z_f| <= 2 here; a candidate by 8 2^-24 of itself: of 2^-23 where tanh is at least 1/4, otherwise by the series' eight roundings.  Each is made
    once a frame and remembered over all T of them at most: (10 + 10 + 8 + 2) T 2^-24, and y 12 2^-24 more."""
    T, B, n = 60, 3, 130
    rng = np.random.default_rng(5)
    z = np.clip(rng.standard_normal((T, B, 3 * n)), -2, 2).astype(np.float32)
    z[:, :, n:2 * n] = (rng.uniform(0.2, 4, (T, B, n)) * size).astype(np.float32)
    y, c, _ = R.gated_scan_fwd(z)
    f = Bn.gated_scan_fwd(dev(z, "f32"))
    for got, ref in ((host(f["y"]), y), (host(f["cT"]), c)):
        assert (np.abs(got - ref) <= (30 * T + 12) * 2.0 ** -24 * np.abs(ref)).all(), float((np.abs(got - ref) / np.abs(ref)).max())
    one = Bn.gated_scan_fwd(dev(z[:1], "f32"), save=False)
    assert (np.abs(host(one["y"]) - y[:1]) <= 42 * 2.0 ** -24 * np.abs(y[:1])).all()


@pytest.mark.parametrize("T,B,n", [(300, 2, 256), (3000, 2, 64), (500, 130, 64)])
def test_scan_repeats_its_bits_on_any_stream_and_in_a_graph(T, B, n):
    z, dy, c0, dcT, L = _inputs(T, B, n, "bf16", 4, "ragged")
    zt, dyt, ct, dct, Lt = dev(z, "bf16"), dev(dy, "bf16"), dev(c0), dev(dcT), dev(L)
    run = lambda: (lambda f: (f["y"], f["cT"], *Bn.gated_scan_bwd(f, zt, dyt, Lt, dct).values()))(Bn.gated_scan_fwd(zt, ct, Lt, direction=-1))
    first = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for k in range(3):
        zt.copy_(dev(np.roll(z, k, axis=1), "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        now = run()
        assert all(torch.equal(a, b) for a, b in zip(held, now))
    zt.copy_(dev(z, "bf16"))
    assert all(torch.equal(a, b) for a, b in zip(first, second)) and all(torch.equal(a, b) for a, b in zip(first, run()))


def test_scan_behind_32_bit_offsets():
    """The last rows of 4.3e9 pre-activations have the bits of a call of their own; the last frames of a text of 2.4e9 those of one that begins 3000 frames before
    the end, up to what compositions round: with f <= sigmoid(1) nothing is left of a state after that, and a frame's roundings add up to 20 2^-24 / (1 - f) of the largest."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *shape: torch.empty(*shape, dtype=torch.bfloat16, device="cuda").uniform_(-1, 1, generator=gen)
    z, dy = rnd(3, 60000, 24000), rnd(3, 60000, 8000)
    f = Bn.gated_scan_fwd(z)
    g = Bn.gated_scan_bwd(f, z, dy, want_db=False)
    own = Bn.gated_scan_fwd(z[:, -2:].contiguous())
    own_g = Bn.gated_scan_bwd(own, z[:, -2:].contiguous(), dy[:, -2:].contiguous(), want_db=False)
    assert torch.equal(f["y"][:, -2:], own["y"]) and torch.equal(f["cT"][-2:], own["cT"])
    assert torch.equal(g["dz"][:, -2:], own_g["dz"]) and torch.equal(g["dc0"][-2:], own_g["dc0"])
    del z, dy, f, g
    z, dy = rnd(800000, 1, 3000), rnd(800000, 1, 1000)
    f = Bn.gated_scan_fwd(z)
    g = Bn.gated_scan_bwd(f, z, dy)
    own = Bn.gated_scan_fwd(z[-3000:])
    own_g = Bn.gated_scan_bwd(own, z[-3000:], dy[-3000:])
    tol = 20 * 2.0 ** -24 / (1 - 0.7311)
    assert ((f["cT"] - own["cT"]).abs() <= tol).all()
    for a, b, most in ((f["y"], own["y"], 1.0), (g["dz"], own_g["dz"], 4.0)):
        a, b = a[-1000:].float(), b[-1000:].float()
        assert ((a - b).abs() <= 2.0 ** -7 * b.abs() + most * tol).all()             # (two roundings to bfloat16)


def test_scan_refuses_what_it_cannot_take():
    z = torch.zeros(4, 2, 24, device="cuda")
    with pytest.raises(AssertionError):
        Bn.gated_scan_fwd(z.cpu())
    with pytest.raises(AssertionError):
        Bn.gated_scan_fwd(z.half())
    with pytest.raises(AssertionError):
        Bn.gated_scan_fwd(z[:, :, :23])
    with pytest.raises(AssertionError):
        Bn.gated_scan_fwd(z.transpose(0, 1))
    with pytest.raises(AssertionError):
        Bn.gated_scan_fwd(z, torch.zeros(2, 7, device="cuda"))
    with pytest.raises(AssertionError):
        Bn.gated_scan_fwd(z, None, torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(AssertionError):
        Bn.gated_scan_fwd(z, out=torch.zeros(4, 2, 8, dtype=torch.bfloat16, device="cuda"))
    f = Bn.gated_scan_fwd(z)
    with pytest.raises(AssertionError):
        Bn.gated_scan_bwd(f, z, torch.zeros(4, 2, 9, device="cuda"))
    with pytest.raises(TypeError):
        Bn.gated_scan_bwd(Bn.gated_scan_fwd(z, save=False), z, torch.zeros(4, 2, 8, device="cuda"))
    for bad in (dict(direction=0),):
        with pytest.raises(Bn.LstmError):
            Bn.gated_scan_fwd(z, **bad)
    with pytest.raises(Bn.LstmError):
        Bn.gated_scan_fwd(torch.zeros(40000, 1, 24, device="cuda"), workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    with pytest.raises(Bn.LstmError):
        Bn.gated_scan_bwd(f, z, torch.zeros(4, 2, 8, device="cuda"), workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
