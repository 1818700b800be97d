"""GPU parity of the label scores (lstm_label_score_fwd / _bwd through the binding) against oracle/train_oracle.py.

Tolerances.  log z is the rounding of float sums of exponentials whose arguments are rounded: with |x| <= X it is off by a few 2^-24 (X + |log z|)
plus the relative error of the sum, some 10 roundings: 1e-5 + 4 * 2^-24 X covers log probabilities and entropies (the latter sums
p log p with the same relative error, weighted by |log p| <= 30 there: 3e-5).  p is off by that much of itself, so the gradient by 4e-5 of
|dlogp| + |dent| (|log p + H| p <= 8 there); a bfloat16 gradient is off by half a step, 2^-8 of itself, more.  Labels are decided by
comparisons of the logits as they are and have to be equal."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import train_oracle as R
from tests.gpu_util import dev, tdtype

Bn = None


@pytest.fixture(scope="module", autouse=True)
def _binding():
    global Bn
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1805_05225_amd import binding
    Bn = binding
    yield


def _f64(t):
    return t.double().cpu().numpy()


def _same(name, got, ref, tol):
    got = _f64(got)
    assert got.shape == ref.shape, name
    special = ~np.isfinite(ref)
    assert np.array_equal(got[special], ref[special], equal_nan=True), name
    got, ref, tol = got[~special], ref[~special], (tol + np.zeros(ref.shape))[~special]
    assert np.isfinite(got).all() and (np.abs(got - ref) <= tol).all(), (name, float(np.max(np.abs(got - ref) - tol)))


def _check(x, label, dt, lens=None, top=0, wl=None, we=None, view=None):
    T, B, V = x.shape
    print("  label score T=%d B=%d V=%d %s top %d" % (T, B, V, dt, top), flush=True)
    xt = dev(x, dt) if view is None else view
    lt, Lt = None if label is None else dev(label.astype(np.int32)), dev(lens)
    x64 = _f64(xt)
    ref = R.label_score_fwd(x64, label, lens, top)
    f = Bn.label_score_fwd(xt, lt, Lt, top=top)
    torch.cuda.synchronize()
    big = np.abs(x64[np.isfinite(x64)]).max(initial=0)
    tol = 1e-5 + 4 * 2.0 ** -24 * big
    _same("lse", f["stats"].double().sum(-1), ref["lse"], tol)
    _same("entropy", f["entropy"], ref["entropy"], 3 * tol)
    if label is not None:
        _same("logp", f["logp"], ref["logp"], tol)
    else:
        assert f["logp"] is None
    if top:
        assert np.array_equal(f["top_label"].cpu().numpy(), ref["top_label"])
        _same("top_logp", f["top_logp"], ref["top_logp"], tol)
    if wl is not None or we is not None:
        d = Bn.label_score_bwd(f, xt, lt, dev(wl), dev(we), Lt)
        torch.cuda.synchronize()
        do = R.label_score_bwd(x64, label, wl, we, lens)
        size = (0 if wl is None else np.abs(wl)) + (0 if we is None else 8 * np.abs(we))
        _same("dlogits", d, do, 4 * tol * size[:, :, None] + (2.0 ** -8 * np.abs(np.nan_to_num(do)) if dt == "bf16" else 0) + 1e-37)
        return f, d
    return f, None


def _case(T, B, V, seed, spread=3.0):
    rng = np.random.default_rng(seed)
    return rng, (rng.standard_normal((T, B, V)) * spread).astype(np.float32), rng.integers(0, V, (T, B))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,V", [(1, 1, 1), (3, 2, 2), (2, 5, 63), (4, 3, 64), (1, 7, 255), (2, 2, 1000), (3, 3, 4099), (1, 5, 20000), (1, 3, 12001), (1, 2, 32768), (1, 257, 5000), (2, 2, 33001)])
def test_scores_and_gradients(T, B, V, dt):
    rng, x, label = _case(T, B, V, T + V)
    label.flat[0] = -1
    lens = rng.integers(0, T + 1, B).astype(np.int32)
    lens[0] = T
    w = lambda: rng.standard_normal((T, B)).astype(np.float32)
    _check(x, label, dt, lens, min(V, 16), w(), w())
    _check(x, label, dt, None, 0, w(), None)
    _check(x, label, dt, None, 1, None, w())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [131071, 262145])
@pytest.mark.parametrize("B", [1, 3, 40])
def test_large_vocabularies(B, V, dt):
    rng, x, label = _case(1, B, V, V + B)
    _check(x, label, dt, None, 16, rng.standard_normal((1, B)).astype(np.float32), rng.standard_normal((1, B)).astype(np.float32))


def test_many_rows():
    rng, x, label = _case(70, 50, 130, 11)
    _check(x, label, "f32", rng.integers(0, 71, 50).astype(np.int32), 4, rng.standard_normal((70, 50)).astype(np.float32), None)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 20000, 100003])
def test_alternatives_of_rows_with_ties(V, dt):
    """Constant rows, plateaus, ramps up and down, a few equal maxima far apart, fewer possible labels than alternatives: the smaller label first."""
    x = np.zeros((1, 9, V), dtype=np.float32)
    x[0, 1] = np.arange(V) // max(1, V // 40)
    x[0, 2] = -(np.arange(V) // max(1, V // 200)).astype(np.float32)
    x[0, 3, [V - 1, V // 2, 5]] = 2.0
    x[0, 4] = -np.inf
    x[0, 4, [7, V - 2]] = [1.0, 1.0]
    x[0, 5] = np.arange(V) % 7
    x[0, 6, ::2] = -np.inf
    x[0, 7] = np.linspace(-3, 3, V)
    x[0, 8] = -0.0
    x[0, 8, 1::3] = 0.0
    _check(x, np.full((1, 9), 7), dt, None, 16, np.ones((1, 9), np.float32), np.full((1, 9), 0.5, np.float32))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [70, 20000, 80001])
def test_rows_with_nothing_and_rows_with_too_much(V, dt):
    x = np.random.default_rng(V).standard_normal((2, 6, V)).astype(np.float32)
    x[0, 0] = -np.inf                                            # nothing can occur
    x[0, 1, V - 1] = np.nan
    x[0, 2, 3] = np.inf
    x[0, 3] = np.finfo(np.float32).min if dt == "f32" else float(torch.finfo(torch.bfloat16).min)        # a mask of the type's lowest value, on every label
    x[0, 4, 1:] = -np.inf                                        # one label left: certain
    x[0, 5, : V // 2] = np.finfo(np.float32).min if dt == "f32" else float(torch.finfo(torch.bfloat16).min)
    x[1, :, :] = np.nan                                          # padded, except row 0 whose weights are 0
    label = np.array([[0, 0, 1, 2, 0, V - 1], [0, -5, V, 1, 2, 1 << 30]])
    lens = np.array([2, 1, 1, 1, 1, 1], dtype=np.int32)
    wl = np.array([[1, 1, 1, 1, 1, 1], [0, np.nan, np.nan, 1, np.inf, 1]], dtype=np.float32)
    we = np.array([[1, 1, 1, .5, 1, 1], [0, np.nan, 1, 1, 1, 1]], dtype=np.float32)
    finite = np.array([True, False, False, True, True, True])
    f = Bn.label_score_fwd(dev(x, dt), dev(label.astype(np.int32)), dev(lens), top=5)
    ref = R.label_score_fwd(_f64(dev(x, dt)), label, lens, 5)
    # relative to the magnitude of the row: the type's lowest value is 3.4e38, its log sum is that value
    for k in ("logp", "entropy", "lse"):
        got, want = _f64(f[k] if k != "lse" else f["stats"].double().sum(-1)), ref[k]
        special = ~np.isfinite(want)
        assert np.array_equal(got[special], want[special], equal_nan=True), k
        assert np.allclose(got[~special], want[~special], rtol=3e-5, atol=3e-5), k
    assert np.array_equal(f["top_label"].cpu().numpy(), ref["top_label"])
    d = _f64(Bn.label_score_bwd(f, dev(x, dt), dev(label.astype(np.int32)), dev(wl), dev(we), dev(lens)))
    do = R.label_score_bwd(_f64(dev(x, dt)), label, wl, we, lens)
    assert np.isnan(d[0, 1]).all() and np.isnan(d[0, 2]).all() and not d[1].any() and not d[0, 0].any()
    assert np.allclose(d[0][finite], do[0][finite], rtol=2.0 ** -8 if dt == "bf16" else 1e-4, atol=1e-4)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [9, 30000])
def test_rows_of_nan_alone(V, dt):
    """No maximum to be found: values and gradient are NaN all the same, not those of a row where nothing can occur."""
    x = np.full((1, 3, V), np.nan, dtype=np.float32)
    x[0, 1, ::2] = -np.inf
    x[0, 2] = -np.inf
    label, w = torch.zeros(1, 3, dtype=torch.int32, device="cuda"), torch.ones(1, 3, device="cuda")
    f = Bn.label_score_fwd(dev(x, dt), label, top=2)
    d = Bn.label_score_bwd(f, dev(x, dt), label, w, w)
    for k in ("logp", "entropy"):
        assert torch.isnan(f[k][0, :2]).all()
    assert torch.isnan(f["stats"][0, :2]).all() and torch.isnan(d[0, :2]).all()
    assert f["logp"][0, 2] == -np.inf and f["entropy"][0, 2] == 0 and not d[0, 2].any()
    assert (f["top_logp"] == -np.inf).all() and not f["top_label"].any()


def test_more_alternatives_than_labels():
    rng, x, label = _case(2, 3, 5, 2)
    _check(x, label, "f32", None, 16, None, None)


def test_large_logits():
    rng, x, label = _case(1, 8, 5000, 3, spread=2000.0)
    _check(x, label, "f32", None, 8, np.ones((1, 8), np.float32), None)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("shift,extra", [(0, 1), (1, 0), (3, 2), (5, 8)])
@pytest.mark.parametrize("V", [97, 10007])
def test_rows_at_any_element(V, shift, extra, dt):
    T, B = 2, 3
    rng, x, label = _case(T, B, V, 5)
    full = torch.full((T, B, V + shift + extra), 50.0, dtype=tdtype(dt), device="cuda")
    view = full[:, :, shift:shift + V]
    view.copy_(dev(x, dt))
    w = rng.standard_normal((T, B)).astype(np.float32)
    f, d = _check(x, label, dt, None, 7, w, w, view=view)
    out = torch.full((T, B, V + 2 * shift + 1), 9.0, dtype=tdtype(dt), device="cuda")
    to = out[:, :, shift + 1:shift + 1 + V]
    got = Bn.label_score_bwd(f, view, dev(label.astype(np.int32)), dev(w), dev(w), out=to)
    assert got.data_ptr() == to.data_ptr() and torch.equal(to, d)
    assert (out[:, :, :shift + 1] == 9).all() and (out[:, :, shift + 1 + V:] == 9).all()
    Bn.label_score_bwd(f, view, dev(label.astype(np.int32)), dev(w), dev(w), out=view)               # in place
    assert torch.equal(view, d) and (full[:, :, :shift] == 50).all() and (full[:, :, shift + V:] == 50).all()


def test_without_label_and_without_time():
    rng, x, _ = _case(1, 6, 777, 1)
    f = Bn.label_score_fwd(dev(x[0], "f32"), top=3, want_entropy=False)
    assert f["logp"] is None and f["entropy"] is None and f["stats"].shape == (6, 2) and f["top_label"].shape == (6, 3)
    _check(x, None, "f32", None, 3, None, np.ones((1, 6), np.float32))
    e = Bn.label_score_fwd(torch.empty(0, 5, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), top=2)
    assert e["logp"].shape == (0,) and e["top_logp"].shape == (0, 2)


def test_repeats_its_bits_on_any_stream_and_in_a_graph():
    T, B, V = 3, 5, 9000
    rng, x, label = _case(T, B, V, 8)
    xt, lt, w = dev(x, "bf16"), dev(label.astype(np.int32)), dev(rng.standard_normal((T, B)).astype(np.float32))

    def run():
        f = Bn.label_score_fwd(xt, lt, top=6)
        return [f[k] for k in ("logp", "entropy", "stats", "top_logp", "top_label")] + [Bn.label_score_bwd(f, xt, lt, w, w)]

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
        xt.copy_(dev(np.roll(x, k, axis=2), "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, run()))
    xt.copy_(dev(x, "bf16"))
    assert all(torch.equal(a, b) for a, b in zip(first, second)) and all(torch.equal(a, b) for a, b in zip(first, run()))


def test_rows_behind_32_bit_offsets():
    """The last rows of 2.4e9 logits against a call of their own, whose sums are put together differently: 60001 terms in float, a few hundred a
    lane and then lane by lane, under 500 2^-24 of the sum (of the entropy's, |x - m| <= 40 times that); a gradient is a product with p and is rounded once on either side."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.empty(40000, 60001, dtype=torch.bfloat16, device="cuda").normal_(0, 3, generator=gen)
    label = torch.randint(0, 60001, (40000,), generator=gen, device="cuda", dtype=torch.int32)
    w = torch.rand(40000, generator=gen, device="cuda")
    f = Bn.label_score_fwd(x, label, top=4)
    d = Bn.label_score_bwd(f, x, label, w, w)
    own = Bn.label_score_fwd(x[-3:], label[-3:], top=4)
    own_d = Bn.label_score_bwd(own, x[-3:], label[-3:], w[-3:], w[-3:])
    assert torch.equal(f["top_label"][-3:], own["top_label"]) and torch.equal(f["stats"][-3:, 0], own["stats"][:, 0])
    tol = 500 * 2.0 ** -24
    for k in ("logp", "top_logp"):
        assert ((f[k][-3:] - own[k]).abs() <= tol + 2.0 ** -22 * own[k].abs()).all(), k
    assert ((f["entropy"][-3:] - own["entropy"]).abs() <= 40 * tol).all()
    assert ((d[-3:].float() - own_d.float()).abs() <= (2.0 ** -7 + 100 * tol) * own_d.float().abs() + 1e-30).all()
    assert torch.equal(d[-3:] == 0, own_d == 0)


def test_refusals():
    x, l = torch.zeros(2, 3, 10, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    bad = AssertionError
    for call in (lambda: Bn.label_score_fwd(x.cpu(), l), lambda: Bn.label_score_fwd(x.half(), l), lambda: Bn.label_score_fwd(x, l.long()),
                 lambda: Bn.label_score_fwd(x, l[:1].contiguous()), lambda: Bn.label_score_fwd(x.transpose(0, 2), l),
                 lambda: Bn.label_score_fwd(x.transpose(0, 1), l), lambda: Bn.label_score_fwd(x, l, torch.ones(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(bad):
            call()
    f = Bn.label_score_fwd(x, l)
    w = torch.zeros(2, 3, device="cuda")
    for call in (lambda: Bn.label_score_bwd(f, x, l, w[:1].contiguous()), lambda: Bn.label_score_bwd(f, x, l, w.double()),
                 lambda: Bn.label_score_bwd(f, x, l, w, out=torch.zeros(2, 3, 11, device="cuda"))):
        with pytest.raises(bad):
            call()
    for call in (lambda: Bn.label_score_fwd(x, l, top=17), lambda: Bn.label_score_fwd(x, l, top=-1),
                 lambda: Bn.label_score_fwd(torch.zeros(1, 20000, device="cuda"), l[0, :1], workspace=torch.empty(1, dtype=torch.uint8, device="cuda")),
                 lambda: Bn.label_score_bwd(dict(stats=f["stats"], entropy=None), x, l, w, w), lambda: Bn.label_score_bwd(f, x, None, w)):
        with pytest.raises(Bn.LstmError):
            call()
