"""GPU parity of the update (lstm_grad_norm, lstm_adamw_step through the binding) against oracle/train_oracle.py.

Tolerances.  m and v are two products and a sum: 4 * 2^-24 of |m| + |g| (v: of v + g^2).  w = w0 keep - step: keep, its product and the sum are rounded
(3 * 2^-24 |w0|, 2^-24 |step|).  step = rate m / (sqrt(v) / root + eps): rate, root, the root, both divisions, the sum and the product are rounded, and
half of v's three roundings enters: under 12 * 2^-24 |step|; m itself may be the small difference of b1 m0 and (1 - b1) g, whose constants, products
and sum are rounded: 3 * 2^-24 (b1 |m0| + (1 - b1) |g|) of it, whatever is left of m.  A bfloat16 parameter is the rounding of w: 2^-8 more.  In 8 bits a state is off by half a step, 2^-4 of itself or 2^-10 of the block's scale (a positive root that
would become 0: 2^-9), and a scale by 4 roundings.  The norm is summed in 64 bits and rounded once: 2^-24 of itself, twice."""
import ctypes
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import train_oracle as R
from tests.gpu_util import dev, tdtype

Bn = None
E = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _binding():
    global Bn
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_1805_05225_amd import binding
    Bn = binding
    yield


def _f64(t):
    return t.detach().double().cpu().numpy().reshape(-1)


def _model(counts, param, grad, bits, seed, shift=0, master=True):
    """Tensors of these sizes, `shift` elements behind an aligned address, with states that training has left."""
    rng = np.random.default_rng(seed)

    def put(a, dt):
        full = torch.zeros(a.size + shift, dtype=dt, device="cuda")
        full[shift:].copy_(torch.from_numpy(a.astype(np.float32)).to(dt))
        return full[shift:]

    s = dict(params=[], grads=[], m=[], v=[], masters=[] if master and param == "bf16" else None)
    if bits == 8:
        s.update(m_scale=[], v_scale=[])
    for n in counts:
        w = rng.standard_normal(n) * 0.3
        s["params"].append(put(w, tdtype(param)))
        if s["masters"] is not None:
            s["masters"].append(put(w, torch.float32))
        s["grads"].append(put(rng.standard_normal(n) * 10.0 ** rng.uniform(-4, 0), tdtype(grad)))
        if bits == 8:
            code = rng.standard_normal(n) * 100
            s["m"].append(put(np.clip(code, -448, 448), torch.float8_e4m3fn))
            s["v"].append(put(np.clip(np.abs(code), 2.0 ** -9, 448), torch.float8_e4m3fn))
            s["m_scale"].append(put(rng.uniform(0.1, 1, -(-n // 256)) * 1e-5, torch.float32))
            s["v_scale"].append(put(rng.uniform(0.1, 1, -(-n // 256)) * 1e-4, torch.float32))
        else:
            s["m"].append(put(rng.standard_normal(n) * 1e-3, torch.float32))
            s["v"].append(put(rng.standard_normal(n) ** 2 * 1e-5, torch.float32))
    return s


def _state(s, i):
    """m and v in 64 bits."""
    m, v = _f64(s["m"][i]), _f64(s["v"][i])
    if "m_scale" in s:
        return m * R.spread(_f64(s["m_scale"][i]), m.size), (v * R.spread(_f64(s["v_scale"][i]), v.size)) ** 2
    return m, v


def _step_and_compare(s, step=7, lr=1e-2, decay=None, scale=None, **hyper):
    n = len(s["params"])
    decay = [0.01 * (i % 2) for i in range(n)] if decay is None else decay
    src = s["masters"] if s["masters"] is not None else s["params"]
    old = [(_f64(src[i]), _f64(s["grads"][i]), *_state(s, i)) for i in range(n)]
    gs = None if scale is None else torch.tensor([scale], dtype=torch.float32, device="cuda")
    Bn.adamw_step(lr=lr, step=step, weight_decay=decay, grad_scale=gs, **hyper, **s)
    torch.cuda.synchronize()
    h = dict(beta1=0.9, beta2=0.999, eps=1e-8)
    h.update(hyper)
    for i in range(n):
        w0, g, m0, v0 = old[i]
        g = g * (1.0 if scale is None else float(np.float32(scale)))
        w, m, v = R.adamw(w0, g, m0, v0, step, lr, decay=float(np.float32(decay[i])), **h)
        moved = np.abs(w - w0) + lr * decay[i] * np.abs(w0)
        b1, b2 = h["beta1"], h["beta2"]
        of_m = lr / (1 - b1 ** step) * (b1 * np.abs(m0) + (1 - b1) * np.abs(g)) / (np.sqrt(v / (1 - b2 ** step)) + h["eps"])
        tol = 4 * E * np.abs(w0) + 12 * E * moved + 3 * E * of_m + 1e-38
        got = _f64(src[i])
        assert (np.abs(got - w) <= tol).all(), ("w", i, float((np.abs(got - w) / tol).max()))
        if s["masters"] is not None:
            assert torch.equal(s["params"][i], src[i].to(torch.bfloat16)), i
        gm, gv = _state(s, i)
        tm, tv = 4 * E * (np.abs(m) + np.abs(m0) + np.abs(g)) + 1e-45, 4 * E * (v + v0 + g * g) + 1e-45
        if "m_scale" not in s:
            assert (np.abs(gm - m) <= tm).all() and (np.abs(gv - v) <= tv).all(), i
            continue
        r = np.sqrt(v)
        for name, kept, want, scales in (("m", gm, m, s["m_scale"][i]), ("r", np.sqrt(gv), r, s["v_scale"][i])):
            sc = R.block_scale(want)
            assert (np.abs(_f64(scales) - sc) <= 8 * E * sc + (tm.max() if name == "m" else 0) / 448 + 1e-45).all(), (name, i)
            each = R.spread(sc, want.size)
            off = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * each) * (1 + 1e-5) + tm.max()
            if name == "r":
                off = np.where(want < 2.0 ** -9 * each, 2.0 ** -9 * each * (1 + 1e-5), off)
                assert (kept[want > 0] > 0).all()
            assert (np.abs(kept - want) <= off).all(), (name, i, float((np.abs(kept - want) / off).max()))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad,master", [("f32", "f32", False), ("bf16", "f32", True), ("bf16", "bf16", True)])
@pytest.mark.parametrize("counts", [[1], [255, 256, 257], [3, 4096, 4097, 1, 16383, 70001]])
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_adamw(counts, param, grad, master, bits, shift):
    print("  adamw %s %s %s %d bits, shift %d" % (counts, param, grad, bits, shift), flush=True)
    s = _model(counts, param, grad, bits, sum(counts) + shift, shift, master)
    _step_and_compare(s)
    _step_and_compare(s, step=8, scale=0.37, beta1=0.8, beta2=0.95, eps=1e-6, lr=3e-3)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_of_a_bfloat16_parameter_without_master(bits):
    s = _model([1000, 7], "bf16", "f32", bits, 3, master=False)
    w = [_f64(p) for p in s["params"]]
    ref = [R.adamw(w[i], _f64(s["grads"][i]), *_state(s, i), 2, 1e-2, decay=float(np.float32(0.1)))[0] for i in range(2)]
    Bn.adamw_step(lr=1e-2, step=2, weight_decay=0.1, **s)
    for p, r in zip(s["params"], ref):
        assert (np.abs(_f64(p) - r) <= (2.0 ** -8 + 20 * E) * np.abs(r) + 1e-9).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [43, 57, 58, 59, 200])
def test_adamw_of_many_tensors(count, bits):
    rng = np.random.default_rng(count)
    s = _model([int(n) for n in rng.integers(0, 9000, count)], "f32", "f32", bits, count)
    _step_and_compare(s)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_from_zero_states_over_steps(bits):
    """The first steps from adamw_state's zeros: the oracle takes the gradients, its own states in 32 bits or the kernel's in 8."""
    s = _model([700, 3], "bf16", "f32", bits, 5)
    s.update(Bn.adamw_state(s["params"], bits))
    rng = np.random.default_rng(1)
    for t in range(1, 5):
        for g in s["grads"]:
            g.copy_(torch.from_numpy(rng.standard_normal(g.numel()).astype(np.float32)))
        s["grads"][0][256:512] = 0.0                              # a block without gradients: states and scales stay 0, weights only decay
        _step_and_compare(s, step=t)
    if bits == 8:
        assert s["m_scale"][0][1] == 0 and not s["m"][0].view(torch.uint8)[256:512].any()


def test_8_bit_roots_stay_positive():
    """An element whose root is far below its block's largest keeps a denominator: without a gradient its weight moves by less than a step of full size."""
    n = 256
    s = dict(params=[torch.zeros(n, device="cuda")], grads=[torch.full((n,), 1e-6, device="cuda")], **Bn.adamw_state([torch.zeros(n, device="cuda")], 8))
    s["grads"][0][0] = 100.0
    Bn.adamw_step(lr=1e-3, step=1, **s)
    r = s["v"][0].float() * s["v_scale"][0]
    assert (r > 0).all()
    before = s["params"][0].clone()
    s["grads"][0].zero_()
    Bn.adamw_step(lr=1e-3, step=2, **s)
    assert ((s["params"][0] - before).abs() <= 2e-3).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("scale", [math.nan, math.inf])
def test_a_scale_that_is_not_finite_changes_nothing(bits, scale):
    s = _model([300, 5000], "bf16", "f32", bits, 6)
    before = {k: [t.clone() for t in v] for k, v in s.items()}
    Bn.adamw_step(lr=1e-2, step=3, weight_decay=0.1, grad_scale=torch.tensor([scale], device="cuda"), **s)
    bits_of = lambda t: t.view(torch.uint8) if t.element_size() == 1 else t
    for k, v in s.items():
        assert all(torch.equal(bits_of(a), bits_of(b)) for a, b in zip(v, before[k])), k


@pytest.mark.parametrize("bits", [32, 8])
def test_nan_and_infinite_gradients_stay_where_they_are(bits):
    n = 1000
    s = _model([n], "f32", "f32", bits, 7)
    same = _model([n], "f32", "f32", bits, 7)
    s["grads"][0][300] = math.nan
    same["grads"][0][300] = 0.0
    Bn.adamw_step(lr=1e-2, step=3, **s)
    Bn.adamw_step(lr=1e-2, step=3, **same)
    w, ref = s["params"][0], same["params"][0]
    others = torch.arange(n, device="cuda") != 300
    assert torch.isnan(w[300]) and torch.equal(w[others], ref[others])
    m = s["m"][0].float()
    assert torch.isnan(m[300]) and torch.isfinite(m[others]).all()
    s["grads"][0][700] = math.inf                                 # 8 bits: the block of 256 that it lies in is lost, no other
    Bn.adamw_step(lr=1e-2, step=4, **s)
    Bn.adamw_step(lr=1e-2, step=5, **s)
    rest = others & ((torch.arange(n, device="cuda") // 256 != 700 // 256) if bits == 8 else torch.arange(n, device="cuda") != 700)
    assert torch.isfinite(s["params"][0][rest]).all() and not torch.isfinite(s["params"][0][700])


@pytest.mark.parametrize("g", [1e-17, 1e-19, 1e-20])
def test_first_step_of_tiny_gradients_without_eps(g):
    """m / sqrt(v) is g / |g| at the first step however small v is: v = 0.001 g^2 is rounded to 2^-149 at the least, its root by half of that relative to v."""
    w0, sign = torch.ones(300, device="cuda"), torch.where(torch.arange(300, device="cuda") % 2 == 0, 1.0, -1.0)
    w, m, v = w0.clone(), torch.zeros_like(w0), torch.zeros_like(w0)
    Bn.adamw_step([w], [sign * g], [m], [v], lr=0.25, step=1, eps=0.0)
    off = 2.0 ** -149 / (1e-3 * g * g) + 20 * E
    assert (np.abs(_f64(w) - (1 - 0.25 * _f64(sign))) <= 0.25 * off + 4 * E).all()


def test_a_tensor_of_more_elements_than_a_table_entry():
    """Behind 2^28 elements (2^31 for the norm) a tensor goes on in the table's next entry: the elements around there fare as they do in a tensor of their own."""
    n, cut = (1 << 28) + 300, (1 << 28) - 512
    gen = torch.Generator(device="cuda").manual_seed(1)
    p = torch.rand(n, generator=gen, device="cuda").to(torch.bfloat16)
    g = torch.rand(n, generator=gen, device="cuda").to(torch.bfloat16)
    st = Bn.adamw_state([p], 8)
    q, h = p[cut:].clone(), g[cut:].clone()
    own = Bn.adamw_state([q], 8)
    for step in (1, 2):
        Bn.adamw_step([p], [g], lr=1e-2, step=step, **st)
        Bn.adamw_step([q], [h], lr=1e-2, step=step, **own)
    assert torch.equal(p[cut:], q) and not torch.equal(g[cut:], q)
    for k in ("m", "v"):
        assert torch.equal(st[k][0][cut:].view(torch.uint8), own[k][0].view(torch.uint8)) and torch.equal(st[k + "_scale"][0][cut // 256:], own[k + "_scale"][0])
    del p, g, st
    ones = torch.ones((1 << 31) + 5, dtype=torch.bfloat16, device="cuda")
    assert float(Bn.grad_norm([ones])[0]) == float(np.float32(math.sqrt((1 << 31) + 5)))


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("counts", [[1], [16383, 16384, 16385], [5, 0, 100003, 1, 40000], [3] * 400, [300] * 255])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_grad_norm(counts, grad, shift):
    s = _model(counts, "f32", grad, 32, len(counts), shift)
    norm, clip = R.grad_norm([_f64(g) for g in s["grads"]], 0.5)
    got = Bn.grad_norm(s["grads"], 0.5).cpu().numpy().astype(np.float64)
    assert abs(got[0] - norm) <= 2 * E * norm and abs(got[1] - clip) <= 2 * E * clip
    assert Bn.grad_norm(s["grads"], norm * 2)[1] == 1 and Bn.grad_norm(s["grads"])[1] == 1


def test_grad_norm_of_extremes():
    t = lambda *v: torch.tensor(v, device="cuda")
    assert Bn.grad_norm([t(0.0, 0.0)], 1.0).tolist() == [0.0, 1.0]
    big = Bn.grad_norm([t(3e38), t(2e38)], 1.0)                   # squares beyond a float's range
    assert torch.isinf(big[0]) or abs(big[0].item() / math.hypot(3e38, 2e38) - 1) < 1e-6
    assert abs(Bn.grad_norm([t(3e30, 4e30)], 1.0)[0].item() / 5e30 - 1) < 1e-6
    assert abs(Bn.grad_norm([t(3e-30, 4e-30)], 1.0)[0].item() / 5e-30 - 1) < 1e-6
    for bad in (math.nan, math.inf, -math.inf):
        r = Bn.grad_norm([t(1.0), t(1.0, bad)], 1.0)
        assert not torch.isfinite(r[0]) and torch.isnan(r[1])
    out = torch.full((2,), 9.0, device="cuda")
    assert Bn.grad_norm([], 1.0, out=out).tolist() == [0.0, 1.0] and Bn.grad_norm([t(), t()], 1.0, out=out).tolist() == [0.0, 1.0]


@pytest.mark.parametrize("bits", [32, 8])
def test_clip_and_step_in_a_graph_follow_a_schedule(bits):
    """Norm and step captured once; learning rate and step number are read from device memory at every replay."""
    s, e = (_model([5000, 300, 77], "bf16", "f32", bits, 9) for _ in range(2))
    lr, step = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
    out = torch.empty(2, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Bn.grad_norm(s["grads"], 0.7, out=out, workspace=ws)
        Bn.adamw_step(lr=lr, step=step, weight_decay=0.01, grad_scale=out[1:], **s)
    bits_of = lambda t: t.view(torch.uint8) if t.element_size() == 1 else t
    for t in range(1, 5):
        for a, b in zip(s["grads"], e["grads"]):
            a.normal_(generator=torch.Generator(device="cuda").manual_seed(t))
            b.copy_(a)
        lr.fill_(1e-2 / t)
        step.fill_(t)
        graph.replay()
        torch.cuda.synchronize()
        Bn.adamw_step(lr=float(np.float32(1e-2 / t)), step=t, weight_decay=0.01, grad_scale=Bn.grad_norm(e["grads"], 0.7)[1:], **e)
        for k in s:
            assert all(torch.equal(bits_of(a), bits_of(b)) for a, b in zip(s[k], e[k])), (t, k)


def test_update_repeats_its_bits_on_another_stream():
    a, b = (_model([70000, 3], "bf16", "f32", 8, 2) for _ in range(2))
    na = Bn.grad_norm(a["grads"], 1.0)
    Bn.adamw_step(lr=1e-2, step=1, grad_scale=na[1:], **a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        nb = Bn.grad_norm(b["grads"], 1.0)
        Bn.adamw_step(lr=1e-2, step=1, grad_scale=nb[1:], **b)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(na, nb) and all(torch.equal(x, y) for x, y in zip(a["params"], b["params"]))


def test_refusals():
    p, g = [torch.zeros(10, device="cuda")], [torch.zeros(10, device="cuda")]
    st = Bn.adamw_state(p)
    e8 = Bn.adamw_state(p, 8)
    ok = dict(lr=1e-3, step=1)
    for call in (lambda: Bn.adamw_step(p, [g[0].cpu()], **st, **ok), lambda: Bn.adamw_step(p, [g[0].half()], **st, **ok),
                 lambda: Bn.adamw_step(p, [g[0][:9]], **st, **ok), lambda: Bn.adamw_step(p, g + g, **st, **ok),
                 lambda: Bn.adamw_step(p, [torch.zeros(20, device="cuda")[::2]], **st, **ok),
                 lambda: Bn.adamw_step(p, g, e8["m"], e8["v"], **ok), lambda: Bn.adamw_step(p, g, **e8, weight_decay=[0.1, 0.1], **ok),
                 lambda: Bn.adamw_step(p, g, e8["m"], e8["v"], m_scale=e8["m_scale"], **ok), lambda: Bn.adamw_step([p[0].half()], g, **st, **ok),
                 lambda: Bn.adamw_step(p, g, **st, lr=1e-3, step=torch.ones(1, device="cuda")), lambda: Bn.grad_norm([g[0].double()])):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: Bn.adamw_step(p, g, **st, lr=1e-3, step=0), lambda: Bn.adamw_step(p, g, **st, lr=-1.0, step=1),
                 lambda: Bn.adamw_step(p, g, **st, **ok, beta1=1.0), lambda: Bn.adamw_step(p, g, **st, **ok, weight_decay=-0.1),
                 lambda: Bn.adamw_step(p, g, **st, **ok, masters=p), lambda: Bn.grad_norm(g, 0.0), lambda: Bn.grad_norm(g, math.nan),
                 lambda: Bn.grad_norm(g, workspace=torch.empty(1, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(Bn.LstmError):
            call()
    assert ctypes.sizeof(Bn.AdamwItem) == 80
