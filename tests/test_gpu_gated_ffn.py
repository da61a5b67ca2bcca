"""The dense gated FFN, forward and backward, against its definition in 64 bits: every element within the bound that the
stated roundings allow.  A rounding to bf16 is off by at most 2^-8 of the value, an fp32 sum of n terms by at most
n 2^-24 of the sum of their magnitudes (taken twice, for products and the activation's own rounding)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

R = 2.0 ** -8      # half a step of bf16, relative
R24 = 2.0 ** -15  # 24 bits, the rest dropped
A2 = 0.9           # beyond the largest |a''| of silu (0.5) and of gelu's tanh form (0.80)
SECOND = 1.03      # products of two or three of the errors above


@pytest.fixture(scope="module")
def hire():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2402_09360_amd import hire as H
    return H


def activation(g, act):
    """The activation and its derivative in 64 bits."""
    if act == "relu":
        return g.clamp(min=0.0), (g > 0).double()
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1.0 - s)
    c = (2.0 / torch.pi) ** 0.5
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * g * g)


def expected(x, wg, wu, w2, dy, act):
    """name -> (value, bound of the error) in 64 bits; the fp32 sums' part by their length."""
    x, wg, wu, w2, dy = (t.double() for t in (x, wg, wu, w2, dy))
    T, d = x.shape
    F = wg.shape[0]
    f32 = lambda n: 2.0 * (n + 8) * 2.0 ** -24
    g, u = x @ wg.t(), x @ wu.t()
    a, da = activation(g, act)
    a2 = 0.0 if act == "relu" else A2
    err_g, err_u = f32(d) * (x.abs() @ wg.abs().t()), f32(d) * (x.abs() @ wu.abs().t())
    err_a = 1.2 * err_g + 2.0 ** -21 * (a.abs() + g.abs() * da.abs())  # |a'| < 1.2; the activation's own fp32 steps
    h = a * u
    err_h = R * h.abs() + (err_a * u.abs() + a.abs() * err_u)
    y = h @ w2
    out = dict(y=(y, R * y.abs() + err_h @ w2.abs() + f32(F) * (h.abs() @ w2.abs())))
    dh = dy @ w2.t()
    err_dh = f32(d) * (dy.abs() @ w2.abs().t())
    dg, du = dh * u * da, dh * a
    kept_g, kept_u = R24 * g.abs() + err_g, R24 * u.abs() + err_u
    err_dg = (R * dg.abs() + err_dh * (u * da).abs() + dh.abs() * (kept_u * da.abs() + u.abs() * a2 * kept_g) +
              2.0 ** -19 * (dh * u).abs() * (1.0 + g.abs()))
    err_du = R * du.abs() + err_dh * a.abs() + dh.abs() * (1.2 * kept_g + 2.0 ** -20 * (a.abs() + g.abs()))
    dx = dg @ wg + du @ wu
    out["dx"] = (dx, R * dx.abs() + (err_dg + f32(2 * F) * dg.abs()) @ wg.abs() + (err_du + f32(2 * F) * du.abs()) @ wu.abs())
    for name, left, err, right in (("dwg", dg, err_dg, x), ("dwu", du, err_du, x), ("dw2u", h, err_h, dy)):
        v = left.t() @ right
        out[name] = (v, R * v.abs() + (err + f32(T) * left.abs()).t() @ right.abs())
    return out


def inputs(seed, T, d, F, exact=False):
    """Seeded layer, tokens and output gradients; exact: multiples of 1/4 whose sums are exact in fp32, so that the gate's
    sign is the same in any precision."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def draw(shape, scale):
        v = torch.randn(shape, generator=gen, device="cuda") * scale
        return ((v * 4 / scale).round() / 4 if exact else v).to(torch.bfloat16)

    return (draw((T, d), 1.0), draw((F, d), d ** -0.5), draw((F, d), d ** -0.5), draw((F, d), F ** -0.5), draw((T, d), 1.0))


def run(hire, data, act, train=True, dirty=True):
    x, wg, wu, w2, dy = data
    T = x.shape[0]
    layer = hire.GatedLayer(wg, wu, w2, act=act)
    out = hire.GatedOutputs(layer, T, train=train)
    nbytes = hire.hire_gated_ffn_workspace_bytes(layer, T)
    if train:
        nbytes = max(nbytes, hire.hire_gated_ffn_backward_workspace_bytes(layer, T))
    ws = hire.alloc_workspace(nbytes)
    if dirty:
        ws.fill_(0xFF)   # NaN in whatever a kernel might read before it is written
    out.y.fill_(float("nan"))
    hire.hire_gated_ffn_step(layer, x, out, ws)
    got = dict(y=out.y)
    if train:
        grads = hire.GatedGradients(layer, T)
        for t in (grads.dx, grads.dwg, grads.dwu, grads.dw2u):
            t.fill_(float("nan"))
        hire.hire_gated_ffn_backward(layer, x, out, dy, grads, ws)
        got.update(dx=grads.dx, dwg=grads.dwg, dwu=grads.dwu, dw2u=grads.dw2u)
    torch.cuda.synchronize()
    return got


def check(got, data, act):
    want = expected(*data, act)
    for name, v in got.items():
        value, bound = want[name]
        over = (v.double() - value).abs() - SECOND * bound
        assert bool((over <= 2.0 ** -120).all()), (name, float(over.max()), float(value.abs().max()))


@pytest.mark.parametrize("T", [1, 2, 3, 15, 16, 17, 33, 48, 63, 64, 65, 100, 127, 129, 256, 257, 520])
def test_token_counts(hire, T):
    print(f"T={T}", flush=True)
    data = inputs(T, T, 264, 328)
    check(run(hire, data, "silu"), data, "silu")


@pytest.mark.parametrize("T,d,F,act", [
    (1, 8, 8, "silu"), (5, 8, 1048, "gelu"), (7, 1048, 8, "silu"), (31, 136, 72, "gelu"), (65, 8, 8, "gelu"),
    (300, 40, 648, "silu"), (200, 1032, 264, "gelu"), (64, 2048, 1024, "silu"), (16, 256, 4104, "gelu"),
    (2, 4096, 1528, "silu"), (700, 512, 256, "gelu"), (1, 256, 1024, "silu"), (333, 800, 2504, "gelu")])
def test_widths(hire, T, d, F, act):
    print(f"T={T} d={d} F={F} {act}", flush=True)
    data = inputs(T + d, T, d, F)
    check(run(hire, data, act), data, act)


@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("T,d,F", [(70, 2056, 72), (130, 4104, 264), (257, 1048, 40), (3000, 72, 136), (1531, 8, 8), (513, 264, 2600)])
def test_products_in_parts(hire, T, d, F, act):
    """Few tiles and many k: of the first layer's products, of the weights' gradients, of y and dx."""
    print(f"T={T} d={d} F={F} {act}", flush=True)
    data = inputs(T + d, T, d, F, exact=act == "relu")
    check(run(hire, data, act), data, act)


@pytest.mark.parametrize("T,d,F,act", [
    (17, 1024, 8200, "silu"), (40, 2056, 4104, "gelu"), (64, 3000, 2808, "silu"), (33, 5000, 1688, "gelu"),
    (48, 16384, 520, "silu"), (12, 8192, 4104, "gelu"), (16, 2048, 16384, "silu"), (31, 1032, 8136, "gelu"),
    (40, 2056, 8200, "gelu"), (64, 5000, 3400, "silu"), (17, 1032, 16400, "silu")])
def test_few_tokens_of_large_layers(hire, T, d, F, act):
    print(f"T={T} d={d} F={F} {act}", flush=True)
    data = inputs(T + d, T, d, F)
    check(run(hire, data, act), data, act)
    assert torch.equal(run(hire, data, act, train=False)["y"], run(hire, data, act)["y"])


@pytest.mark.parametrize("T,d,F", [(1, 64, 128), (40, 96, 264), (130, 64, 512), (300, 128, 136)])
def test_relu_at_zero(hire, T, d, F):
    """Exact pre-activations, some of them 0 (of 128 with one token none is): the slope there is 0."""
    data = inputs(7 * T, T, d, F, exact=True)
    assert T == 1 or int((data[0].double() @ data[1].double().t() == 0).sum()) > 0
    check(run(hire, data, "relu"), data, "relu")


@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("T", [4, 90])
def test_far_gates(hire, act, T):
    """Gates of thousands on either side: the logistic function saturates, its derivative's factors overflow or vanish."""
    x, wg, wu, w2, dy = inputs(11, T, 64, 72, exact=True)
    data = (x, (wg * 1024).to(torch.bfloat16), wu, w2, dy)
    got = run(hire, data, act)
    assert all(bool(torch.isfinite(v).all()) for v in got.values())
    check(got, data, act)


def test_gradients_against_differences(hire):
    """d(sum(dy y)) along a direction, from the gradients and from the 64-bit definition's differences."""
    data = inputs(21, 70, 72, 200)
    got = run(hire, data, "gelu")
    x, wg, wu, w2, dy = (t.double() for t in data)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(22)

    def loss(x, wg, wu, w2):
        return float((dy * ((activation(x @ wg.t(), "gelu")[0] * (x @ wu.t())) @ w2)).sum())

    for i, name in enumerate(("dx", "dwg", "dwu", "dw2u")):
        base = [x, wg, wu, w2]
        step = torch.randn(base[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        eps = 1e-5
        up, down = list(base), list(base)
        up[i], down[i] = base[i] + eps * step, base[i] - eps * step
        slope = (loss(*up) - loss(*down)) / (2 * eps)
        value, bound = expected(*data, "gelu")[name]
        room = float((SECOND * bound * step.abs()).sum()) + 1e-6 * float((value * step).abs().sum())
        assert abs(float((got[name].double() * step).sum()) - slope) <= room, name


@pytest.mark.parametrize("T", [1, 20, 150])
def test_repeats_are_equal_and_parts_can_be_left_out(hire, T):
    data = inputs(31, T, 520, 1160)
    first, again = run(hire, data, "silu"), run(hire, data, "silu", dirty=False)
    for name in first:
        assert torch.equal(first[name], again[name]), name
    assert torch.equal(run(hire, data, "silu", train=False)["y"], first["y"])
    x, wg, wu, w2, dy = data
    layer = hire.GatedLayer(wg, wu, w2)
    out = hire.GatedOutputs(layer, T, train=True)
    ws = hire.alloc_workspace(max(hire.hire_gated_ffn_workspace_bytes(layer, T),
                                  hire.hire_gated_ffn_backward_workspace_bytes(layer, T)))
    hire.hire_gated_ffn_step(layer, x, out, ws)
    names = ("dx", "dwg", "dwu", "dw2u")
    for keep in (("dx",), ("dwg",), ("dwu", "dw2u"), ("dw2u",), ("dx", "dwu")):
        grads = hire.GatedGradients(layer, T)
        for n in names:
            if n not in keep:
                setattr(grads, n, None)
        hire.hire_gated_ffn_backward(layer, x, out, dy, grads, ws)
        torch.cuda.synchronize()
        for n in keep:
            assert torch.equal(getattr(grads, n), first[n]), (keep, n)


def test_rows_behind_the_last_stay(hire):
    """Outputs inside larger buffers: nothing in front of them or behind them is written."""
    for T in (3, 70):
        x, wg, wu, w2, dy = inputs(41, T, 72, 136)
        layer = hire.GatedLayer(wg, wu, w2)
        out = hire.GatedOutputs(layer, T, train=True)
        grads = hire.GatedGradients(layer, T)
        big = {}
        saved = torch.full((out.saved.numel() + 512,), 0x5A, dtype=torch.uint8, device="cuda")
        out.saved = saved[256:256 + out.saved.numel()]
        for o, names in ((out, ("y",)), (grads, ("dx", "dwg", "dwu", "dw2u"))):
            for n in names:
                t = getattr(o, n)
                big[n] = torch.full((t.shape[0] + 16, t.shape[1]), 7.0, dtype=torch.bfloat16, device="cuda")
                setattr(o, n, big[n][8:8 + t.shape[0]])
        nbytes = max(hire.hire_gated_ffn_workspace_bytes(layer, T), hire.hire_gated_ffn_backward_workspace_bytes(layer, T))
        ws = torch.full((nbytes + 512,), 0x5A, dtype=torch.uint8, device="cuda")
        inner = ws[256:256 + nbytes]
        hire.hire_gated_ffn_step(layer, x, out, inner)
        hire.hire_gated_ffn_backward(layer, x, out, dy, grads, inner)
        torch.cuda.synchronize()
        for n, t in big.items():
            assert bool((t[:8] == 7.0).all()) and bool((t[-8:] == 7.0).all()), n
        for t in (ws, saved):
            assert bool((t[:256] == 0x5A).all()) and bool((t[-256:] == 0x5A).all())


@pytest.mark.parametrize("T", [1, 24, 200])
def test_captured_and_replayed(hire, T):
    """Forward and backward in one graph, replayed on new inputs with eager work in between, on a stream of its own."""
    x, wg, wu, w2, dy = inputs(51, T, 264, 520)
    layer = hire.GatedLayer(wg, wu, w2)
    ws = hire.alloc_workspace(max(hire.hire_gated_ffn_workspace_bytes(layer, T),
                                  hire.hire_gated_ffn_backward_workspace_bytes(layer, T)))
    out, grads = hire.GatedOutputs(layer, T, train=True), hire.GatedGradients(layer, T)

    def step():
        hire.hire_gated_ffn_step(layer, x, out, ws)
        hire.hire_gated_ffn_backward(layer, x, out, dy, grads, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (52, 53, 54):
        fresh = inputs(seed, T, 264, 520)
        x.copy_(fresh[0])
        dy.copy_(fresh[4])
        graph.replay()
        torch.cuda.synchronize()
        got = dict(y=out.y.clone(), dx=grads.dx.clone(), dwg=grads.dwg.clone(), dwu=grads.dwu.clone(),
                   dw2u=grads.dw2u.clone())
        eager = run(hire, (x, wg, wu, w2, dy), "silu")
        for n in got:
            assert torch.equal(got[n], eager[n]), n


def test_binding_refuses(hire):
    x, wg, wu, w2, dy = inputs(61, 4, 64, 72)
    layer = hire.GatedLayer(wg, wu, w2)
    out = hire.GatedOutputs(layer, 4)
    ws = hire.alloc_workspace(hire.hire_gated_ffn_workspace_bytes(layer, 4))
    for bad in (x.float(), x.cpu(), x.t().contiguous(), x[:, ::2], torch.cat([x, x])[::2]):
        with pytest.raises(hire.HireError):
            hire.hire_gated_ffn_step(layer, bad, out, ws)
    with pytest.raises(hire.HireError):
        hire.hire_gated_ffn_backward(layer, x, out, dy, hire.GatedGradients(layer, 4), ws)   # nothing was kept
    with pytest.raises(hire.HireError):
        hire.hire_gated_ffn_step(layer, x, out, ws[:256])
    with pytest.raises(hire.HireError):
        hire.GatedLayer(wg, wu, w2, act="tanh")
    with pytest.raises(hire.HireError):
        hire.GatedLayer(wg, wu[:-8], w2)
