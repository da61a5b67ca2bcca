"""The dense gated FFN where a part of its operands lies beyond 4 GiB, and at its largest sizes block by block: a tile that is
missing or misplaced shows, which a norm over a million rows would not."""
import pytest
import torch

from test_gpu_gated_ffn import SECOND, expected

pytestmark = pytest.mark.gpu

ROUND = 2.0 ** -8   # half a step of bf16


@pytest.fixture(scope="module")
def hire():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2402_09360_amd import hire as H
    return H


def drawer(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return lambda *shape, std=1.0: (torch.randn(shape, generator=gen, device="cuda") * std).to(torch.bfloat16)


def run(hire, x, wg, wu, w2, dy, act):
    """All outputs, each filled with NaN in front of the calls."""
    layer, T = hire.GatedLayer(wg, wu, w2, act=act), x.shape[0]
    out, grads = hire.GatedOutputs(layer, T, train=True), hire.GatedGradients(layer, T)
    for t in (out.y, grads.dx, grads.dwg, grads.dwu, grads.dw2u):
        t.fill_(float("nan"))
    ws = hire.alloc_workspace(max(hire.hire_gated_ffn_workspace_bytes(layer, T),
                                  hire.hire_gated_ffn_backward_workspace_bytes(layer, T)))
    hire.hire_gated_ffn_step(layer, x, out, ws)
    hire.hire_gated_ffn_backward(layer, x, out, dy, grads, ws)
    torch.cuda.synchronize()
    return dict(y=out.y, dx=grads.dx, dwg=grads.dwg, dwu=grads.dwu, dw2u=grads.dw2u)


def within(got, want, name):
    value, bound = want[name]
    over = (got.double() - value).abs() - SECOND * bound
    assert bool((over <= 2.0 ** -120).all()), (name, float(over.max()), float(value.abs().max()))


@pytest.mark.parametrize("T,d,F,act", [(140000, 64, 16384, "silu"), (1 << 20, 2304, 64, "gelu")])
def test_gradients_from_tokens_beyond_4_gib(hire, T, d, F, act):
    """Only the last tokens have an output gradient, so the weights' gradients are theirs alone: the planes, or x and dy, are read
    beyond 4 GiB for them, and a place that wrapped would give zeros."""
    print(T, d, F, flush=True)
    last = 300
    draw = drawer(T + d)
    wg, wu, w2 = draw(F, d, std=d ** -0.5), draw(F, d, std=d ** -0.5), draw(F, d, std=F ** -0.5)
    x = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    for i in range(0, T, 1 << 16):
        x[i:i + (1 << 16)] = draw(min(1 << 16, T - i), d)
    dy = torch.zeros_like(x)
    dy[-last:] = draw(last, d)
    got = run(hire, x, wg, wu, w2, dy, act)
    want = expected(x[-last:], wg, wu, w2, dy[-last:], act)
    for name in ("dwg", "dwu", "dw2u"):
        within(got[name], want, name)
    within(got["y"][-last:], want, "y")
    within(got["dx"][-last:], want, "dx")
    assert bool((got["dx"][:-last] == 0).all()) and bool(torch.isfinite(got["y"]).all())


@pytest.mark.parametrize("T", [1, 40, 100])
def test_units_beyond_4_gib(hire, T):
    """All units but the last are zero: y, dx and the last units' gradients are those of a layer of the last units alone."""
    d, F, last = 2304, 1 << 20, 256
    print(T, flush=True)
    draw = drawer(T)
    x, dy = draw(T, d), draw(T, d)
    mats = [torch.zeros((F, d), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    for m, std in zip(mats, (d ** -0.5, d ** -0.5, last ** -0.5)):
        m[-last:] = draw(last, d, std=std)
    got = run(hire, x, *mats, dy, "silu")
    want = expected(x, *[m[-last:] for m in mats], dy, "silu")
    within(got["y"], want, "y")
    within(got["dx"], want, "dx")
    for name in ("dwg", "dwu", "dw2u"):
        within(got[name][-last:], want, name)
        assert bool((got[name][:-last] == 0).all()), name


@pytest.mark.parametrize("T,d,F", [(1 << 20, 8, 8), (1, 1 << 20, 8), (20, 1 << 20, 8), (70, 1 << 20, 8), (1, 8, 1 << 20),
                                   (64, 8, 1 << 20), (70, 8, 1 << 20)])
def test_largest_sizes_block_by_block(hire, T, d, F):
    """Norms of blocks of 128 along the longest axis.  A result and each factor of its sum are rounded to bf16 at most once, each off by
    at most 2^-8 of its value.  A factor's error passes to a block of 128 through a random matrix of 8 or 16 by 128, whose largest and
    smallest singular values are about sqrt(128) + 4 and sqrt(128) - 4, a factor of 2.1.  fp32 sums of a million terms are off by far
    less than 2^-8 of their norm.  In all below (1 + 2.1) 2^-8; 4 2^-8 is allowed."""
    print(T, d, F, flush=True)
    draw = drawer(T + d + F + 1)
    x, wg, wu, w2, dy = draw(T, d), draw(F, d, std=d ** -0.5), draw(F, d, std=d ** -0.5), draw(F, d, std=F ** -0.5), draw(T, d)
    got = run(hire, x, wg, wu, w2, dy, "silu")
    want = {name: value for name, (value, _) in expected(x, wg, wu, w2, dy, "silu").items()}
    for name, t in got.items():
        assert bool(torch.isfinite(t).all()), name
        a, b = t.double(), want[name]
        axis = 0 if b.shape[0] >= b.shape[1] else 1
        if b.shape[axis] % 128 == 0:
            a, b = a.unflatten(axis, (-1, 128)), b.unflatten(axis, (-1, 128))
            rest = tuple(i for i in range(3) if i != axis)
            error, norm = (a - b).pow(2).sum(rest).sqrt(), b.pow(2).sum(rest).sqrt()
        else:
            error, norm = (a - b).norm(), b.norm()
        assert bool((error <= 4 * ROUND * norm).all()), (name, float((error / norm).max()))
