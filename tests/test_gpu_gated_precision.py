"""The dense gated FFN of up to sixteen tokens holds h, dg and du in two terms, sixteen bits of significand together: results are the
definition's values rounded once, but where one lies within the small error of these terms from a rounding border."""
import pytest
import torch

from test_gpu_gated_ffn import expected, inputs, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hire():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2402_09360_amd import hire as H
    return H


# layers in one kernel and in two, rows in registers and streamed, in parts of d and of the rows
@pytest.mark.parametrize("T,d,F,act", [(1, 256, 1024, "silu"), (3, 264, 328, "gelu"), (16, 512, 2048, "relu"), (16, 1024, 4096, "gelu"),
                                       (9, 800, 6008, "silu"), (4, 4096, 8192, "silu"), (16, 2048, 16384, "gelu"),
                                       (12, 8192, 4104, "silu"), (1, 2048, 20000, "gelu")])
def test_rounded_once(hire, T, d, F, act):
    """Rounded to one bf16 term, h (or dg and du) is off by about 0.4 2^-8 of its value, and so is a sum of many, while a result's
    rounding step is 2^-8 to 2^-7 of it: a quarter to two fifths of the results would come out as a neighbour.  Two terms, and g and u kept in 24
    bits, are off by 2^-15 at most: less than one in a hundred.  Two in a hundred are allowed."""
    print(T, d, F, act, flush=True)
    wrong = dict(y=0, dx=0, dwg=0, dwu=0, dw2u=0)
    count = dict.fromkeys(wrong, 0)
    for seed in range(4):
        data = inputs(100 * seed + T, T, d, F, exact=act == "relu")
        got, want = run(hire, data, act), expected(*data, act)
        for name in wrong:
            wrong[name] += int((got[name] != want[name][0].to(torch.bfloat16)).sum())
            count[name] += got[name].numel()
    print({name: round(n / count[name], 4) for name, n in wrong.items()}, flush=True)
    assert all(n <= 0.02 * count[name] for name, n in wrong.items()), (wrong, count)


@pytest.mark.parametrize("T,d,F", [(1, 256, 1024), (5, 1024, 8192), (16, 4096, 8192)])
def test_infinite_hidden_values(hire, T, d, F):
    """h beyond the type's range: the sums are infinite, as the definition's, and no NaN."""
    x = torch.full((T, d), 2.0 ** 40, device="cuda", dtype=torch.bfloat16)
    w = torch.full((F, d), 2.0 ** 30, device="cuda", dtype=torch.bfloat16)
    v = torch.full((F, d), 0.5, device="cuda", dtype=torch.bfloat16)
    y = run(hire, (x, w, w, v, torch.zeros_like(x)), "relu", train=False)["y"]
    assert bool((y == float("inf")).all())


@pytest.mark.parametrize("T,d,F", [(1, 256, 1024), (7, 512, 9000), (5, 1024, 8192), (16, 4096, 8192)])
def test_infinite_factors(hire, T, d, F):
    """One infinite weight, one infinite output gradient: what they meet is infinite of h's sign, not NaN, as in one term."""
    x, wg, wu, w2, dy = inputs(T, T, d, F)
    unit, column = F // 3, d // 2
    w2[unit, column] = float("inf")
    token = T - 1
    got = run(hire, (x, wg, wu, w2, torch.zeros_like(dy)), "silu", train=False)["y"]
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    h = g * torch.sigmoid(g) * u
    assert bool((h[:, unit] != 0).all())
    assert torch.equal(got[:, column].double(), torch.sign(h[:, unit]) * float("inf"))
    others = torch.arange(d, device="cuda") != column
    assert bool(torch.isfinite(got[:, others]).all())
    w2[unit, column] = 1.0
    dy[token, column] = float("-inf")
    got = run(hire, (x, wg, wu, w2, dy), "silu")["dw2u"]
    assert torch.equal(got[:, column].double(), torch.sign(h[token]) * float("-inf"))
    assert bool(torch.isfinite(got[:, others]).all())
