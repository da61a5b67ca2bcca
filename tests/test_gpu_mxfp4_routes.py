"""Microscaled products on every route that a call can take: scale bytes at the ends of their range in the weights (0, 1, 254, and 255, which
stands for no number), subnormal weights and tokens, and the tokens shared in LDS over many chunks of columns.  Against the
definition in 64 bits, within n 2^-24 of the sum of the magnitudes, twice (fp32 sums)."""
import pytest
import torch

from test_gpu_mxfp4 import GRID, matrix, power, product_case

pytestmark = pytest.mark.gpu

LARGEST = torch.finfo(torch.bfloat16).max


@pytest.fixture(scope="module")
def hire():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2402_09360_amd import hire as H
    return H


def values(q):
    """What a packed matrix stands for, in 64 bits."""
    table = torch.tensor(GRID + [-g for g in GRID], dtype=torch.float64, device="cuda")
    nibbles = torch.stack((q.codes & 15, q.codes >> 4), dim=2).view(q.rows, q.cols)
    byte = q.scales.long()
    v = table[nibbles.long()].view(q.rows, -1, 32) * power(torch.where(byte == 255, byte * 0, byte) - 127).unsqueeze(2)
    v[byte == 255] = float("nan")
    return v.view(q.rows, q.cols)


# Rows with scale bytes that packing hardly ever or never writes.  tiny: below bf16's normal numbers; huge: +-0.5 and +-1 times
# 2^127; beyond: one value of 6 2^127; strong: 2^98.
def exceptional(hire, rows, cols):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows + cols)
    draw = lambda low, high, *shape: torch.randint(low, high, shape, dtype=torch.uint8, generator=gen, device="cuda")
    codes, scales = draw(0, 256, rows, cols // 2), draw(118, 131, rows, cols // 32)
    kinds = dict(nan=[0, 16, rows - 1, rows - 7], tiny=[1, 17, rows - 2], huge=[2, 18, rows - 3], beyond=[3, 19, rows - 4],
                 strong=[4, 20, rows - 5])
    scales[0, 0] = scales[16, -1] = scales[rows - 1, -1] = scales[rows - 7, cols // 64] = 255
    codes[[0, 16]] = 0   # no number whatever the codes
    for r in kinds["tiny"]:
        scales[r] = draw(0, 2, cols // 32)
    pairs = torch.tensor([0x11, 0x12, 0x21, 0x22, 0x19, 0x91, 0x2A, 0xA2], dtype=torch.uint8, device="cuda")
    for r in kinds["huge"]:
        codes[r] = pairs[draw(0, 8, cols // 2).long()]
        scales[r, 0] = scales[r, -1] = 254
    for r in kinds["beyond"]:
        codes[r, -16:] = 0
        codes[r, -13] = 7
        scales[r, -1] = 254
    for r in kinds["strong"]:
        scales[r] = 225
    return hire.Mxfp4(codes, scales), kinds


ROUTES = [(1, 300, 96, False), (1, 300, 512, False), (1, 300, 1024, False), (1, 300, 2048, False), (1, 300, 4096, False),
          (1, 300, 8192, False), (1, 300, 16416, False), (1, 300, 32800, False),                        # vectors; a list of parts
          (5, 200, 416, False), (20, 200, 416, False), (5, 16400, 96, False), (40, 16400, 96, False), (20, 9000, 416, False),
          (5, 9000, 96, False),                                                                         # tokens from the L2
          (20, 32771, 800, False), (6, 65541, 96, False), (64, 65541, 800, False),                      # tokens shared in LDS
          (9, 8205, 2048, False), (9, 8205, 4096, False), (33, 8205, 2048, False), (20, 8205, 4096, False),
          (20, 16400, 4096, False),                                                                     # streamed rows
          (5, 901, 2048, True), (9, 8205, 4096, True), (40, 901, 2048, True), (40, 9000, 1024, True),   # streamed, packed tokens
          (5, 200, 416, True), (40, 200, 416, True), (5, 16400, 96, True), (40, 9000, 416, True),
          (70, 200, 416, True), (70, 200, 512, True), (200, 4096, 416, True), (9, 65541, 96, True)]     # tiles


@pytest.mark.parametrize("T,rows,cols,packed", ROUTES)
def test_exceptional_scales(hire, T, rows, cols, packed):
    w, kinds = exceptional(hire, rows, cols)
    wv = values(w)
    if not packed:   # the weights are those of hire_unpack_mxfp4
        wv[wv.abs() > LARGEST] = wv[wv.abs() > LARGEST].sign() * float("inf")
    ws = hire.alloc_workspace(hire.hire_mxfp4_product_workspace_bytes(T, rows, cols))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(T)
    # tokens' size, rows whose sums or terms would overflow or vanish with it
    for log2, without in ((-9, ("tiny",)), (100, ("huge", "beyond", "strong")), (-127, ("tiny", None))):
        x = (torch.randn((T, cols), generator=gen, device="cuda", dtype=torch.float64) * 2.0 ** log2).to(torch.bfloat16)
        y = torch.full((T, rows), 7.0, device="cuda")
        if packed:
            xq = hire.hire_pack_mxfp4(x)
            xv = values(xq)
            hire.hire_mxfp4_product(xq, w, y, ws)
        else:
            xv = x.double()
            hire.hire_mxfp4_product_bf16(x, w, y, ws)
        torch.cuda.synchronize()
        keep = torch.ones(rows, dtype=torch.bool, device="cuda")
        if None in without:   # ordinary weights: the sums are subnormal
            keep[:] = False
            for name in ("nan", "huge", "beyond", "strong"):
                keep[kinds[name]] = True
        for name in without:
            if name:
                keep[kinds[name]] = False
        part = wv[keep]
        want, got = xv @ part.t(), y[:, keep].double()
        assert torch.equal(torch.isnan(got), torch.isnan(want)), (log2, "NaN")
        infinite = torch.isinf(want)
        assert torch.equal(torch.isinf(got), infinite) and torch.equal(got[infinite], want[infinite]), (log2, "infinite")
        room = 2.0 * (cols + 8) * 2.0 ** -24 * (xv.abs() @ part.abs().t())
        finite = torch.isfinite(want)
        assert bool(((got - want).abs() <= room)[finite].all()), (log2, float(((got - want).abs() / room)[finite].max()))
        assert bool(torch.isnan(want).any()) and bool(finite.any())


@pytest.mark.parametrize("rows", [32771, 65541])
@pytest.mark.parametrize("cols", [2048, 1056, 800])
def test_shared_tokens(hire, rows, cols):
    """Many chunks of 256 columns, the last one in part, by workgroups of four and of eight groups of rows."""
    for T in (6, 17, 33, 48, 64):
        print(f"T={T} {rows}x{cols}", flush=True)
        product_case(hire, T, rows, cols, False, torch.float32 if T % 2 else torch.bfloat16)


@pytest.mark.parametrize("T,rows", [(6, 65541), (20, 32771), (33, 65541), (64, 32771)])
def test_shared_tokens_with_scales_anywhere(hire, T, rows):
    cols = 2048
    w, x = hire.hire_pack_mxfp4(matrix(rows, rows, cols)), matrix(T, T, cols)
    buffer = torch.full((w.scales.numel() + 1,), 255, dtype=torch.uint8, device="cuda")
    buffer[1:] = w.scales.flatten()
    y = torch.empty((T, rows), device="cuda")
    ws = hire.alloc_workspace(hire.hire_mxfp4_product_workspace_bytes(T, rows, cols))
    hire.hire_mxfp4_product_bf16(x, hire.Mxfp4(w.codes, buffer[1:].view(w.scales.shape)), y, ws)
    wv = values(w)
    room = 2.0 * (cols + 8) * 2.0 ** -24 * (x.double().abs() @ wv.abs().t())
    assert bool(((y.double() - x.double() @ wv.t()).abs() <= room).all())
