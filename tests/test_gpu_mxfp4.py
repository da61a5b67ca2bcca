"""Microscaled 4-bit floating point against its definition in 64 bits: packing code by code, products within the error of
fp32 sums (n 2^-24 of the sum of the magnitudes, twice) and of one rounding of the result."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


@pytest.fixture(scope="module")
def hire():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2402_09360_amd import hire as H
    return H


def power(e):
    """2^e in 64 bits, e whole."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def quantise(w):
    """Codes [rows, cols] and scale bytes by the definition, on the CPU: the nearest grid value, of two the even code."""
    b = w.cpu().double().view(w.shape[0], -1, 32)
    amax = b.abs().amax(dim=2)
    byte = torch.full(amax.shape, 127, dtype=torch.int64)
    for r in range(amax.shape[0]):
        for c in range(amax.shape[1]):
            a = float(amax[r, c])
            if not math.isfinite(a):
                byte[r, c] = 255
            elif a > 0.0:
                byte[r, c] = max(math.frexp(a)[1] - 1 - 2, -127) + 127
    scale = power(torch.where(byte == 255, torch.zeros_like(byte), byte - 127)).unsqueeze(2)
    r = torch.nan_to_num(b.abs() / scale, nan=0.0, posinf=0.0)
    away = (r.unsqueeze(3) - torch.tensor(GRID, dtype=torch.float64)).abs()
    # doubled distance, one more for odd codes: of two equal distances the even code wins; differences are far coarser
    code = (away * 2.0 ** 40 + torch.arange(8, dtype=torch.float64) % 2).argmin(dim=3)
    code = code + 8 * torch.signbit(b).long()
    code[byte == 255] = 0
    return code.view(w.shape[0], -1), byte


def values(code, byte):
    table = torch.tensor(GRID + [-g for g in GRID], dtype=torch.float64)
    v = table[code].view(code.shape[0], -1, 32) * power(torch.where(byte == 255, torch.zeros_like(byte), byte) - 127).unsqueeze(2)
    v[byte == 255] = float("nan")
    return v.view(code.shape)


def nibbles(codes):
    c = codes.cpu().long()
    return torch.stack((c & 15, c >> 4), dim=2).view(c.shape[0], -1)


def matrix(seed, rows, cols, spread=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    w = torch.randn((rows, cols), generator=gen, device="cuda")
    return (w * torch.exp(spread * torch.randn((rows, cols // 32, 1), generator=gen, device="cuda")).expand(
        rows, cols // 32, 32).reshape(rows, cols)).to(torch.bfloat16)


@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 64), (5, 96), (64, 2048), (129, 416), (1000, 32), (7, 8192)])
def test_packing(hire, rows, cols):
    print(f"pack {rows} x {cols}", flush=True)
    w = matrix(rows + cols, rows, cols, spread=3.0)
    packed = hire.hire_pack_mxfp4(w)
    code, byte = quantise(w)
    assert torch.equal(packed.scales.cpu().long(), byte) and torch.equal(nibbles(packed.codes), code)
    assert torch.equal(hire.hire_unpack_mxfp4(packed).cpu().double(), values(code, byte))


def test_packing_every_value(hire):
    """Every finite bf16 in blocks of its own largest magnitude: both signs, subnormals, zeros, half steps."""
    bits = torch.arange(65536, dtype=torch.int32)
    bits = bits[(bits & 0x7F80) != 0x7F80]
    w = torch.zeros((bits.numel(), 32), dtype=torch.int16)
    w[:, 5] = bits.to(torch.int16)
    for i, step in enumerate((0, 1, 2, 64, 128, 192, 256, 300, 384)):   # smaller neighbours
        w[:, 10 + i] = torch.clamp((bits & 0x7FFF) - step, min=0).to(torch.int16)
    w = w.view(torch.bfloat16).cuda()
    packed = hire.hire_pack_mxfp4(w)
    amax = w.cpu().double().abs().amax(dim=1)
    byte = torch.clamp(torch.frexp(amax)[1].long() - 3, min=-127) + 127
    byte[amax == 0] = 127
    assert torch.equal(packed.scales.cpu().long()[:, 0], byte)
    scale = power(byte - 127).unsqueeze(1)
    r = w.cpu().double().abs() / scale
    got = torch.tensor(GRID, dtype=torch.float64)[nibbles(packed.codes) & 7]
    nearest = (r.unsqueeze(2) - torch.tensor(GRID, dtype=torch.float64)).abs().amin(dim=2)
    assert torch.equal((r - got).abs(), nearest)
    tie = (r.unsqueeze(2) - torch.tensor(GRID, dtype=torch.float64)).abs() == nearest.unsqueeze(2)
    odd = (nibbles(packed.codes) & 1) == 1
    assert not bool((odd & (tie.sum(dim=2) > 1)).any())
    assert torch.equal((nibbles(packed.codes) >> 3) == 1, torch.signbit(w.cpu()))
    assert torch.equal(hire.hire_unpack_mxfp4(packed).cpu().double().abs(), got * scale)


def test_blocks_without_a_number(hire):
    w = matrix(3, 6, 128)
    w[1, 40], w[2, 3], w[4, 100] = float("inf"), float("nan"), float("-inf")
    packed = hire.hire_pack_mxfp4(w)
    code, byte = quantise(w)
    assert torch.equal(packed.scales.cpu().long(), byte) and torch.equal(nibbles(packed.codes), code)
    back = hire.hire_unpack_mxfp4(packed).cpu().double()
    assert torch.equal(torch.isnan(back), torch.isnan(values(code, byte)))
    assert torch.equal(torch.nan_to_num(back), torch.nan_to_num(values(code, byte)))
    other = hire.hire_pack_mxfp4(matrix(4, 5, 128))
    for T in (5, 70):
        x = matrix(5, T, 128)
        ws = hire.alloc_workspace(hire.hire_mxfp4_product_workspace_bytes(T, 6, 128))
        y = torch.zeros((T, 6), device="cuda")
        hire.hire_mxfp4_product(hire.hire_pack_mxfp4(x), packed, y, ws)
        assert torch.equal(torch.isnan(y).cpu(), torch.tensor([False, True, True, False, True, False]).expand(T, 6))
    y = torch.zeros((5, 6), device="cuda")
    hire.hire_mxfp4_product_bf16(x[:5].contiguous(), packed, y, ws)
    assert torch.equal(torch.isnan(y).cpu(), torch.tensor([False, True, True, False, True, False]).expand(5, 6))
    assert bool(torch.isfinite(hire.hire_unpack_mxfp4(other)).all())


def test_outer_scales(hire):
    """Scale bytes that packing never writes: 0 with small codes, up to 254; magnitudes beyond bf16 become infinite."""
    byte = torch.arange(256, dtype=torch.uint8).view(8, 32)
    codes = torch.arange(16, dtype=torch.uint8).repeat(8, 32)
    packed = hire.Mxfp4(codes.view(8, 512).cuda().contiguous(), byte.cuda())
    want = values(nibbles(packed.codes), byte.long())
    largest = torch.finfo(torch.bfloat16).max
    want[want.abs() > largest] = want[want.abs() > largest].sign() * float("inf")
    got = hire.hire_unpack_mxfp4(packed).cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got, nan=0.0), torch.nan_to_num(want, nan=0.0))


def product_case(hire, T, rows, cols, packed_tokens, dtype, seed=0):
    w, x = matrix(seed + rows, rows, cols), matrix(seed + T, T, cols)
    wq = hire.hire_pack_mxfp4(w)
    xq = hire.hire_pack_mxfp4(x) if packed_tokens else None
    lead = 16 // dtype.itemsize   # 16 bytes in
    big = torch.full((T * rows + 2 * lead,), 7.0, dtype=dtype, device="cuda")
    y = big[lead:lead + T * rows].view(T, rows)
    ws = hire.alloc_workspace(hire.hire_mxfp4_product_workspace_bytes(T, rows, cols))
    if packed_tokens:
        hire.hire_mxfp4_product(xq, wq, y, ws)
    else:
        hire.hire_mxfp4_product_bf16(x, wq, y, ws)
    torch.cuda.synchronize()
    xv = hire.hire_unpack_mxfp4(xq).double() if packed_tokens else x.double()
    wv = hire.hire_unpack_mxfp4(wq).double()
    want = xv @ wv.t()
    bound = 2.0 * (cols + 8) * 2.0 ** -24 * (xv.abs() @ wv.abs().t()) + want.abs() * torch.finfo(dtype).eps / 2
    over = (y.double() - want).abs() - 1.01 * bound
    assert bool((over <= 0).all()), (T, rows, cols, float(over.max()))
    assert bool((big[:lead] == 7.0).all()) and bool((big[lead + T * rows:] == 7.0).all())


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 32, 33, 48, 49, 64])
@pytest.mark.parametrize("packed", [False, True])
def test_few_tokens(hire, T, packed):
    for rows, cols in ((1, 32), (17, 96), (100, 160), (333, 2048), (64, 544)):
        print(f"T={T} {rows}x{cols} packed={packed}", flush=True)
        product_case(hire, T, rows, cols, packed, torch.float32 if T % 2 else torch.bfloat16)


@pytest.mark.parametrize("T,rows,cols", [
    (65, 1, 32), (65, 33, 64), (100, 257, 224), (128, 128, 256), (129, 300, 2080), (255, 511, 288), (256, 256, 512),
    (257, 1000, 96), (700, 77, 4096), (1021, 516, 1312)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_tokens(hire, T, rows, cols, dtype):
    print(f"T={T} {rows}x{cols}", flush=True)
    product_case(hire, T, rows, cols, True, dtype)


@pytest.mark.parametrize("T,rows,cols", [(65, 1, 4128), (100, 257, 8224), (300, 40, 16384), (1021, 77, 8192), (130, 512, 2048)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_products_in_parts(hire, T, rows, cols, dtype):
    """Few tiles of long rows."""
    print(f"T={T} {rows}x{cols}", flush=True)
    product_case(hire, T, rows, cols, True, dtype)


@pytest.mark.parametrize("rows,cols", [(16397, 1024), (10923, 1536), (8205, 2048), (5001, 4096), (8200, 8192), (13500, 5120),
                                       (901, 2048), (1999, 7168)])
@pytest.mark.parametrize("T,packed", [(2, False), (9, False), (16, False), (31, False), (33, False), (64, False), (1, True), (16, True), (32, True), (47, True),
                                      (64, True)])
def test_streamed_rows(hire, T, packed, rows, cols):
    print(f"T={T} {rows}x{cols} packed={packed}", flush=True)
    product_case(hire, T, rows, cols, packed, torch.float32 if T % 2 else torch.bfloat16)


def test_scales_that_start_anywhere(hire):
    """The same results, up to the order of the sums, from scale bytes at any address."""
    rows, cols = 5000, 4096
    wq = hire.hire_pack_mxfp4(matrix(1, rows, cols))
    wv = hire.hire_unpack_mxfp4(wq).double()
    for T, packed in ((3, False), (20, False), (64, False), (3, True), (30, True), (64, True), (100, True)):
        x = matrix(T, T, cols)
        xq = hire.hire_pack_mxfp4(x)
        xv = hire.hire_unpack_mxfp4(xq).double() if packed else x.double()
        want, room = xv @ wv.t(), 2.02 * (cols + 8) * 2.0 ** -24 * (xv.abs() @ wv.abs().t())
        for at in (0, 1, 4, 8):
            def moved(q):
                buffer = torch.zeros(q.scales.numel() + 16, dtype=torch.uint8, device="cuda")
                buffer[at:at + q.scales.numel()] = q.scales.flatten()
                return hire.Mxfp4(q.codes, buffer[at:at + q.scales.numel()].view(q.scales.shape))
            y = torch.empty((T, rows), device="cuda")
            ws = hire.alloc_workspace(hire.hire_mxfp4_product_workspace_bytes(T, rows, cols))
            if packed:
                hire.hire_mxfp4_product(moved(xq), moved(wq), y, ws)
            else:
                hire.hire_mxfp4_product_bf16(x, moved(wq), y, ws)
            assert bool(((y.double() - want).abs() <= room).all()), (T, packed, at)


@pytest.mark.parametrize("rows,cols", [(40000, 256), (33000, 96), (3, 65536)])
def test_long_matrices(hire, rows, cols):
    for T, packed in ((1, False), (1, True), (20, False), (64, False), (50, True)):
        print(f"T={T} {rows}x{cols} packed={packed}", flush=True)
        product_case(hire, T, rows, cols, packed, torch.float32)


@pytest.mark.parametrize("T,packed", [(1, False), (40, True), (300, True)])
def test_captured_and_replayed(hire, T, packed):
    x, wq = matrix(7, T, 512), hire.hire_pack_mxfp4(matrix(8, 700, 512))
    xq = hire.Mxfp4.empty(T, 512)
    y = torch.empty((T, 700), device="cuda")
    ws = hire.alloc_workspace(hire.hire_mxfp4_product_workspace_bytes(T, 700, 512))

    def step():
        if packed:
            hire.hire_pack_mxfp4(x, out=xq)
            hire.hire_mxfp4_product(xq, wq, y, ws)
        else:
            hire.hire_mxfp4_product_bf16(x, wq, y, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (9, 10, 11):
        x.copy_(matrix(seed, T, 512))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        y.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, y)


def test_binding_refuses(hire):
    w = matrix(1, 64, 128)
    wq = hire.hire_pack_mxfp4(w)
    x, y = matrix(2, 4, 128), torch.empty((4, 64), device="cuda")
    ws = hire.alloc_workspace(hire.hire_mxfp4_product_workspace_bytes(4, 64, 128))
    for call in (lambda: hire.hire_pack_mxfp4(w.float()), lambda: hire.hire_pack_mxfp4(w[:, :48].contiguous()),
                 lambda: hire.hire_pack_mxfp4(w.t()), lambda: hire.hire_pack_mxfp4(w, out=hire.Mxfp4.empty(64, 96)),
                 lambda: hire.Mxfp4.empty(4, 33), lambda: hire.Mxfp4(wq.codes, wq.scales[:, :3].contiguous()),
                 lambda: hire.Mxfp4(wq.codes.cpu(), wq.scales.cpu()),
                 lambda: hire.hire_unpack_mxfp4(wq, out=torch.empty((64, 128), device="cuda")),
                 lambda: hire.hire_mxfp4_product_bf16(x.float(), wq, y, ws),
                 lambda: hire.hire_mxfp4_product_bf16(x, wq, y.half(), ws),
                 lambda: hire.hire_mxfp4_product_bf16(x, wq, y[:3], ws),
                 lambda: hire.hire_mxfp4_product_bf16(matrix(3, 65, 128), wq, torch.empty((65, 64), device="cuda"), ws),
                 lambda: hire.hire_mxfp4_product(hire.Mxfp4.empty(4, 96), wq, y, ws),
                 lambda: hire.hire_mxfp4_product_bf16(x, wq, y, ws[:0])):
        with pytest.raises(hire.HireError):
            call()
