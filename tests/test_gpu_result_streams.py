"""Results that a call allocates itself belong to the stream it is given: memory that the current stream's work may still use is
not handed to another stream."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hire():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2402_09360_amd import hire as H
    return H


def freed(shapes):
    """Addresses of blocks of the current stream that were given back a moment ago."""
    torch.cuda.synchronize()
    blocks = [torch.empty(shape, dtype=dtype, device="cuda") for shape, dtype in shapes]
    return {t.data_ptr() for t in blocks}


def test_packing_and_reading_back(hire):
    rows, cols = 4096, 2048   # 4 MiB of codes: a block of its own
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    w = torch.randn((rows, cols), generator=gen, device="cuda").to(torch.bfloat16)
    want = hire.hire_pack_mxfp4(w)
    values = hire.hire_unpack_mxfp4(want)
    side = torch.cuda.Stream()
    old = freed([((rows, cols // 2), torch.uint8), ((rows, cols // 32), torch.uint8)])
    got = hire.hire_pack_mxfp4(w, stream=side)
    assert got.codes.data_ptr() not in old and got.scales.data_ptr() not in old
    old = freed([((rows, cols), torch.bfloat16)])
    back = hire.hire_unpack_mxfp4(got, stream=side)
    assert back.data_ptr() not in old
    torch.cuda.synchronize()
    assert torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales) and torch.equal(back, values)
    old = freed([((rows, cols), torch.bfloat16)])   # on the current stream they are used again
    assert hire.hire_unpack_mxfp4(got).data_ptr() in old


def test_selection(hire):
    """Outputs and the workspace of a call that makes its own, which is initialised on the stream that uses it."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    scores = torch.randn((64, 40000), generator=gen, device="cuda")
    want = hire.topk_select(scores, 20000)
    side = torch.cuda.Stream()
    old = freed([((64, 20000), torch.int32), ((64, 20000), torch.float32)])
    side.wait_stream(torch.cuda.current_stream())
    idx, val = hire.topk_select(scores, 20000, stream=side)
    assert idx.data_ptr() not in old and val.data_ptr() not in old
    torch.cuda.synchronize()
    assert torch.equal(idx, want[0]) and torch.equal(val, want[1])


def test_int4_packing(hire):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    w = torch.randn((4096, 2048), generator=gen, device="cuda").to(torch.bfloat16)
    want = hire.hire_pack_int4(w)
    codes = hire.hire_unpack_int4(want[0], 4096, 2048)
    side = torch.cuda.Stream()
    old = freed([(want[0].shape, torch.uint8), ((4096,), torch.float32)])
    blob, scale = hire.hire_pack_int4(w, stream=side)
    assert blob.data_ptr() not in old and scale.data_ptr() not in old
    old = freed([((4096, 2048), torch.int8)])
    back = hire.hire_unpack_int4(blob, 4096, 2048, stream=side)
    assert back.data_ptr() not in old
    torch.cuda.synchronize()
    assert torch.equal(blob, want[0]) and torch.equal(scale, want[1]) and torch.equal(back, codes)
