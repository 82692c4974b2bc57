"""What the serving calls take and refuse beside their sizes: the leading dimension of a single row, packed buffers of another weight, codes of
more than four bits."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


def _packed(torch, cafeq, rows, cols, group=32):
    codes = torch.randint(-8, 8, (rows, cols), device="cuda:0", dtype=torch.int8)
    return cafeq.pack_nibbles(codes, torch.rand((rows, cols // group), device="cuda:0"), group)


def _one_row(torch, dtype, cols, ld):
    """A row of `cols` that is a slice of a buffer with rows of `ld`."""
    x = torch.randn((1, cols), device="cuda:0").to(dtype)
    buf = torch.zeros((1, ld), device="cuda:0", dtype=dtype)
    buf[:, :cols] = x
    view = buf.as_strided((1, cols), (ld, 1))
    assert view.stride(0) == ld
    return x, view


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ld", [65, 100, (1 << 24) + 3])
def test_products_of_one_row_take_any_leading_dimension(env, dtype, ld):
    torch, cafeq = env
    packed = _packed(torch, cafeq, 40, 64)
    x, view = _one_row(torch, torch.float32 if dtype == "f32" else torch.bfloat16, 64, ld)
    assert torch.equal(cafeq.infer_packed(view, packed), cafeq.infer_packed(x, packed))


def test_the_last_token_of_a_long_prompt(env):
    torch, cafeq = env
    h = torch.randn((1, 4097, 4608), device="cuda:0", dtype=torch.bfloat16)     # rows 18.9 M elements apart, were there two
    packed = _packed(torch, cafeq, 40, 4608)
    assert torch.equal(cafeq.infer_packed(h[:, -1], packed), cafeq.infer_packed(h[:, -1].clone(), packed))
    P = torch.linalg.qr(torch.randn((36, 128, 128)))[0].contiguous().cuda()
    a, b = cafeq.norm_quantize(h[:, -1], Tinv=P, group=128), cafeq.norm_quantize(h[:, -1].clone(), Tinv=P, group=128)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)


@pytest.mark.parametrize("k", [0, 32])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norms_of_one_row_take_any_leading_dimension(env, dtype, k):
    torch, cafeq = env
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    P = torch.linalg.qr(torch.randn((3, 32, 32)))[0].contiguous().cuda() if k else None
    (x, xv), (r, rv), (_, sv) = (_one_row(torch, t, 96, ld) for ld in (97, 111, 1000))
    want = cafeq.norm_quantize(x, residual=r, Tinv=P, group=32, values=torch.bfloat16)
    got = cafeq.norm_quantize(xv, residual=rv, Tinv=P, group=32, values=torch.bfloat16, sum_out=sv)
    assert got.sum is sv
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("n", [1, 4])
def test_packed_buffers_that_do_not_fit_are_refused(env, n):
    torch, cafeq = env
    packed = _packed(torch, cafeq, 40, 64)
    x = torch.ones((n, 64), device="cuda:0")
    full = packed.data
    for data in (full[:-16], full[:0], torch.cat((full, full)), full.view(torch.float32), torch.cat((full, full))[::2]):
        with pytest.raises(cafeq.CafeqError):
            cafeq.infer_packed(x, packed._replace(data=data))
    for rows, group in ((100, 32), (40, 0), (40, 48), (-1, 32)):
        with pytest.raises(cafeq.CafeqError):
            cafeq.infer_packed(x, packed._replace(rows=rows, group=group))
    assert torch.equal(cafeq.infer_packed(x, packed._replace(data=full.clone())), cafeq.infer_packed(x, packed))


@pytest.mark.parametrize("bits", [5, 8])
def test_codes_of_more_than_four_bits_are_refused(env, bits):
    torch, cafeq = env
    W = torch.randn((40, 64), device="cuda:0")
    codes, scales, _ = cafeq.rtn_quantize(W, bits, 32)
    with pytest.raises(cafeq.CafeqError):
        cafeq.pack_nibbles(codes, scales, 32)
    codes, scales, _ = cafeq.rtn_quantize(W, 4, 32)
    for low, high, good in ((-8, 7, True), (-9, 0, False), (0, 8, False)):
        codes[3, 5], codes[39, 63] = low, high
        if good:
            cafeq.pack_nibbles(codes, scales, 32)
        else:
            with pytest.raises(cafeq.CafeqError):
                cafeq.pack_nibbles(codes, scales, 32)


def test_packing_in_a_captured_graph(env):
    torch, cafeq = env
    codes, scales, _ = cafeq.rtn_quantize(torch.randn((40, 64), device="cuda:0"), 4, 32)
    cafeq.pack_nibbles(codes, scales, 32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = cafeq.pack_nibbles(codes, scales, 32)
    x = torch.randn((2, 64), device="cuda:0")
    for _ in range(3):
        codes.copy_(torch.randint(-8, 8, (40, 64), device="cuda:0", dtype=torch.int8))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(cafeq.infer_packed(x, held), cafeq.infer_packed(x, cafeq.pack_nibbles(codes, scales, 32)))
