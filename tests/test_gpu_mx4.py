"""4-bit matrices on the GPU against their 64-bit references."""
import pytest
import torch

from paper_2511_12934_b200 import binding as B
from tests import mx4_reference as R

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16]


def spread_rows(rows, cols, dtype, seed):
    """Rows whose blocks differ in magnitude by many powers of two, with zero blocks and values next to the midpoints."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-20, 20, (rows, cols // 32), generator=g).double()).repeat_interleave(32, 1)
    x.view(-1)[::7] = 0
    x[:, :32][::3] = 0
    if rows > 1:
        x[1, :11] = torch.tensor([6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -5.0, -0.25, 7.99])
    return x.to(dtype).cuda()


def unpacked(m):
    codes = torch.stack((m.codes & 15, m.codes >> 4), -1).flatten(-2)
    return codes, m.scales.cpu()[R.scale_places(m.rows, m.cols // 32)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, cols", [(1, 32), (2, 64), (7, 96), (127, 160), (128, 128), (129, 2816), (300, 32), (1000, 512)])
def test_quantise_and_back(rows, cols, dtype):
    x = spread_rows(rows, cols, dtype, rows + cols)
    m = B.mx4_quantize(x)
    value, code, byte = R.quantise(x)
    got_code, got_byte = unpacked(m)
    assert torch.equal(got_byte, byte.cpu()) and torch.equal(got_code, code)
    out = torch.full_like(x, 9.0)
    assert torch.equal(B.mx4_dequantize(m, out).double(), value)   # two bits and a power of two: exact in either type
    # bytes of rows and blocks that only fill up a tile are the smallest scale
    filled = torch.zeros(m.scales.numel(), dtype=torch.bool)
    filled[R.scale_places(rows, cols // 32).flatten()] = True
    assert not m.scales.cpu()[~filled].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_blocks_with_infinities_read_as_nan(dtype, bad):
    x = torch.randn(5, 96, device="cuda").to(dtype)
    x[2, 40] = bad
    out = B.mx4_dequantize(B.mx4_quantize(x), torch.empty_like(x))
    assert torch.isnan(out[2, 32:64]).all()
    out[2, 32:64] = 0
    assert not torch.isnan(out).any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_smallest_and_largest_magnitudes(dtype):
    tiny = 2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -149
    x = torch.zeros(4, 32, dtype=torch.float64)
    x[0], x[1, :3], x[2, :2], x[3, 0] = tiny, torch.tensor([2.0 ** -126, 2.0 ** -128, -2.0 ** -127]), torch.tensor([2.0 ** 127 * 1.5, -2.0 ** 126]), -0.0
    x = x.to(dtype).cuda()
    out = B.mx4_dequantize(B.mx4_quantize(x), torch.empty_like(x))
    assert torch.equal(out.double(), R.quantise(x)[0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shift, pad", [(0, 8), (1, 0), (1, 3), (4, 4)])
def test_strides_and_alignment(dtype, shift, pad):
    rows, cols = 70, 64
    store = torch.randn(rows * (cols + pad) + shift, device="cuda").to(dtype)
    x = store[shift:].view(rows, cols + pad)[:, :cols]
    a, b = B.mx4_quantize(x), B.mx4_quantize(x.contiguous())
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    back = torch.full_like(store, 3.0)
    out = back[shift:].view(rows, cols + pad)[:, :cols]
    B.mx4_dequantize(a, out)
    assert torch.equal(out.double(), R.quantise(x)[0])
    out.fill_(3.0)
    assert (back == 3.0).all()   # nothing but the rows was written


def product_bound(x, w, ref, bias, dtype):
    """fp32 sums of exact products: every addition off by at most 2^-23 of the magnitudes so far (bias included); then one rounding to the type."""
    k = x.shape[1]
    mass = x.abs() @ w.abs().T + (0 if bias is None else bias.abs())
    return (k + 1) * 2.0 ** -23 * mass + (1.01 * 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23) * ref.abs() + 1e-30


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, k, n", [(1, 32, 1), (1, 64, 8), (7, 96, 33), (128, 256, 128), (129, 288, 130), (77, 2816, 1024), (300, 512, 520), (2000, 1024, 256), (20000, 160, 72)])
@pytest.mark.parametrize("relu, with_bias", [(False, True), (True, False), (True, True)])
def test_linear(m, k, n, dtype, relu, with_bias):
    g = torch.Generator().manual_seed(m + k + n)
    x = (torch.randn(m, k, generator=g) * 0.05).to(dtype).cuda()
    w = (torch.randn(n, k, generator=g) * 0.1).cuda()
    bias = torch.randn(n, generator=g).cuda() * 0.02 if with_bias else None
    xv, wv = R.quantise(x)[0], R.quantise(w)[0]
    ref = xv @ wv.T + (0 if bias is None else bias.double())
    bound = product_bound(xv, wv, ref, None if bias is None else bias.double(), dtype)
    if relu:
        ref = ref.clamp(min=0)
    out = torch.full((m, n), 7.0, dtype=dtype, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    w4 = B.mx4_quantize(w)
    B.mx4_linear(x, w4, out, bias=bias, relu=relu, status=status)
    assert ((out.double() - ref).abs() <= bound).all() and status.item() == 0
    again = torch.empty_like(out)
    B.mx4_linear(B.mx4_quantize(x), w4, again, bias=bias, relu=relu)   # quantised beforehand: the same bits
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, k, n", [(1, 32, 1), (300, 128, 256), (1000, 96, 33), (40000, 160, 129), (37888, 512, 256), (40001, 1024, 128), (70000, 64, 8), (38000, 1088, 200), (45000, 288, 72)])
def test_rows_quantised_within_the_product(m, k, n, dtype):
    """Rows as they are and rows quantised before give the same bits, whichever kernels do it; another product on the stream right behind."""
    x = (torch.randn(m, k, device="cuda") * 0.1).to(dtype)
    x[m // 2, 5] = float("inf")
    w, b = B.mx4_quantize(torch.randn(n, k, device="cuda")), torch.randn(n, device="cuda")
    first, second = (torch.full((m, n), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mx4_linear(x, w, first, bias=b, status=status)
    B.mx4_linear(x, w, second, bias=b, status=status)
    want = B.mx4_linear(B.mx4_quantize(x), w, torch.empty_like(first), bias=b, status=status)
    rest = torch.arange(m, device="cuda") != m // 2
    assert torch.equal(first[rest], want[rest]) and torch.equal(second[rest], want[rest])
    assert torch.isnan(first[m // 2]).all() and torch.isnan(want[m // 2]).all() and status.item() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n, pad, shift", [(40, 24, 0), (40, 3, 0), (33, 31, 0), (64, 8, 1), (130, 62, 8)])
def test_linear_output_strides(dtype, n, pad, shift):
    m, k = 150, 64
    x, w = torch.randn(m, k, device="cuda").to(dtype), torch.randn(n, k, device="cuda")
    store = torch.full((m * (n + pad) + shift,), 5.0, dtype=dtype, device="cuda")
    out = store[shift:].view(m, n + pad)[:, :n]
    B.mx4_linear(x, B.mx4_quantize(w), out)
    dense = B.mx4_linear(x, B.mx4_quantize(w), torch.empty(m, n, dtype=dtype, device="cuda"))
    assert torch.equal(out, dense)
    out.fill_(5.0)
    assert (store == 5.0).all()


def test_linear_strided_input_and_nan_rows():
    x = torch.randn(64, 200, device="cuda").bfloat16()[:, 5:165]
    w = torch.randn(16, 160, device="cuda")
    a = B.mx4_linear(x, B.mx4_quantize(w), torch.empty(64, 16, dtype=torch.bfloat16, device="cuda"))
    b = B.mx4_linear(x.contiguous(), B.mx4_quantize(w), torch.empty(64, 16, dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(a, b)
    x = x.contiguous()
    x[9, 100] = float("inf")
    c = B.mx4_linear(x, B.mx4_quantize(w), torch.empty(64, 16, dtype=torch.bfloat16, device="cuda"), relu=True)
    assert torch.isnan(c[9]).all()   # the rectifier keeps NaN
    keep = torch.arange(64, device="cuda") != 9
    assert torch.equal(c[keep], b.clamp(min=0)[keep])


def test_linear_captured_and_on_two_streams():
    m, k, n = 700, 256, 192
    w4 = B.mx4_quantize(torch.randn(n, k, device="cuda"))
    x = torch.zeros(m, k, device="cuda", dtype=torch.bfloat16)
    out = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.mx4_linear(x, w4, out)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            B.mx4_linear(x, w4, out)
    for seed in (1, 2):
        x.copy_(torch.randn(m, k, generator=torch.Generator().manual_seed(seed)))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, B.mx4_linear(x, w4, torch.empty_like(out)))
    xs = [torch.randn(3000, k, device="cuda").bfloat16() for _ in range(2)]
    want = [B.mx4_linear(y, w4, torch.empty(3000, n, dtype=torch.bfloat16, device="cuda")) for y in xs]
    outs = [torch.empty_like(y) for y in want]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(10):
        for y, o, st in zip(xs, outs, streams):
            B.mx4_linear(y, w4, o, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    g.reset()


def test_binding_refusals():
    x = torch.randn(4, 64, device="cuda")
    w4, out = B.mx4_quantize(torch.randn(8, 64, device="cuda")), torch.empty(4, 8, device="cuda")
    for bad in (dict(x=x.cpu()), dict(x=x.half()), dict(x=x[:3]), dict(x=x[:, :32]), dict(x=x.t().contiguous().t()), dict(out=out.half()), dict(out=out.cpu()),
                dict(bias=torch.zeros(7, device="cuda")), dict(bias=torch.zeros(8)), dict(x=x.bfloat16()), dict(x=B.mx4_quantize(x[:, :32].contiguous())),
                dict(w=B.Mx4(w4.codes, w4.scales[:-1]))):
        kw = {**dict(x=x, w=w4, out=out), **bad}
        with pytest.raises((ValueError, B.AifError)):
            B.mx4_linear(**kw)
    with pytest.raises((ValueError, B.AifError)):
        B.mx4_quantize(torch.randn(4, 40, device="cuda"))
    with pytest.raises(ValueError):
        B.mx4_quantize(x, B.mx4_empty(5, 64))
    assert B.mx4_linear(x[:0], w4, out[:0]).shape == (0, 8)


def test_item_tower_in_four_bits_fills_the_item_table():
    """Eq. 4's two layers by aif_mx4_linear, its rows into the item table, and the same rows back through the gather."""
    d, M = 64, 300
    ctx = B.Aif(B.make_config(dtype=B.BF16, M=M, d=d, L_max=16, hidden=(64, 32), F=4, B=16, dc=8))
    raw = torch.randn(M, 128, device="cuda").bfloat16() * 0.1
    w0, w1 = torch.randn(96, 128, device="cuda") * 0.1, torch.randn(d, 96, device="cuda") * 0.1
    b0, b1 = torch.randn(96, device="cuda") * 0.01, torch.randn(d, device="cuda") * 0.01
    hidden = B.mx4_linear(raw, B.mx4_quantize(w0), torch.empty(M, 96, dtype=torch.bfloat16, device="cuda"), bias=b0, relu=True)
    rows = B.mx4_linear(hidden, B.mx4_quantize(w1), torch.empty(M, d, dtype=torch.bfloat16, device="cuda"), bias=b1)
    ref = R.quantise(hidden)[0] @ R.quantise(w1)[0].T + b1.double()
    assert ((rows.double() - ref).abs() <= product_bound(R.quantise(hidden)[0], R.quantise(w1)[0], ref, b1.double(), torch.bfloat16)).all()
    ctx.item_nearline_refresh(None, rows)
    out = torch.empty_like(rows)
    ctx.gather_rows(torch.arange(M, dtype=torch.int32, device="cuda"), out)
    torch.cuda.synchronize()
    assert torch.equal(out, rows)
    ctx.close()
