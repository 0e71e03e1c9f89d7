"""The 4-bit sequence cache on the GPU at its borders: lists of offsets that are none, numbers of any size."""
import math

import pytest
import torch

from paper_2511_12934_b200 import binding as B
from tests import mx4_reference as R
from tests.test_gpu_cache4 import filled, ids, offsets

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [2, 40, 200])
@pytest.mark.parametrize("dtype, shared", [(torch.bfloat16, True), (torch.float32, False)])
def test_append_with_bad_offsets_leaves_everything(n, dtype, shared):
    """Offsets that descend or leave the rows, by little and by more than 32 bits: the whole call is undone."""
    c, k, v = filled([(11 * i) % 60 for i in range(n)], 32, shared=shared, page_rows=16, spare=2 * n)
    rows = [torch.randn(5 * n, 32, device="cuda").to(dtype) for _ in range(1 if shared else 2)]
    off = offsets([5] * n)
    names = ("k_codes", "k_scales", "table", "lengths", "refs", "free_pages", "n_free") + (() if shared else ("v_codes", "v_scales"))
    before = {name: getattr(c, name).clone() for name in names}
    for at in (0, n // 2, n):
        for value in (-1, -2 ** 31, -2 ** 32 + 5, -2 ** 32 + 10 ** 5, -2 ** 63, 5 * n + 1, 2 ** 32 + 5, 2 ** 63 - 1):
            bad = off.clone()
            bad[at] = value
            c.append(ids(*range(n)), bad, *rows)
            assert c.poll_status() == B.STATUS_BAD_ID, (at, value)
    bad = off.clone()
    bad[n] = 5 * n - 6   # descends at the end
    c.append(ids(*range(n)), bad, *rows)
    assert c.poll_status() == B.STATUS_BAD_ID
    for name in names:
        assert torch.equal(getattr(c, name), before[name]), name
    c.append(ids(*range(n)), off, *rows)
    assert c.poll_status() == 0 and c.lengths.tolist() == [(11 * i) % 60 + 5 for i in range(n)]


# every kernel: fp32 by one and by four rows, bf16 of few rows, of many by d
KERNELS = [(torch.float32, 128, 1), (torch.float32, 64, 5), (torch.bfloat16, 32, 2), (torch.bfloat16, 64, 3), (torch.bfloat16, 128, 9), (torch.bfloat16, 256, 2), (torch.bfloat16, 96, 2),
           (torch.bfloat16, 160, 7), (torch.bfloat16, 64, 100), (torch.bfloat16, 128, 300), (torch.bfloat16, 256, 60)]


def hold(q, k, v, out, columns=slice(None), scale=None):
    """out [rows, 1, d] of a call over all of k, v [keys, d] (float64) against the reference, in these columns: scores are sums of d fp32 products, whatever the elements' magnitudes."""
    d = k.shape[1]
    scale = scale or 1 / math.sqrt(d)
    for r in range(0, q.shape[0], max(1, q.shape[0] // 5)):
        ref, spread, mass, _ = R.attention(q[r].double(), k, v, scale)
        reach = float((q[r].double().abs() @ k.abs().T).max() * scale)
        bound = R.attention_bound(q.dtype, ref, spread, mass, reach, d)
        err = (out[r].double() - ref).abs()
        assert (err <= bound)[:, columns].all(), (r, (err / bound)[:, columns].max().item())


@pytest.mark.parametrize("dtype, d, rows", KERNELS)
def test_a_block_of_values_that_is_no_number_spoils_its_columns_alone(dtype, d, rows):
    """Values of their own: an infinity in row 40 makes one block of 32 values NaN, which reaches those 32 columns of every output and no other."""
    n, block = 90, d // 32 - 1
    g = torch.Generator(device="cuda").manual_seed(d)
    k, v = [torch.randn(n, 1, d, generator=g, device="cuda") * 0.3 for _ in range(2)]
    v[40, 0, 32 * block + 5] = math.inf
    c = B.Cache4(d=d, n_pages=8, page_rows=16, n_seqs=1, max_pages=8, shared=False)
    c.append(ids(0), offsets([n]), k, v)
    q = (torch.randn(rows, 1, d, generator=g, device="cuda") * 4).to(dtype)
    out = c.attention(q, torch.empty_like(q), offsets=offsets([rows]))
    spoilt = torch.zeros(d, dtype=torch.bool, device="cuda")
    spoilt[32 * block:] = True
    assert torch.equal(torch.isnan(out), spoilt.expand_as(out)) and c.poll_status() == 0
    kq, vq = R.quantise(k)[0][:, 0], torch.nan_to_num(R.quantise(v)[0][:, 0])
    hold(q, kq, vq, out, ~spoilt)


@pytest.mark.parametrize("dtype, d, rows", [x for x in KERNELS if x[1] > 32])
@pytest.mark.parametrize("shared", [True, False])
@pytest.mark.parametrize("power", [-24, -30, -60])
def test_columns_far_smaller_than_the_others(dtype, d, rows, shared, power):
    """A block of 32 columns of every row 2^power of the rest: those columns of the output are as exact as the others."""
    n = 150
    g = torch.Generator(device="cuda").manual_seed(d)
    x = [torch.randn(n, 1, d, generator=g, device="cuda") * 0.3 for _ in range(1 if shared else 2)]
    x[-1][:, :, d - 32:] *= 2.0 ** power
    c = B.Cache4(d=d, n_pages=12, page_rows=16, n_seqs=1, max_pages=12, shared=shared)
    c.append(ids(0), offsets([n]), *x)
    q = (torch.randn(rows, 1, d, generator=g, device="cuda") * 4).to(dtype)
    out = c.attention(q, torch.empty_like(q), offsets=offsets([rows]))
    k, v = [R.quantise(y)[0][:, 0] for y in (x[0], x[-1])]
    hold(q, k, v, out)


@pytest.mark.parametrize("dtype, d, rows", [x for x in KERNELS if x[1] > 32])
@pytest.mark.parametrize("power", [20, 26, 34, 60])
def test_one_row_with_a_block_far_larger_than_the_rest(dtype, d, rows, power):
    """Values of their own: a row of ordinary weight has one block 2^power times everything else.  The other columns do not feel it."""
    n = 150
    g = torch.Generator(device="cuda").manual_seed(d + power)
    k, v = [torch.randn(n, 1, d, generator=g, device="cuda") * 0.3 for _ in range(2)]
    v[77, :, :32] *= 2.0 ** power
    c = B.Cache4(d=d, n_pages=12, page_rows=16, n_seqs=1, max_pages=12, shared=False)
    c.append(ids(0), offsets([n]), k, v)
    q = (torch.randn(rows, 1, d, generator=g, device="cuda") * 4).to(dtype)
    out = c.attention(q, torch.empty_like(q), offsets=offsets([rows]))
    hold(q, R.quantise(k)[0][:, 0], R.quantise(v)[0][:, 0], out)


@pytest.mark.parametrize("dtype, d, rows", [x for x in KERNELS if x[1] > 32])
def test_queries_far_smaller_where_keys_are_larger(dtype, d, rows):
    """Elements of a query 2^20 apart against keys 2^20 apart the other way round: both halves of a score count alike."""
    n = 150
    g = torch.Generator(device="cuda").manual_seed(d)
    k, v = [torch.randn(n, 1, d, generator=g, device="cuda") * 0.3 for _ in range(2)]
    q = torch.randn(rows, 1, d, generator=g, device="cuda") * 4
    k[:, :, :32] *= 2.0 ** 20
    q[:, :, :32] *= 2.0 ** -20
    q = q.to(dtype)
    c = B.Cache4(d=d, n_pages=12, page_rows=16, n_seqs=1, max_pages=12, shared=False)
    c.append(ids(0), offsets([n]), k, v)
    out = c.attention(q, torch.empty_like(q), offsets=offsets([rows]))
    hold(q, R.quantise(k)[0][:, 0], R.quantise(v)[0][:, 0], out)


def test_sums_of_millions_of_keys_stay_finite():
    """2^23 keys of 1536, all with the same large score: the sums of weights without an offset may not leave fp32."""
    n, d, rows = 1 << 23, 64, 40
    c = B.Cache4(d=d, n_pages=8200, page_rows=1024, n_seqs=1, max_pages=8200)
    x = torch.full((n, d), 1536.0, dtype=torch.bfloat16, device="cuda")
    c.append(ids(0), offsets([n]), x)
    for score in (95.0, 80.0, -95.0, 200.0):   # in powers of two
        q = torch.full((rows, d), score / (1.4426950408889634 * 1536 * d) * math.sqrt(d), device="cuda").bfloat16()
        out = c.attention(q, torch.empty_like(q), offsets=offsets([rows]))
        assert (out == 1536).all(), score


@pytest.mark.parametrize("dtype, d, rows", [x for x in KERNELS if x[1] > 32])
@pytest.mark.parametrize("score, power", [(-90, -60), (-75, -45), (-60, -100), (40, 30), (75, 60)])
def test_small_columns_where_all_scores_are_far_from_zero(dtype, d, rows, score, power):
    """All scores near 2^score, a block of values 2^power of the rest: no product of weight and value may leave fp32."""
    n = 100
    g = torch.Generator(device="cuda").manual_seed(d)
    k = torch.full((n, 1, d), 1.0, device="cuda")
    v = torch.randn(n, 1, d, generator=g, device="cuda")
    v[:, :, d - 32:] *= 2.0 ** power
    c = B.Cache4(d=d, n_pages=12, page_rows=16, n_seqs=1, max_pages=12, shared=False)
    c.append(ids(0), offsets([n]), k, v)
    q = torch.full((rows, 1, d), score / 1.4426950408889634 / math.sqrt(d), device="cuda").to(dtype)
    out = c.attention(q, torch.empty_like(q), offsets=offsets([rows]))
    hold(q, R.quantise(k)[0][:, 0], R.quantise(v)[0][:, 0], out)


@pytest.mark.parametrize("max_pages", [4, 20000])   # one CTA, one cluster
def test_a_copy_without_room_leaves_its_destination_empty(max_pages):
    """Two copies of three pages each where five are to be had: the first is served, the destination of the second has lost its page and has no row; a copy of nothing is served all the same."""
    c = B.Cache4(d=32, n_pages=8, page_rows=16, n_seqs=6, max_pages=max_pages)
    c.append(ids(0, 3), offsets([40, 16]), torch.randn(56, 32, device="cuda"))   # pages 0 .. 2 and 3; 4 .. 7 are free
    c.copy(ids(0, 0, 5), ids(2, 3, 4))
    assert c.poll_status() == B.STATUS_FULL
    assert c.lengths.tolist() == [40, 0, 40, 0, 0, 0] and c.table[3].tolist() == [-1] * c.max_pages
    assert c.n_free.item() == 2 and c.refs.sum().item() == 6
    c.append(ids(3), offsets([32]), torch.randn(32, 32, device="cuda"))   # it can be used again
    assert c.poll_status() == 0 and c.lengths[3].item() == 32 and c.n_free.item() == 0
