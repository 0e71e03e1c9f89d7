"""The 4-bit sequence cache on the GPU: its books against a list model, its rows and its attention against 64-bit references."""
import math
import random

import pytest
import torch

from paper_2511_12934_b200 import binding as B
from tests import mx4_reference as R

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16]


def ids(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(counts):
    return torch.tensor([0] + list(counts), dtype=torch.int64).cumsum(0).cuda()


def filled(lengths, d, heads=1, shared=True, page_rows=32, dtype=torch.bfloat16, seed=0, spare=4, scatter=True, sigma=0.1):
    """A cache of sequences of these lengths, and the rows' values [heads, length, d] as float64 (keys, values)."""
    n = len(lengths)
    width = max(1, -(-max(lengths) // page_rows)) + 1
    c = B.Cache4(d=d, n_pages=sum(-(-x // page_rows) for x in lengths) + spare + n, page_rows=page_rows, n_seqs=n, max_pages=width, heads=heads, shared=shared)
    if scatter:   # pages in any order
        c.free_pages.copy_(torch.randperm(c.n_pages, generator=torch.Generator().manual_seed(seed)).int())
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = [(torch.randn(sum(lengths), heads, d, generator=g, device="cuda") * sigma).to(dtype) for _ in range(1 if shared else 2)]
    c.append(ids(*range(n)), offsets(lengths), *rows)
    values = [R.quantise(x)[0] for x in rows]
    at, k, v = 0, [], []
    for x in lengths:
        k.append(values[0][at:at + x].transpose(0, 1))
        v.append(values[-1][at:at + x].transpose(0, 1))
        at += x
    assert c.poll_status() == 0
    return c, k, v


def check_books(c, model):
    table = torch.full((model.n_seqs, model.max_pages), -1, dtype=torch.int32)
    for s, ps in enumerate(model.pages):
        table[s, :len(ps)] = torch.tensor(ps, dtype=torch.int32)
    assert torch.equal(c.table.cpu(), table)
    assert c.lengths.tolist() == model.length and c.refs.tolist() == model.refs
    assert c.n_free.item() == len(model.free) and c.free_pages.tolist()[:len(model.free)] == model.free


def check_rows(c, model, values):
    counts = list(model.length)
    if not sum(counts):
        return
    out = [torch.empty(sum(counts), c.heads, c.d, device="cuda") for _ in values]
    c.read(ids(*range(model.n_seqs)), offsets(counts), *out)
    tags = torch.tensor([t for rows in model.rows for t in rows], device="cuda")
    for o, v in zip(out, values):
        assert torch.equal(o.double(), v[tags])


@pytest.mark.parametrize("seed, n_seqs, heads, shared, page_rows, d", [(0, 5, 1, True, 16, 32), (1, 40, 2, False, 16, 64), (2, 9, 1, True, 32, 128), (3, 70, 1, False, 16, 96), (4, 200, 1, True, 16, 32),
                                                                  (5, 1100, 1, True, 16, 32)])
def test_books_against_the_model(seed, n_seqs, heads, shared, page_rows, d):
    """Random appends, forks, copies, frees and compactions, duplicates, bad ids and full caches among them."""
    rng = random.Random(seed)
    max_pages, n_pages = 5, 3 * n_seqs
    c = B.Cache4(d=d, n_pages=n_pages, page_rows=page_rows, n_seqs=n_seqs, max_pages=max_pages, heads=heads, shared=shared)
    model = R.Books(n_pages, page_rows, n_seqs, max_pages)
    g = torch.Generator(device="cuda").manual_seed(seed)
    n_stock = max(4000, (2 * page_rows + 5) * n_seqs)
    stock = [torch.randn(n_stock, heads, d, generator=g, device="cuda").bfloat16() for _ in range(1 if shared else 2)]
    values = [R.quantise(x)[0] for x in stock]
    used = 0

    def some(n=None):
        got = rng.sample(range(n_seqs), rng.randint(1, n or n_seqs))
        if rng.random() < 0.2:
            got[rng.randrange(len(got))] = rng.choice([-1, n_seqs, got[0], 2 ** 31 - 1])
        return got

    for step in range(40):
        op = rng.choice(["append", "append", "append", "fork", "copy", "free", "compact"])
        model.bad = model.full = False
        if op == "append":
            who = some()
            counts = [rng.choice([0, 1, 3, page_rows - 1, page_rows, page_rows + 5, rng.randint(0, 2 * page_rows)]) for _ in who]
            if used + sum(counts) > n_stock:
                used = 0
            tags = list(range(used, used + sum(counts)))
            c.append(ids(*who), offsets(counts), *[x[used:used + sum(counts)] for x in stock])
            model.append(who, counts, tags)
            used += sum(counts)
        elif op == "compact":
            smaller = rng.choice([n_pages, n_pages + 7, max(1, sum(r > 0 for r in model.refs)), 1])
            into = B.Cache4(d=d, n_pages=smaller, page_rows=page_rows, n_seqs=n_seqs, max_pages=max_pages, heads=heads, shared=shared)
            c.compact(into)
            moved = model.compact(smaller)
            check_books(into, moved)
            check_rows(into, moved, values)
            assert into.poll_status() == (B.STATUS_FULL if moved.full else 0)
            if smaller == n_pages:
                c, model = into, moved
        elif op == "free":
            who = some()
            c.free(ids(*who))
            model.free_seqs(who)
        else:
            dst = some(max(1, n_seqs // 2))
            src = [rng.choice([rng.randrange(n_seqs), rng.randrange(n_seqs), rng.randrange(n_seqs), -3, n_seqs + 1]) for _ in dst]
            (c.fork if op == "fork" else c.copy)(ids(*src), ids(*dst))
            model.share(src, dst, op == "copy")
        check_books(c, model)
        assert c.poll_status() == (B.STATUS_BAD_ID if model.bad else 0) | (B.STATUS_FULL if model.full else 0), (step, op)
    check_rows(c, model, values)


def test_books_of_long_tables():
    """Few sequences whose tables are longer than what one CTA goes through."""
    c = B.Cache4(d=32, n_pages=2100, page_rows=16, n_seqs=4, max_pages=20000)
    model = R.Books(2100, 16, 4, 20000)
    rows = torch.randn(33000, 1, 32, device="cuda").bfloat16()
    values = [R.quantise(rows)[0]]
    c.append(ids(2, 0), offsets([30000, 1500]), rows[:31500])
    model.append([2, 0], [30000, 1500], list(range(31500)))
    check_books(c, model)
    c.fork(ids(2, 0), ids(1, 3))
    model.share([2, 0], [1, 3], False)
    c.append(ids(1, 3, 2), offsets([20, 700, 0]), rows[31500:32220])
    model.append([1, 3, 2], [20, 700, 0], list(range(31500, 32220)))
    check_books(c, model)
    check_rows(c, model, values)
    c.free(ids(2, 3))
    model.free_seqs([2, 3])
    check_books(c, model)
    c.append(ids(2), offsets([33000]), rows)   # 2063 pages: there are not as many left
    model.full = False
    model.append([2], [33000], list(range(33000)))
    assert model.full and c.poll_status() == B.STATUS_FULL
    check_books(c, model)
    check_rows(c, model, values)


def test_snapshot_is_untouched_by_appends():
    c, k, _ = filled([70, 5], 64, page_rows=32, spare=10)
    c2 = B.Cache4(d=64, n_pages=20, page_rows=32, n_seqs=3, max_pages=4)
    rows = torch.randn(40, 64, device="cuda").bfloat16()
    c2.append(ids(0), offsets([40]), rows)
    c2.fork(ids(0), ids(2))
    q = torch.randn(1, 64, device="cuda").bfloat16() * 5
    before = c2.attention(q, torch.empty_like(q), seq_ids=ids(2)).clone()
    c2.append(ids(0), offsets([30]), torch.randn(30, 64, device="cuda").bfloat16())
    assert torch.equal(before, c2.attention(q, torch.empty_like(q), seq_ids=ids(2)))
    assert c2.lengths.tolist() == [70, 0, 40] and c2.table[0, 0] == c2.table[2, 0] and c2.table[0, 1] != c2.table[2, 1]
    out = torch.empty(40, 64, device="cuda")
    c2.read(ids(0), offsets([40]), out)
    assert torch.equal(out.double(), R.quantise(rows)[0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads, d, pad, shift", [(1, 32, 0, 0), (1, 128, 8, 0), (2, 64, 1, 1), (3, 96, 0, 0), (1, 256, 3, 3), (64, 256, 0, 0)])
def test_append_and_read_strides(dtype, heads, d, pad, shift):
    counts = [3, 0, 17, 1]
    total, width = sum(counts), heads * d
    store = torch.randn(total * (width + pad) + shift, device="cuda").to(dtype)
    x = store[shift:].view(total, width + pad)[:, :width].unflatten(1, (heads, d))
    c = B.Cache4(d=d, n_pages=9, page_rows=16, n_seqs=4, max_pages=2, heads=heads)
    c.append(ids(2, 0, 1, 3), offsets(counts), x)
    back = torch.full((total * (width + pad) + shift,), 4.0, dtype=dtype, device="cuda")
    y = back[shift:].view(total, width + pad)[:, :width].unflatten(1, (heads, d))
    c.read(ids(2, 0, 1, 3), offsets(counts), y)
    assert torch.equal(y.double(), R.quantise(x)[0]) and c.poll_status() == 0
    y.fill_(4.0)
    assert (back == 4.0).all()


def test_read_of_rows_that_are_not_there():
    c, k, _ = filled([20, 3], 32, page_rows=16)
    out = torch.full((60, 32), 8.0, device="cuda")
    c.read(ids(0, 7, 1), torch.tensor([2, 27, 30, 50], device="cuda"), out)
    assert c.poll_status() == B.STATUS_BAD_ID
    assert torch.equal(out[2:22].double(), k[0][0]) and torch.equal(out[30:33].double(), k[1][0])
    assert (out[22:30] == 0).all() and (out[33:50] == 0).all() and (out[:2] == 8).all() and (out[50:] == 8).all()
    c.read(ids(0, 1), torch.tensor([0, 5, 3], device="cuda"), out.fill_(8.0))   # offsets descend: nothing happens
    assert (out == 8).all() and c.poll_status() == B.STATUS_BAD_ID
    c.read(ids(0, 1), torch.tensor([0, 5, 61], device="cuda"), out)
    assert (out == 8).all() and c.poll_status() == B.STATUS_BAD_ID
    before = c.lengths.tolist()
    c.append(ids(0, 1), torch.tensor([0, 5, 3], device="cuda"), torch.randn(8, 32, device="cuda"))
    assert c.lengths.tolist() == before and c.poll_status() == B.STATUS_BAD_ID


# ---- attention --------------------------------------------------------------------------------------------------

def reference(q, k, v, i, row, heads, window, sinks, scale):
    """One query row [n_heads, d] against sequence i: out and the parts of its bound."""
    n_heads, d = q.shape[1:]
    length = k[i].shape[1]
    keep = torch.arange(length, device="cuda")
    if window and length > window:
        keep = keep[(keep >= length - window) | (keep < sinks)]
    outs = []
    for h in range(n_heads):
        j = h // (n_heads // heads)
        outs.append(R.attention(q[row:row + 1, h].double(), k[i][j][keep], v[i][j][keep], scale))
    return outs


def check_attention(c, k, v, q, counts, who, out, window=0, sinks=0, scale=0.0, rows=None):
    at, d = 0, c.d
    rng = random.Random(5)
    for i, n in zip(who, counts):
        for row in (range(at, at + n) if rows is None else rng.sample(range(at, at + n), min(n, rows))):
            for h, (ref, spread, mass, reach) in enumerate(reference(q, k, v, i, row, c.heads, window, sinks, scale or 1 / math.sqrt(d))):
                got = out[row, h].double()
                bound = R.attention_bound(q.dtype, ref[0], spread[0], (mass[0][0], mass[1][0]), reach, d)
                assert ((got - ref[0]).abs() <= bound).all(), (i, row, h, ((got - ref[0]).abs() / bound).max().item())
        at += n


LENGTHS = [0, 1, 15, 16, 17, 63, 64, 65, 100, 129, 257, 600]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d, page_rows", [(32, 16), (64, 64), (96, 16), (128, 32), (160, 32), (256, 128)])
@pytest.mark.parametrize("n_heads, heads, shared", [(1, 1, True), (4, 2, False)])
@pytest.mark.parametrize("rows", [1, 3, 40])
def test_attention_over_ragged_sequences(dtype, d, page_rows, n_heads, heads, shared, rows):
    """Every kernel: a row or a few, and tiles of many; lengths about the edges of groups, blocks and pages."""
    c, k, v = filled(LENGTHS, d, heads, shared, page_rows, torch.bfloat16, seed=d + rows)
    counts = [rows] * len(LENGTHS)
    if rows == 40:
        counts[2], counts[5], counts[8] = 0, 200, 300
    g = torch.Generator(device="cuda").manual_seed(rows)
    q = (torch.randn(sum(counts), n_heads, d, generator=g, device="cuda") * 10).to(dtype)
    out = torch.full_like(q, 7.0)
    c.attention(q, out, offsets=offsets(counts))
    assert c.poll_status() == 0
    check_attention(c, k, v, q, counts, range(len(LENGTHS)), out, rows=6)
    assert (out[:counts[0]] == 0).all()   # no keys: zero rows


@pytest.mark.parametrize("dtype, d, rows", [(torch.float32, 64, 2), (torch.float32, 128, 1), (torch.bfloat16, 64, 1), (torch.bfloat16, 128, 2), (torch.bfloat16, 128, 90),
                                            (torch.bfloat16, 64, 300), (torch.bfloat16, 256, 50), (torch.bfloat16, 96, 5)])
@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 1), (16, 0), (17, 4), (60, 33), (100, 64), (500, 200), (1 << 30, 5), (64, 1 << 30)])
def test_window_and_sinks(dtype, d, rows, window, sinks):
    lengths = [0, 1, 16, 40, 61, 165, 700]
    c, k, v = filled(lengths, d, page_rows=16, seed=window + sinks)
    q = (torch.randn(rows * len(lengths), 1, d, device="cuda") * 8).to(dtype)
    out = torch.empty_like(q)
    c.attention(q, out, offsets=offsets([rows] * len(lengths)), window=window, sinks=sinks)
    assert c.poll_status() == 0
    check_attention(c, k, v, q, [rows] * len(lengths), range(len(lengths)), out, window, sinks, rows=3)


@pytest.mark.parametrize("dtype, d, rows, shared", [(torch.float32, 128, 1, True), (torch.bfloat16, 128, 1, True), (torch.bfloat16, 128, 3, False), (torch.bfloat16, 64, 500, True),
                                                    (torch.bfloat16, 128, 260, False), (torch.bfloat16, 256, 130, True), (torch.bfloat16, 256, 1, False)])
def test_long_sequences_are_cut_and_joined(dtype, d, rows, shared):
    c, k, v = filled([9000, 20, 4111], d, shared=shared, page_rows=64, seed=3)
    q = (torch.randn(3 * rows, 1, d, device="cuda") * 12).to(dtype)
    out = torch.empty_like(q)
    c.attention(q, out, offsets=offsets([rows] * 3))
    assert c.poll_status() == 0
    check_attention(c, k, v, q, [rows] * 3, range(3), out, rows=5)
    assert torch.equal(out, c.attention(q, torch.empty_like(q), offsets=offsets([rows] * 3)))   # the same bits every time


@pytest.mark.parametrize("dtype, d, rows", [(torch.float32, 64, 2), (torch.bfloat16, 64, 3), (torch.bfloat16, 128, 100), (torch.bfloat16, 256, 60)])
@pytest.mark.parametrize("sigma", [1e-30, 1e-6, 30.0, 1e6])
def test_magnitudes_far_from_one(dtype, d, rows, sigma):
    """Keys from tiny to huge, peaked and flat weights, scores far beyond where exponentials need no offset."""
    c, k, v = filled([200, 33], d, sigma=sigma, dtype=torch.float32)
    for spread in (1.0, 300.0):
        q = (torch.randn(2 * rows, 1, d, device="cuda") * spread / math.sqrt(d) / sigma).to(dtype)
        out = torch.empty_like(q)
        c.attention(q, out, offsets=offsets([rows] * 2))
        check_attention(c, k, v, q, [rows] * 2, range(2), out, rows=4)


@pytest.mark.parametrize("dtype, d, rows", [(torch.float32, 64, 2), (torch.bfloat16, 32, 3), (torch.bfloat16, 128, 100), (torch.bfloat16, 256, 60)])
def test_rows_of_very_different_magnitudes(dtype, d, rows):
    """One row 2^40 times the others, and elements of a row 2^30 apart: the small ones still count where the large ones have no weight."""
    n = 100
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(n, 1, d, generator=g, device="cuda") * 0.3
    x[7] *= 2.0 ** 40
    x[7, 0] = -x[7, 0].abs()
    x[20, 0, :32] *= 2.0 ** -30
    q = (torch.randn(rows, 1, d, generator=g, device="cuda").abs() * 2).to(dtype)   # row 7 scores far below the others
    c = B.Cache4(d=d, n_pages=8, page_rows=16, n_seqs=1, max_pages=8)
    c.append(ids(0), offsets([n]), x)
    k = [R.quantise(x)[0].transpose(0, 1)]
    out = c.attention(q, torch.empty_like(q), offsets=offsets([rows]))
    keep = torch.arange(n, device="cuda") != 7
    for r in range(0, rows, 9):
        ref, spread, mass, _ = R.attention(q[r].double(), k[0][0][keep], k[0][0][keep], 1 / math.sqrt(d))
        reach = float((q[r].double().abs() @ k[0][0][keep].abs().T).max() / math.sqrt(d))
        assert ((out[r].double() - ref).abs() <= R.attention_bound(dtype, ref, spread, mass, reach, d)).all()


@pytest.mark.parametrize("dtype, d, rows", [(torch.float32, 64, 2), (torch.bfloat16, 64, 3), (torch.bfloat16, 128, 100), (torch.bfloat16, 256, 60), (torch.bfloat16, 96, 2)])
def test_what_is_not_visible_does_not_matter(dtype, d, rows):
    """NaN scales in rows behind the end and outside the window, infinities in the page, change nothing; in a visible row they make NaN."""
    c, k, v = filled([90], d, page_rows=32)
    q = (torch.randn(rows, 1, d, device="cuda") * 8).to(dtype)
    want = c.attention(q, torch.empty_like(q), offsets=offsets([rows]), window=40, sinks=3).clone()
    flat = [c.k_scales[c.table[0, i // 32], :, i % 32] for i in range(96)]
    for i in list(range(3, 50)) + list(range(90, 96)):
        flat[i].fill_(255)
    got = c.attention(q, torch.empty_like(q), offsets=offsets([rows]), window=40, sinks=3)
    assert torch.equal(got, want) and c.poll_status() == 0
    flat[60].fill_(255)
    assert torch.isnan(c.attention(q, torch.empty_like(q), offsets=offsets([rows]), window=40, sinks=3)).all()


@pytest.mark.parametrize("dtype, d, rows", [(torch.float32, 128, 1), (torch.bfloat16, 128, 2), (torch.bfloat16, 64, 70), (torch.bfloat16, 256, 40)])
def test_bad_sequences_and_pages(dtype, d, rows):
    c, k, v = filled([50, 40, 30, 20], d, page_rows=16)
    q = (torch.randn(6 * rows + 4, 1, d, device="cuda") * 8).to(dtype)
    good = c.attention(q[:rows], torch.empty_like(q[:rows]), seq_ids=ids(1), offsets=offsets([rows])).clone()
    out = torch.full_like(q, 7.0)
    c.lengths[3] = -5
    c.table[2, 1] = c.n_pages + 3
    off = offsets([rows] * 6) + 2
    c.attention(q, out, seq_ids=ids(1, -1, 4, 2, 3, 1), offsets=off)
    assert c.poll_status() == B.STATUS_BAD_ID
    part = [out[2 + i * rows:2 + (i + 1) * rows] for i in range(6)]
    assert all(torch.isnan(part[i]).all() for i in (1, 2, 3, 4)) and not torch.isnan(part[0]).any() and not torch.isnan(part[5]).any()
    assert (out[:2] == 7).all() and (out[-2:] == 7).all()   # rows that no sequence names stay as they are
    out.fill_(7.0)
    c.attention(q, out, seq_ids=ids(1, 1), offsets=torch.tensor([0, 9, 5], device="cuda"))
    assert (out == 7).all() and c.poll_status() == B.STATUS_BAD_ID
    c.attention(q[:rows], out[:rows], seq_ids=ids(1), offsets=offsets([rows]))
    assert torch.equal(out[:rows], good) and c.poll_status() == 0


@pytest.mark.parametrize("dtype, heads, d, rows", [(torch.float32, 2, 64, 3), (torch.bfloat16, 1, 128, 5), (torch.bfloat16, 2, 64, 100), (torch.bfloat16, 1, 256, 70)])
def test_strides_repeats_and_scale(dtype, heads, d, rows):
    c, k, v = filled([77, 130], d, heads, shared=False)
    width = 2 * heads * d
    big = (torch.randn(3 * rows, width + 16, device="cuda") * 5).to(dtype)
    q = big[:, 8:8 + width].unflatten(1, (2 * heads, d))
    store = torch.full((3 * rows, width + 24), 3.0, dtype=dtype, device="cuda")
    out = store[:, 16:16 + width].unflatten(1, (2 * heads, d))
    c.attention(q, out, seq_ids=ids(1, 0, 1), offsets=offsets([rows] * 3), scale=0.07)
    check_attention(c, k, v, q, [rows] * 3, [1, 0, 1], out, scale=0.07, rows=4)
    out.fill_(3.0)
    assert (store == 3.0).all()


def test_one_row_per_sequence_without_offsets():
    c, k, v = filled([40, 0, 9], 64)
    q = torch.randn(3, 64, device="cuda").bfloat16() * 9
    out = c.attention(q, torch.empty_like(q))
    check_attention(c, k, v, q.unsqueeze(1), [1] * 3, range(3), out.unsqueeze(1))
    assert c.attention(q[:0], out[:0], seq_ids=ids()).shape == (0, 64)


def test_many_sequences():
    n = 3000
    lengths = [(7 * i) % 50 for i in range(n)]
    c, k, v = filled(lengths, 32, page_rows=16)
    q = torch.randn(n, 1, 32, device="cuda") * 9
    for dtype in DTYPES:
        out = c.attention(q.to(dtype), torch.empty(n, 1, 32, dtype=dtype, device="cuda"))
        for i in range(0, n, 97):
            check_attention(c, [k[i]], [v[i]], q.to(dtype)[i:i + 1], [1], [0], out[i:i + 1])


@pytest.mark.parametrize("n", [128, 129, 700])
@pytest.mark.parametrize("dtype, d", [(torch.float32, 64), (torch.bfloat16, 128)])
def test_bad_offsets_anywhere(n, dtype, d):
    c, k, v = filled([(11 * i) % 60 for i in range(n)], d, page_rows=16)
    q = (torch.randn(2 * n, 1, d, device="cuda") * 8).to(dtype)
    off = offsets([2] * n)
    for at, value in ((0, -1), (n // 2, 0), (n - 1, 2 * n + 1), (n, 2 * n + 1)):
        bad, out = off.clone(), torch.full_like(q, 7.0)
        bad[at] = value
        c.attention(q, out, offsets=bad)
        assert (out == 7).all() and c.poll_status() == B.STATUS_BAD_ID, (at, value)
    out = c.attention(q, torch.empty_like(q), offsets=off)
    assert c.poll_status() == 0
    for i in range(0, n, 61):
        check_attention(c, [k[i]], [v[i]], q[2 * i:2 * i + 2], [2], [0], out[2 * i:2 * i + 2])


def test_pages_behind_four_gigabytes():
    """Codes beyond 2^32 bytes from the beginning of the pool."""
    per_page = 64 * 1024 * 128
    c = B.Cache4(d=256, n_pages=(1 << 32) // per_page + 20, page_rows=1024, n_seqs=2, max_pages=2, heads=64)
    c.free_pages.copy_(c.free_pages.flip(0))   # the last pages first
    x = torch.randn(1100, 64, 256, device="cuda").bfloat16() * 0.1
    c.append(ids(1), offsets([1100]), x)
    assert c.table[1, 0].item() * per_page > 1 << 32
    out = torch.empty_like(x)
    c.read(ids(1), offsets([1100]), out)
    assert torch.equal(out.double(), R.quantise(x)[0])
    k = [None, R.quantise(x)[0].transpose(0, 1)]
    for rows in (1, 40):
        q = torch.randn(rows, 64, 256, device="cuda").bfloat16() * 8
        got = c.attention(q, torch.empty_like(q), seq_ids=ids(1), offsets=offsets([rows]))
        check_attention(c, k, k, q, [rows], [1], got, rows=1)


@pytest.mark.parametrize("dtype, d, rows", [(torch.float32, 64, 1), (torch.bfloat16, 128, 2), (torch.bfloat16, 128, 80), (torch.bfloat16, 256, 40)])
def test_captured_calls_follow_the_cache(dtype, d, rows):
    """Append and attention in one graph: every replay finds the sequence longer than the one before."""
    c = B.Cache4(d=d, n_pages=60, page_rows=16, n_seqs=2, max_pages=30)
    x, q = torch.zeros(7, d, device="cuda").to(dtype), torch.zeros(2 * rows, 1, d, device="cuda").to(dtype)
    out, both, off, cnt = torch.empty_like(q), ids(0, 1), offsets([4, 3]), offsets([rows, rows])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.append(both, off, x)
        c.attention(q, out, seq_ids=both, offsets=cnt)
        s.synchronize()
        c.reset()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.append(both, off, x)
            c.attention(q, out, seq_ids=both, offsets=cnt)
    seen = []
    for step in range(9):
        x.copy_(torch.randn(7, d) * 0.2)
        q.copy_(torch.randn(2 * rows, 1, d) * 6)
        g.replay()
        seen.append(R.quantise(x)[0].unsqueeze(1))
        torch.cuda.synchronize()
    k = [torch.cat([y[:4] for y in seen]).transpose(0, 1), torch.cat([y[4:] for y in seen]).transpose(0, 1)]
    assert c.lengths.tolist() == [36, 27] and c.poll_status() == 0
    check_attention(c, k, k, q, [rows, rows], [0, 1], out, rows=4)
    g.reset()


@pytest.mark.parametrize("n", [40, 150])
def test_captured_books(n):
    """Fork, append, free and read in one graph, replayed, against the same calls one by one."""
    rows = torch.randn(5 * n, 64, device="cuda").bfloat16()
    first, second, off = ids(*range(n)), ids(*range(n, 2 * n)), offsets([5] * n)

    def calls(c, out):
        c.fork(first, second)
        c.append(first, off, rows)
        c.read(second, off, out)
        c.free(second)

    caches = [B.Cache4(d=64, n_pages=4 * n, page_rows=16, n_seqs=2 * n, max_pages=4) for _ in range(2)]
    outs = [torch.zeros(5 * n, 64, dtype=torch.bfloat16, device="cuda") for _ in caches]
    for c in caches:
        c.append(first, off, rows)
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            calls(caches[0], outs[0])
    torch.cuda.synchronize()
    for _ in range(6):
        g.replay()
        torch.cuda.synchronize()
        calls(caches[1], outs[1])
        a, b = caches
        for name in ("table", "lengths", "refs", "n_free"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name
        assert torch.equal(a.free_pages[:a.n_free.item()], b.free_pages[:b.n_free.item()]) and torch.equal(outs[0], outs[1])
    assert a.lengths.tolist() == [35] * n + [0] * n and a.poll_status() == 0 and b.poll_status() == 0
    g.reset()


def test_calls_on_two_streams_side_by_side():
    """Readers of one cache at the same time, each with a workspace of its own."""
    c, k, v = filled([3000, 2500], 128)
    qs = [torch.randn(2 * r, 1, 128, device="cuda").bfloat16() * 8 for r in (1, 300)]
    offs = [offsets([q.shape[0] // 2] * 2) for q in qs]
    want = [c.attention(q, torch.empty_like(q), offsets=o).clone() for q, o in zip(qs, offs)]
    outs, streams = [torch.empty_like(q) for q in qs], [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for q, o, out, s in zip(qs, offs, outs, streams):
            c.attention(q, out, offsets=o, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_binding_refusals():
    c, _, _ = filled([10], 64)
    q = torch.randn(1, 64, device="cuda").bfloat16()
    for bad in (dict(q=q.cpu()), dict(q=q.half()), dict(out=q.float()), dict(q=q[:, :32]), dict(out=q[:0]), dict(seq_ids=ids(0).long()), dict(seq_ids=ids(0).cpu()),
                dict(offsets=torch.tensor([0, 1], dtype=torch.int32, device="cuda")), dict(offsets=torch.tensor([0, 1])), dict(window=-1), dict(scale=-0.5)):
        with pytest.raises((ValueError, B.AifError)):
            c.attention(**{**dict(q=q, out=torch.empty_like(q), seq_ids=ids(0)), **bad})
    for bad in (dict(k=q.half()), dict(k=q[:, :32]), dict(v=q), dict(offsets=offsets([1, 0])), dict(seq_ids=torch.zeros(1, device="cuda"))):
        with pytest.raises((ValueError, B.AifError)):
            c.append(**{**dict(seq_ids=ids(0), offsets=offsets([1]), k=q), **bad})
    with pytest.raises(B.AifError):
        c.append(ids(0, 0), offsets([0, 1]), q)    # more entries than sequences
    for bad in (dict(d=48), dict(page_rows=20), dict(heads=0), dict(n_pages=0), dict(max_pages=0)):
        with pytest.raises(B.AifError):
            B.Cache4(**{**dict(d=64, n_pages=4, page_rows=16, n_seqs=1, max_pages=4), **bad})
    with pytest.raises(B.AifError):
        c.compact(B.Cache4(d=32, n_pages=4, page_rows=32, n_seqs=1, max_pages=4))


def test_a_request_from_the_cache():
    """Behaviours kept in the cache, a snapshot for a request, its sequence into the user-side call, the candidates scored, and their target attention
    straight from the cache next to the one inside the scoring model's inputs."""
    d, L, M = 128, 150, 400
    ctx = B.Aif(B.make_config(dtype=B.BF16, M=M, d=d, L_max=L, hidden=(128, 64), F=4, B=16, dc=8))
    g = torch.Generator(device="cuda").manual_seed(2)

    def randn(*shape, scale=0.1):
        return torch.randn(*shape, generator=g, device="cuda").mul(scale)

    width = ctx.input_width
    mlp = {"W": [randn(128, width).bfloat16(), randn(64, 128).bfloat16()], "b": [randn(128), randn(64)], "w_out": randn(64).bfloat16(), "b_out": randn(1)}
    ctx.load_weights(mlp)
    items = randn(M, d).bfloat16()
    ctx.item_nearline_refresh(None, items)
    cache = B.Cache4(d=d, n_pages=40, page_rows=16, n_seqs=2, max_pages=20)
    behaviours = randn(L, d).bfloat16()
    cache.append(ids(0), offsets([L - 10]), behaviours[:L - 10])
    cache.append(ids(0), offsets([10]), behaviours[L - 10:])
    cache.fork(ids(0), ids(1))
    cache.append(ids(0), offsets([5]), randn(5, d).bfloat16())   # what comes in meanwhile is not the request's
    seq = torch.empty(L, d, dtype=torch.bfloat16, device="cuda")
    cache.read(ids(1), offsets([L]), seq)
    assert torch.equal(seq.double(), R.quantise(behaviours)[0])
    cross = randn(4, 16, 8).bfloat16()
    state = ctx.user_precompute(1, mode=B.USER_PROJECTED, profile=randn(d).bfloat16(), seq=seq, cross_raw=cross)
    cand = torch.randperm(M, generator=g, device="cuda")[:300].int()
    logits = torch.empty(300, device="cuda")
    ctx.score(state, cand, logits)
    rows = torch.empty(300, d, dtype=torch.bfloat16, device="cuda")
    ctx.gather_rows(cand, rows)
    att = cache.attention(rows, torch.empty_like(rows), seq_ids=ids(1), offsets=offsets([300]))
    torch.cuda.synchronize()
    assert torch.isfinite(logits).all() and ctx.poll_status() == 0 and cache.poll_status() == 0
    ref, spread, mass, reach = R.attention(rows.double(), seq.double(), seq.double(), 1 / math.sqrt(d))
    assert ((att.double() - ref).abs() <= R.attention_bound(torch.bfloat16, ref, spread, mass, reach, d)).all()
    cache.free(ids(1))
    assert cache.lengths.tolist() == [L + 5, 0]
    state.release()
    ctx.close()
