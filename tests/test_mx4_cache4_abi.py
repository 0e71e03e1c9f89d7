"""4-bit matrices and the 4-bit cache: refusals of arguments, which need no GPU, and the plain references' own pins."""
import ctypes as C

import pytest
import torch

from paper_2511_12934_b200 import binding as B
from paper_2511_12934_b200 import build as libbuild
from tests import mx4_reference as R


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return B.load_library()


def test_struct_layouts_match_the_header(lib):
    assert C.sizeof(B.aif_mx4_product) == 8 + 8 + 8 + 7 * 8 + 8 + 8 + 8 + 8 + 8 + 8
    assert C.sizeof(B.aif_cache4) == 8 * 4 + 11 * 8
    assert C.sizeof(B.aif_cache4_query) == 4 * 4 + 2 * 8 + 8 + 2 * 8 + 2 * 8 + 16 + 2 * 8


def test_scale_bytes(lib):
    assert lib.aif_mx4_scale_bytes(1, 32) == 512 and lib.aif_mx4_scale_bytes(128, 128) == 512
    assert lib.aif_mx4_scale_bytes(129, 160) == 2 * 2 * 512 and lib.aif_mx4_scale_bytes(0, 64) == 0
    for rows, cols in ((-1, 32), (1, 0), (1, 31), (1, 48)):
        assert lib.aif_mx4_scale_bytes(rows, cols) == B.ERR_SHAPE
    assert lib.aif_mx4_workspace_bytes(3, 64) == 256 + 512


P = 1 << 20   # an aligned address that no call gets as far as using


def test_matrix_refusals(lib):
    q = lib.aif_mx4_quantize
    assert q(P, 7, 1, 32, 32, P, P, None) == B.ERR_ARG
    assert q(P, B.F32, -1, 32, 32, P, P, None) == B.ERR_SHAPE
    assert q(P, B.F32, 1, 33, 33, P, P, None) == B.ERR_SHAPE
    assert q(P, B.F32, 1, 64, 32, P, P, None) == B.ERR_SHAPE
    assert q(None, B.F32, 1, 32, 32, P, P, None) == B.ERR_ARG
    assert q(P, B.F32, 1, 32, 32, P + 8, P, None) == B.ERR_ARG
    assert q(P + 2, B.F32, 1, 32, 32, P, P, None) == B.ERR_ARG
    assert q(None, B.F32, 0, 32, 32, None, None, None) == B.OK
    d = lib.aif_mx4_dequantize
    assert d(None, P, 1, 32, P, B.BF16, 32, None) == B.ERR_ARG
    assert d(P, P, 1, 32, P + 1, B.BF16, 32, None) == B.ERR_ARG
    assert d(P, P, 1 << 40, 32, P, B.BF16, 32, None) == B.ERR_SHAPE


def product(**kw):
    p = B.aif_mx4_product()
    p.struct_size = C.sizeof(p)
    base = dict(dtype=B.BF16, m=4, n=8, k=64, x=P, x_stride=64, w_codes=P, w_scales=P, out=P, out_stride=8, workspace=P, workspace_bytes=1 << 20)
    for name, value in {**base, **kw}.items():
        setattr(p, name, value)
    return p


@pytest.mark.parametrize("change, code", [
    (dict(struct_size=4), B.ERR_ARG), (dict(dtype=3), B.ERR_ARG), (dict(m=-1), B.ERR_SHAPE), (dict(n=0), B.ERR_SHAPE), (dict(k=48), B.ERR_SHAPE),
    (dict(k=0), B.ERR_SHAPE), (dict(out_stride=7), B.ERR_SHAPE), (dict(w_codes=None), B.ERR_ARG), (dict(w_scales=P + 4), B.ERR_ARG),
    (dict(out=None), B.ERR_ARG), (dict(out=P + 1), B.ERR_ARG), (dict(x_stride=32), B.ERR_SHAPE), (dict(workspace=None), B.ERR_ARG),
    (dict(workspace_bytes=100), B.ERR_ARG), (dict(x=None), B.ERR_ARG), (dict(x=P + 1), B.ERR_ARG), (dict(bias=P + 2), B.ERR_ARG),
])
def test_product_refusals(lib, change, code):
    assert lib.aif_mx4_linear(C.byref(product(**change)), None) == code
    assert lib.aif_mx4_linear(None, None) == B.ERR_ARG
    assert lib.aif_mx4_linear(C.byref(product(m=0)), None) == B.OK


def cache(**kw):
    c = B.aif_cache4()
    c.struct_size = C.sizeof(c)
    base = dict(d=64, heads=2, shared=1, page_rows=32, n_pages=100, n_seqs=4, max_pages=50, k_codes=P, k_scales=P, table=P, lengths=P, refs=P, free_pages=P,
                n_free=P, scratch=P, status=P)
    for name, value in {**base, **kw}.items():
        setattr(c, name, value)
    return c


BAD_CACHES = [
    (dict(struct_size=1), B.ERR_ARG), (dict(d=48), B.ERR_SHAPE), (dict(d=288), B.ERR_SHAPE), (dict(d=0), B.ERR_SHAPE), (dict(heads=0), B.ERR_SHAPE),
    (dict(heads=65), B.ERR_SHAPE), (dict(shared=2), B.ERR_ARG), (dict(page_rows=24), B.ERR_SHAPE), (dict(page_rows=8), B.ERR_SHAPE),
    (dict(page_rows=2048), B.ERR_SHAPE), (dict(n_pages=0), B.ERR_SHAPE), (dict(n_seqs=0), B.ERR_SHAPE), (dict(max_pages=0), B.ERR_SHAPE),
    (dict(n_seqs=1 << 20, max_pages=1 << 12), B.ERR_SHAPE), (dict(max_pages=1 << 27), B.ERR_SHAPE), (dict(table=None), B.ERR_ARG), (dict(k_codes=P + 8), B.ERR_ARG),
    (dict(v_codes=P), B.ERR_ARG), (dict(shared=0), B.ERR_ARG), (dict(status=None), B.ERR_ARG), (dict(scratch=None), B.ERR_ARG),
]


@pytest.mark.parametrize("change, code", BAD_CACHES)
def test_cache_refusals(lib, change, code):
    c = C.byref(cache(**change))
    assert lib.aif_cache4_reset(c, None) == code
    assert lib.aif_cache4_append(c, 1, P, P, P, None, B.BF16, 1, 128, None) == code
    assert lib.aif_cache4_fork(c, 1, P, P, None) == code and lib.aif_cache4_copy(c, 1, P, P, None) == code
    assert lib.aif_cache4_free(c, 1, P, None) == code
    assert lib.aif_cache4_compact(c, C.byref(cache()), None) == code and lib.aif_cache4_compact(C.byref(cache()), c, None) == code
    assert lib.aif_cache4_read(c, 1, P, P, P, None, B.BF16, 1, 128, None) == code
    assert lib.aif_cache4_poll(c, C.byref(C.c_uint32()), None) == code
    assert lib.aif_cache4_attention(c, C.byref(query()), None) == code
    assert lib.aif_cache4_attention_workspace(c, C.byref(query())) == code


def query(**kw):
    q = B.aif_cache4_query()
    q.struct_size = C.sizeof(q)
    base = dict(dtype=B.BF16, n_heads=4, n=2, rows=2, q=P, out=2 * P, q_stride=256, out_stride=256, workspace=P, workspace_bytes=1 << 30)
    for name, value in {**base, **kw}.items():
        setattr(q, name, value)
    return q


@pytest.mark.parametrize("change, code", [
    (dict(struct_size=0), B.ERR_ARG), (dict(dtype=2), B.ERR_ARG), (dict(n_heads=3), B.ERR_SHAPE), (dict(n_heads=0), B.ERR_SHAPE), (dict(n_heads=2 * 65), B.ERR_SHAPE),
    (dict(n=-1), B.ERR_SHAPE), (dict(rows=3), B.ERR_SHAPE), (dict(n=5, rows=5), B.ERR_SHAPE), (dict(q_stride=255), B.ERR_SHAPE), (dict(out_stride=260), B.ERR_SHAPE),
    (dict(window=-1), B.ERR_SHAPE), (dict(sinks=-1), B.ERR_SHAPE), (dict(scale=-1.0), B.ERR_ARG), (dict(scale=float("nan")), B.ERR_ARG),
    (dict(scale=float("inf")), B.ERR_ARG), (dict(rows=1 << 40, offsets=P), B.ERR_SHAPE),
])
def test_query_refusals(lib, change, code):
    assert lib.aif_cache4_attention(C.byref(cache()), C.byref(query(**change)), None) == code
    assert lib.aif_cache4_attention_workspace(C.byref(cache()), C.byref(query(**change))) == code


@pytest.mark.parametrize("change, code", [(dict(q=None), B.ERR_ARG), (dict(out=P + 8), B.ERR_ARG), (dict(workspace=None), B.ERR_ARG), (dict(workspace_bytes=16), B.ERR_ARG),
                                          (dict(n=0, rows=0), B.OK), (dict(n=2, rows=0, offsets=P), B.OK)])
def test_query_buffers(lib, change, code):
    assert lib.aif_cache4_attention(C.byref(cache()), C.byref(query(**change)), None) == code


def test_row_and_list_refusals(lib):
    c = C.byref(cache())
    assert lib.aif_cache4_append(c, 5, P, P, P, None, B.BF16, 1, 128, None) == B.ERR_SHAPE      # more entries than sequences
    assert lib.aif_cache4_append(c, 1, P, P, P, P, B.BF16, 1, 128, None) == B.ERR_ARG           # values for a shared cache
    assert lib.aif_cache4_append(c, 1, P, P, P, None, B.BF16, 1, 127, None) == B.ERR_SHAPE
    assert lib.aif_cache4_append(c, 1, P, P, P, None, 9, 1, 128, None) == B.ERR_ARG
    assert lib.aif_cache4_append(c, 1, P, P, None, None, B.F32, 1, 128, None) == B.ERR_ARG
    assert lib.aif_cache4_append(c, 1, None, P, P, None, B.F32, 1, 128, None) == B.ERR_ARG
    assert lib.aif_cache4_append(c, 0, None, None, None, None, B.F32, 0, 128, None) == B.OK
    assert lib.aif_cache4_read(c, 1, P, P, P + 1, None, B.BF16, 1, 128, None) == B.ERR_ARG
    assert lib.aif_cache4_fork(c, 1, None, P, None) == B.ERR_ARG and lib.aif_cache4_free(c, -1, P, None) == B.ERR_SHAPE
    other = cache(k_codes=2 * P, k_scales=2 * P, table=2 * P, lengths=2 * P, refs=2 * P, free_pages=2 * P, n_free=2 * P, scratch=2 * P)
    other.d = 32
    assert lib.aif_cache4_compact(c, C.byref(other), None) == B.ERR_SHAPE
    assert lib.aif_cache4_compact(c, c, None) == B.ERR_ARG
    assert lib.aif_cache4_scratch_ints(c) > 2 * 100 + 6 * 4 and lib.aif_cache4_scratch_ints(None) == B.ERR_ARG


def test_reference_rounds_ties_to_even_codes():
    x = torch.tensor([6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -5.0, -0.25, 7.99] + [0.0] * 21)
    v, code, byte = R.quantise(x)
    assert v[:11].tolist() == [6.0, 4.0, 4.0, 2.0, 2.0, 1.0, 1.0, 0.0, -4.0, 0.0, 6.0] and byte.tolist() == [127]
    assert code[:11].tolist() == [7, 6, 6, 4, 4, 2, 2, 0, 14, 8, 7]
    v, _, byte = R.quantise(torch.full((32,), 2.0 ** -149))
    assert byte.tolist() == [0] and not v.any()
    v, _, byte = R.quantise(torch.tensor([1.0] * 31 + [float("inf")]))
    assert byte.tolist() == [255] and torch.isnan(v).all()


def test_books_model_gives_pages_back_in_order():
    b = R.Books(8, 16, 4, 4)
    b.append([0, 1], [20, 5], list(range(25)))
    assert b.pages[:2] == [[0, 1], [2]] and b.free == [7, 6, 5, 4, 3]
    b.share([0], [2], copy=False)
    b.append([2, 0], [1, 1], ["a", "b"])   # both copy the page they share; nobody has it then
    assert b.pages[2] == [0, 3] and b.pages[0] == [0, 4] and b.refs[1] == 0 and b.free == [7, 6, 5, 1]
    b.free_seqs([0, 2])
    assert b.free == [7, 6, 5, 1, 3, 4, 0] and b.refs[0] == 0
