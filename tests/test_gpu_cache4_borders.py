"""The 4-bit sequence cache on the GPU at its borders: lists of offsets that are none, numbers of any size."""
import pytest
import torch

from paper_2511_12934_b200 import binding as B
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
