"""Sizes near 2^31 of the paged entry points."""
import numpy as np
import pytest

from gpu_util import dev, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    seer.load_library()
    return seer


@pytest.mark.parametrize("rows", [2 ** 31 - 1, 2 ** 31 - 30000])
@pytest.mark.parametrize("refused", [False, True])
def test_plan_of_two_to_the_31_rows(S, rows, refused):
    """A bound of nearly 2^31 rows (8.6 GB of slots), few of them in use: every slot is written, none beside them."""
    import torch
    pages = S.seer_page_desc(16, 8, 4)
    held, keep = dev(np.array([0, 0, 0])), dev(np.array([1 if refused else 0, 0, 0]))
    cu, kv, status = dev(np.array([0, 20, 20, 23])), dev(np.zeros(3, int)), dev(np.array([5]))
    free, n_in, n_out = dev(np.arange(8)), dev(np.array([8])), dev(np.array([0]))
    table = dev(np.full((3, 4), -1))
    buf = torch.full((rows + 2048,), 7, dtype=torch.int32, device="cuda")
    slots = buf[1024:1024 + rows]
    S.seer_page_plan(pages, held, keep, cu, None, 3, rows, free, n_in, n_out, table, kv, slots, status)
    want = np.full(64, -1)
    if not refused:
        want[:23] = [7 * 16 + i for i in range(16)] + [6 * 16 + i for i in range(4)] + [5 * 16 + i for i in range(3)]
    assert host(status).item() == (S.SEER_PAGES_INVALID if refused else 0)
    assert host(slots[:64]).tolist() == want.tolist()
    for at in range(64, rows, 1 << 28):
        assert bool((slots[at:at + (1 << 28)] == -1).all()), at
    assert bool((buf[:1024] == 7).all()) and bool((buf[1024 + rows:] == 7).all())
    del buf, slots
    torch.cuda.empty_cache()
