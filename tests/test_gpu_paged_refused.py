"""A refused plan is not lost behind the plans that follow it."""
import numpy as np
import pytest

from gpu_util import dev, host
from oracle.paged import EXHAUSTED, INVALID, WIDTH

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    seer.load_library()
    return seer


def test_bits_add_up(S):
    pages = S.seer_page_desc(16, 4, 3)
    held, kv, table = dev(np.array([0, 0])), dev(np.array([9, 9])), dev(np.full((2, 3), -1))
    free, n_in, n_out = dev(np.arange(4)), dev(np.array([4])), dev(np.array([0]))
    slots, status, refused = dev(np.zeros(64, int)), dev(np.array([77])), dev(np.array([0]))

    def plan(keep, cu):
        S.seer_page_plan_latched(pages, held, dev(np.array(keep)), dev(np.array(cu)), None, 2, 64, free, n_in, n_out, table,
                                 kv, slots, status, refused)
        return host(status).item(), host(refused).item()

    assert plan([0, 0], [0, 1, 2]) == (0, 0)
    assert plan([0, 0], [0, 49, 49]) == (WIDTH, WIDTH)
    assert plan([0, 0], [0, 1, 2]) == (0, WIDTH)
    assert plan([0, 0], [0, 20, 60]) == (EXHAUSTED, WIDTH | EXHAUSTED)
    assert plan([1, 0], [0, 1, 2]) == (INVALID, WIDTH | EXHAUSTED | INVALID)
    assert plan([0, 0], [0, 1, 2]) == (0, WIDTH | EXHAUSTED | INVALID)


def test_the_first_of_two_recorded_plans(S):
    """Its status is overwritten by the second one's in every replay."""
    import torch
    from paper_2607_14557_amd.runner import PagedCache, record
    c = PagedCache(2, 1, 64, 1, 8, 16, 2, 64, 100)
    big, small = dev(np.array([0, 65, 65])), dev(np.array([0, 1, 2]))      # 5 pages to a row of 4
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = record(lambda: (c.plan(big, 100, stream=st), c.plan(small, 2, stream=st)), st)
    for i in range(3):
        g.replay(st)
        with pytest.raises(S.SeerError, match="max_len"):
            c.check(st)
        assert host(c.status).item() == 0
        c.check(st.cuda_stream)                                            # said once
        assert host(c.lens).tolist() == [i + 1, i + 1]
    g.replay(st)
    g.replay(st)
    c.plan(small, 2, stream=st)
    with pytest.raises(S.SeerError):
        c.check(st)
    g.close()


def test_arrays_on_another_device_than_the_cache(S):
    """Host tensors given to a cache on the GPU."""
    import torch
    from paper_2607_14557_amd.runner import PagedCache
    c = PagedCache(2, 1, 64, 1, 8, 16, 2, 64, 4)
    cu, q = dev(np.array([0, 1, 2])), torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")
    k = q[:, :64]
    c.plan(cu, 4)
    for call in (lambda: c.plan(cu.cpu(), 4), lambda: c.store(0, k.cpu(), k, 4), lambda: c.store(0, k, k.cpu(), 4),
                 lambda: c.store(0, k, k, 4, c.slots.cpu()), lambda: c.attend(0, q, q.cpu(), cu, 4),
                 lambda: c.attend(0, q.cpu(), q.clone(), cu, 4), lambda: c.prompt(q, k, k, q.clone(), cu.cpu(), 4)):
        with pytest.raises(ValueError, match="device"):
            call()
