"""The page plan and the store on the GPU against the oracle, and the paged
operators together as a serving program uses them."""
import numpy as np
import pytest

from gpu_util import dev, host, log
from gqa_util import TYPES, desc, torch_types
from oracle.paged import EXHAUSTED, INVALID, WIDTH, pages_of, plan

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    seer.load_library()
    return seer


class Book:
    """The device's book-keeping beside the oracle's."""

    def __init__(self, S, B, W, P, page, seed=0):
        self.S, self.page, self.P, self.B = S, page, P, B
        self.pages = S.seer_page_desc(page, P, W)
        self.table, self.held = [[-1] * W for _ in range(B)], [0] * B
        self.free = np.random.default_rng(seed).permutation(P).tolist()
        self.to_device()

    def to_device(self):
        pad = self.free + [-5] * (self.P - len(self.free))
        self.free_d, self.table_d = dev(np.array(pad)), dev(np.array(self.table))
        self.count = [dev(np.array([len(self.free)])), dev(np.array([77]))]
        self.kv = [dev(np.array(self.held)), dev(np.full(self.B, 99))]
        self.status = dev(np.array([55]))

    def step(self, keep, lens, used=None, rows_ub=None, free_count=None):
        rows_ub = sum(lens) + 3 if rows_ub is None else rows_ub
        want = plan(self.held, keep, lens, used, self.table, self.free, self.page, self.P, rows_ub)
        cu = np.concatenate([[0], np.cumsum(lens)])
        slots = dev(np.full(max(rows_ub, 1), -7))
        self.S.seer_page_plan(self.pages, self.kv[0], dev(np.array(keep)), dev(cu),
                              None if used is None else dev(np.array(used)), self.B, rows_ub, self.free_d,
                              self.count[0], self.count[1], self.table_d, self.kv[1], slots if rows_ub else None,
                              self.status)
        assert host(self.status).item() == want["status"]
        assert host(self.kv[1]).tolist() == want["kv_len"]
        assert host(self.table_d).tolist() == want["table"]
        n = host(self.count[1]).item()
        assert n == len(want["free"]) and host(self.free_d)[:n].tolist() == want["free"]
        if rows_ub:
            assert host(slots).tolist() == want["slots"]
        self.table, self.free, self.held = want["table"], want["free"], want["kv_len"]
        self.count.reverse()
        self.kv.reverse()
        return want


@pytest.mark.parametrize("B,W,P,page", [(1, 1, 1, 16), (3, 7, 15, 16), (40, 9, 200, 32), (300, 5, 900, 256),
                                        (1000, 4, 2500, 64)])
def test_plan_over_many_steps(S, B, W, P, page):
    rng = np.random.default_rng(B)
    bk = Book(S, B, W, P, page)
    done = {0: 0}
    for i in range(25):
        log("plan step %d of %d requests" % (i, B))
        keep = [int(rng.integers(0, h + 1)) if rng.random() < 0.3 else (0 if rng.random() < 0.1 else h) for h in bk.held]
        most = [1, 3 * page // 2, 0][i % 3]
        lens = [int(rng.integers(0, most + 1)) for _ in range(B)]
        used = [int(rng.integers(-1, n + 2)) for n in lens] if i % 2 else None
        st = bk.step(keep, lens, used, rows_ub=0 if sum(lens) == 0 else None)["status"]
        done[st] = done.get(st, 0) + 1
    assert done[0] >= 5


def test_plan_refusals_on_the_device(S):
    bk = Book(S, 3, 4, 8, 16)
    assert bk.step([0, 0, 0], [33, 0, 20])["status"] == 0
    assert bk.step([33, 0, 20], [0, 64, 0])["status"] == EXHAUSTED          # 3 free, 4 needed
    assert bk.step([33, 0, 20], [0, 65, 0])["status"] == WIDTH
    assert bk.step([34, 0, 20], [0, 1, 0])["status"] == INVALID             # keeps more than it holds
    assert bk.step([-1, 0, 20], [0, 1, 0])["status"] == INVALID
    assert bk.step([0, 0, 20], [0, 64, 0])["status"] == 0                   # with the pages that the first one gives back
    assert bk.step([0, 64, 20], [16, 0, 0])["status"] == 0
    # a free count that the pool contradicts
    bk.count[0].fill_(9)
    import torch
    before = bk.table_d.clone()
    out = dev(np.array([5]))
    slots = dev(np.array([5, 5]))
    for bad in (9, -1):
        bk.count[0].fill_(bad)
        S.seer_page_plan(bk.pages, bk.kv[0], bk.kv[0], dev(np.array([0, 1, 1, 2])), None, 3, 2, bk.free_d, bk.count[0], out,
                         bk.table_d, bk.kv[1], slots, bk.status)
        assert host(bk.status).item() == INVALID and host(out).item() == bad
        assert torch.equal(before, bk.table_d) and host(slots).tolist() == [-1, -1]


def test_plan_of_long_requests(S):
    """Lengths past 2^31 tokens in the pages' bytes are not reached; lengths near the table's width are."""
    bk = Book(S, 2, 4000, 6000, 256)
    assert bk.step([0, 0], [4000 * 256, 300])["status"] == 0
    assert bk.step([4000 * 256, 300], [1, 0], rows_ub=5)["status"] == WIDTH
    assert bk.step([1, 300], [0, 5])["status"] == 0


@pytest.mark.parametrize("kind,KV,D,page", [("bf16", 2, 128, 16), ("v16", 3, 64, 64), ("f32", 1, 4, 256), ("f32", 5, 80, 32),
                                            ("bf16", 32, 128, 128)])
def test_store(S, kind, KV, D, page):
    import torch
    qt, vt = torch_types(kind)
    rng = np.random.default_rng(KV)
    P, rows = 9, 70
    d, pages = desc(S, kind, KV, KV, D), S.seer_page_desc(page, P, 4)
    buf = torch.randn(rows, 2 * KV * D + 8 * (16 // torch.empty(0, dtype=qt).element_size()), device="cuda").to(qt)
    k, v = buf[:, :KV * D], buf.view(vt)[:, KV * D:2 * KV * D]
    pool = torch.full((P, 2, KV, page, D), 3.0, dtype=qt, device="cuda")
    slots = rng.permutation(P * page)[:rows]
    slots[[0, 5, 8]] = [-1, P * page, 2 ** 31 - 1]               # skipped
    want = pool.clone()
    for r, s in enumerate(slots):
        if 0 <= s < P * page:
            want[s // page, 0, :, s % page] = k[r].view(KV, D)
            want.view(vt)[s // page, 1, :, s % page] = v[r].view(KV, D)
    S.seer_kv_store(d, pages, k, buf.stride(0), v, buf.stride(0), rows, dev(slots), pool)
    assert pool.cpu().view(torch.uint8).equal(want.cpu().view(torch.uint8))


def test_store_of_more_rows_than_a_launch_has_waves(S):
    import torch
    n = (1 << 24) + 5
    d, pages = S.seer_attn_desc(1, 1, 4, S.SEER_DTYPE_F32, 0, 0.0), S.seer_page_desc(16, 2, 1)
    k = torch.zeros(n, 4, device="cuda")
    k[0], k[n - 1], k[1 << 24] = 1.0, 2.0, 3.0
    slots = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    slots[0], slots[n - 1], slots[1 << 24] = 17, 3, 30
    pool = torch.full((2, 2, 1, 16, 4), 9.0, device="cuda")
    S.seer_kv_store(d, pages, k, 4, k, 4, n, slots, pool)
    want = torch.full((2, 2, 1, 16, 4), 9.0)
    want[1, :, 0, 1], want[0, :, 0, 3], want[1, :, 0, 14] = 1.0, 2.0, 3.0
    assert torch.equal(pool.cpu(), want)
