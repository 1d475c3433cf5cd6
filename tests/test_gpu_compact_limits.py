"""Compaction of more rows than an int32 numbers: the same resources listed many times, or one route of that many rows.  What is below the
limits comes out as ever, the rest is reported, and nothing is written outside the lists that were given."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import small_cache as orc
from paper_2608_19662_b200 import ReCache, binding, workloads as wl

from pipeline import dev, f64

pytestmark = pytest.mark.gpu

LIMIT = 2 ** 31 - 4096
POOL = 1 << 20
D = 64


class Listed:
    """A pool whose keep mask drops a token in a thousand, listed whole, many times over."""

    def __init__(self, g, lists, pt, width, capacity=5000, free=10):
        self.g, self.pt, self.n = g, pt, len(lists)
        rng = np.random.default_rng(5)
        self.kc = torch.zeros((g, POOL, D), dtype=torch.bfloat16, device="cuda")
        self.rows = wl.normal(8, (g, 1200, D), torch.bfloat16)
        self.kc[:, :1200] = dev(self.rows)
        keep = np.ones(POOL, np.uint8)
        keep[rng.integers(0, POOL, POOL // 1000)] = 0
        self.kept = np.flatnonzero(keep)
        off = np.cumsum([0] + [len(x) for x in lists]).astype(np.int32)
        flat = [n for x in lists for n in x]                    # lengths; all resources start at row 0
        i32 = lambda x: dev(np.asarray(x, np.int32))
        full = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")
        self.args = (dev(keep), i32(off), i32(np.zeros(len(flat))), i32(flat), torch.ones((g, len(flat)), dtype=torch.uint8, device="cuda"))
        self.lens = [sum(int(np.searchsorted(self.kept, n)) for n in x) for x in lists for _ in range(g)]
        self.cu, self.len = full(len(self.lens) + 1), full(len(self.lens))
        self.around = full(capacity + 2 * POOL)                 # the list lies in the middle of this
        self.idx = self.around[POOL:POOL + capacity]
        self.table = full(len(self.lens), width)
        self.free = rng.permutation(free + 3).astype(np.int32)[:free]
        self.rc = ReCache(g, g, D, 1e4, "bf16", max_pos=64, page_tokens=pt)

    def check_lists(self, first):
        """Prefix, lengths and list; first: the lengths of the resources that the list's room reaches into."""
        want = np.minimum(np.concatenate([[0], np.cumsum(np.asarray(self.lens, np.int64))]), LIMIT)
        assert np.array_equal(self.cu.cpu().numpy(), want)
        assert np.array_equal(self.len.cpu().numpy(), np.minimum(self.lens, LIMIT))
        rows = np.concatenate([self.kept[:np.searchsorted(self.kept, n)] for n in first])[:len(self.idx)]
        assert len(rows) == len(self.idx) and np.array_equal(self.idx.cpu().numpy(), rows)
        around = self.around.cpu().numpy()
        assert (around[:POOL] == -7).all() and (around[POOL + len(self.idx):] == -7).all()
        return rows

    def check_pages8(self, rows, k8, ks, n_pages, route=0):
        table = self.table.cpu().numpy()
        assert np.array_equal(table[route, :n_pages], self.free[:n_pages])
        for p in range(n_pages):
            want, s = orc.pack_page(f64(self.rows)[route % self.g][rows[p * self.pt:(p + 1) * self.pt]])
            assert ks[self.free[p]] == s and np.array_equal(f64(k8.view(torch.float8_e4m3fn).float())[self.free[p], :len(want)], want)


def pages8(n, pt):
    return torch.zeros((n, pt, D), dtype=torch.uint8, device="cuda"), torch.full((n,), -7.0, device="cuda")


def pack8(l):
    (k8, ks), (v8, vs) = pages8(len(l.free) + 3, l.pt), pages8(len(l.free) + 3, l.pt)
    l.rc.compact_routes_q8(l.kc, l.kc, *l.args, l.cu, l.idx, k8, v8, ks, vs, l.table, dev(l.free), route_len=l.len)
    return l.rc.poll_status(), k8, v8, ks, vs


def test_packing_many_routes_of_many_rows():
    """128 routes of 17 million rows."""
    l = Listed(2, [[POOL] * 17] * 64, 64, -(-17 * POOL // 64))
    code, k8, v8, ks, vs = pack8(l)
    assert code == 3
    rows = l.check_lists([POOL])
    l.check_pages8(rows, k8, ks, 10)
    assert torch.equal(k8, v8) and torch.equal(ks, vs) and int((ks == -7).sum()) == 3
    l.table[0, :10] = -1
    assert (l.table == -1).all()


def test_packing_a_route_of_too_many_rows():
    """Between two short ones, whose rows it leaves as they are or pushes out of the list."""
    l = Listed(1, [[1000], [POOL] * 2100, [700]], 64, 40)
    code, k8, v8, ks, vs = pack8(l)
    assert code in (3, 4, 5)                                    # first come: list, page table and free pages are all too short
    rows = l.check_lists([1000, POOL])
    first = -(-l.lens[0] // 64)
    assert first > 10                                           # (the free pages all go to the first route)
    l.check_pages8(rows, k8, ks, 10)
    assert torch.equal(k8, v8) and torch.equal(ks, vs)
    table = l.table.cpu().numpy()
    assert (table[0, 10:] == -1).all() and (table[1:] == -1).all()


def test_packing_many_routes_into_other_pages():
    l = Listed(2, [[POOL] * 17] * 64, 48, 24)
    code, k8, v8, ks, vs = pack8(l)
    assert code in (3, 4, 5)
    rows = l.check_lists([POOL])
    l.check_pages8(rows, k8, ks, 10)
    assert torch.equal(k8, v8) and torch.equal(ks, vs) and int((ks == -7).sum()) == 3
    l.table[0, :10] = -1
    assert (l.table == -1).all()


def test_packing_a_route_of_too_many_rows_into_other_pages():
    l = Listed(1, [[300], [POOL] * 2100, [700]], 48, 40)
    code, k8, v8, ks, vs = pack8(l)
    assert code in (3, 4, 5)
    rows = l.check_lists([300, POOL])
    l.check_pages8(rows[:l.lens[0]], k8, ks, 7)
    table = l.table.cpu().numpy()
    assert (table[0, 7:] == -1).all() and np.array_equal(table[1, :3], l.free[7:]) and (table[1, 3:] == -1).all() and (table[2] == -1).all()
    for p in range(3):                                          # the long route's first rows
        want, s = orc.pack_page(f64(l.rows)[0][l.kept[p * 48:(p + 1) * 48]])
        assert ks[l.free[7 + p]] == s and np.array_equal(f64(k8.view(torch.float8_e4m3fn).float())[l.free[7 + p]], want)


@pytest.mark.parametrize("lists,g", [([[POOL] * 17] * 64, 2), ([[POOL // 2] * 40] * 64, 2), ([[1000], [POOL] * 2100, [700]], 1), ([[1000], [POOL] * 4200, [700]], 1)],
                         ids=["many", "many-planned", "long", "long-planned"])
@pytest.mark.parametrize("copies", [True, False])
def test_packed_rows(lists, g, copies):
    """The copying compaction, with a launch that plans and (up to 4096 pairs of resource and group) without."""
    l = Listed(g, lists, 64, 1)
    out = torch.full((2, 5000 + 4096, D), 9.0, dtype=torch.bfloat16, device="cuda")
    ko, vo = (out[i, 2048:2048 + 5000] for i in range(2))
    l.rc.compact_routes(l.kc, l.kc, *l.args, 0, l.cu, l.idx, *((ko, vo) if copies else (None, None)), route_len=l.len)
    assert l.rc.poll_status() == 3
    rows = l.check_lists([lists[0][0], POOL])
    want = l.kc[0][torch.from_numpy(rows).cuda()] if copies else torch.full_like(ko, 9.0)
    assert torch.equal(ko, want) and torch.equal(vo, want)
    assert (out[:, :2048] == 9).all() and (out[:, 2048 + 5000:] == 9).all()


def test_paged_rows():
    l = Listed(2, [[POOL] * 17] * 64, 64, 24)
    pages = torch.full((2, 13, 64, D), 9.0, dtype=torch.bfloat16, device="cuda")
    l.rc.compact_routes(l.kc, l.kc, *l.args, 1, l.cu, l.idx, pages[0], pages[1], route_len=l.len, page_table=l.table, free_pages=dev(l.free))
    assert l.rc.poll_status() in (3, 4, 5)
    rows = l.check_lists([POOL])
    assert np.array_equal(l.table[0, :10].cpu().numpy(), l.free) and (l.table[0, 10:] == -1).all() and (l.table[1:] == -1).all()
    want = torch.full((13, 64, D), 9.0, dtype=torch.bfloat16, device="cuda")
    want[torch.from_numpy(l.free).cuda().long()] = l.kc[0][torch.from_numpy(rows[:640]).cuda()].view(10, 64, D)
    assert torch.equal(pages[0], want) and torch.equal(pages[1], want)


@pytest.mark.parametrize("call", ["recache_compact_routes", "recache_compact_routes_q8"])
def test_more_routes_than_are_numbered_are_refused(call):
    """On the host, before anything is looked at: no pointer here leads anywhere."""
    rc = ReCache(8, 8, D, 1e4, "bf16", max_pos=64)
    types = binding.SIGNATURES[call][1]
    args = [256 if t is ctypes.c_void_p else 0 for t in types]
    args[0] = rc.h
    n_requests = 8                                              # its place, behind context, caches, pool, mask and lists
    for args[n_requests] in (2 ** 30 // 8 + 1, 2 ** 31 - 1):
        assert getattr(rc.lib, call)(*args) == 2
        assert "2^30 routes" in rc.lib.recache_last_error(rc.h).decode()


def test_words_that_are_not_aligned_are_refused():
    """Scales and workspace, each a byte or two off; with no request, so that nothing would be read there."""
    rc = ReCache(2, 2, D, 1e4, "bf16", max_pos=64)
    room = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    p = room.data_ptr()
    args = dict(ctx=rc.h, k_cache=p, v_cache=p, pool_tokens=0, keep=p, res_off=p, res_slot=p, res_len=p, n_requests=0, total_listed=0, vis=p, route_cu=p + 256, route_len=None,
                route_idx=p, row_capacity=0, k8=p, v8=p, k_scale=p + 512, v_scale=p + 768, page_table=p, max_pages=1, free_pages=p, n_free=1, n_pool=1, workspace=p + 1024,
                workspace_bytes=1 << 15, stream=torch.cuda.current_stream().cuda_stream)
    assert rc.lib.recache_compact_routes_q8(*args.values()) == 0
    for name, by in (("k_scale", 1), ("v_scale", 2), ("workspace", 1), ("workspace", 2), ("workspace", 3)):
        assert rc.lib.recache_compact_routes_q8(*{**args, name: args[name] + by}.values()) == 1
        assert "4-byte aligned" in rc.lib.recache_last_error(rc.h).decode()
    assert rc.poll_status() == 0
