"""8-bit pages, weights and eviction where the other tests do not lead: replays that have everything to write again, larger pools, both launches of the
append, packing past the first turn of its rings, streams and wide tables."""
import copy

import numpy as np
import pytest
import torch

from oracle import recache_oracle as base
from paper_2608_19662_b200 import ReCache, workloads as wl

from pipeline import dev, f64
from small_cache import U, Step, tables

pytestmark = pytest.mark.gpu

PT = 64


def ctx(hq=32, g=8, d=128, dtype="bf16", pt=64):
    return ReCache(hq, g, d, 1e4, dtype, max_pos=16384, page_tokens=pt)


def raw(t):
    return t.contiguous().view(torch.uint8)


def full(value, *shape, t=torch.int32):
    return torch.full(shape, value, dtype=t, device="cuda")


class Pack:
    """A compaction into 8-bit pages; everything it writes holds something else before."""

    def __init__(self, seed, pt=64, g=4, d=128, n_requests=5):
        rng = np.random.default_rng([seed, 9])
        self.rc, self.pt = ctx(2 * g, g, d, pt=pt), pt
        length = rng.integers(20, 700, 8)
        slot = np.concatenate([[0], np.cumsum(length)[:-1]])
        pool = int(length.sum())
        lists = [rng.integers(0, 8, int(rng.integers(1, 6))) for _ in range(n_requests)]
        flat = np.concatenate(lists)
        self.kc, self.vc = (dev(wl.normal(seed * 3 + i, (g, pool, d), torch.bfloat16)) for i in range(2))
        i32 = lambda x: dev(np.asarray(x, np.int32))
        self.lists = (dev((rng.random(pool) < 0.5).astype(np.uint8)), i32(np.cumsum([0] + [len(x) for x in lists])), i32(slot[flat]), i32(length[flat]),
                      dev((rng.random((g, len(flat))) < 0.7).astype(np.uint8)))
        routes, n = n_requests * g, 400
        self.out = dict(cu=full(-7, routes + 1), idx=full(-7, 20000), k8=full(0x55, n, pt, d, t=torch.uint8), v8=full(0x55, n, pt, d, t=torch.uint8),
                        ks=full(-7.0, n, t=torch.float32), vs=full(-7.0, n, t=torch.float32), table=full(-7, routes, 90), len=full(-7, routes))
        self.free = i32(rng.permutation(n))
        self.ws = full(0, 1 << 16, t=torch.uint8)

    def run(self):
        o = self.out
        self.rc.compact_routes_q8(self.kc, self.vc, *self.lists, o["cu"], o["idx"], o["k8"], o["v8"], o["ks"], o["vs"], o["table"], self.free, route_len=o["len"], workspace=self.ws)


class Evict:
    def __init__(self, seed, lens, budget, recent, d=128, wide=0):
        rng = np.random.default_rng([seed, 8])
        self.rc, self.budget, self.recent = ctx(4, 2, d), budget, recent
        t = tables(rng, -(-np.asarray(lens) // PT))
        n, new = int(t.max()) + 1, -(-budget // PT)
        spare = new * len(lens)
        self.table, self.lens = dev(np.concatenate([t, np.full((len(lens), wide), -1, np.int32)], 1)), dev(np.asarray(lens, np.int32))
        self.free = dev((n + rng.permutation(spare)).astype(np.int32))
        k, v = (wl.normal(seed * 5 + i, (n + spare, PT, d), torch.bfloat16) for i in range(2))
        w = torch.from_numpy(np.exp(2 * rng.standard_normal((n + spare, PT))).astype(np.float32))
        for x in (k, v, w):
            x[n:] = float("nan")
        self.out = dict(k=dev(k), v=dev(v), w=dev(w), table=full(-7, len(lens), new), len=full(-7, len(lens)), kept=full(-7, len(lens), budget))

    def run(self):
        o = self.out
        self.rc.evict_rows(o["k"], o["v"], o["w"], self.table, self.lens, self.budget, self.recent, self.free, o["table"], o["len"], o["kept"])


class Decode:
    def __init__(self, seed, q8, batch=6):
        s = self.st = Step(seed, 16, 4, 128, "bf16", batch, (0, 500), (1, 400), q8)
        self.rc = ctx(16, 4)
        self.x = {k: dev(getattr(s, k)) for k in ("q", "pos", "rt", "res", "ht", "hist", "kn", "vn", "w")}
        self.q8 = [dev(x) for x in (s.k8, s.v8, s.ks, s.vs)] if q8 else []
        kp, vp = s.kp.clone(), s.vp.clone()
        last = s.hist - 1
        for p in (kp, vp):                                      # what the append has to write
            p[s.ht[np.arange(len(last)), last // PT], last % PT] = float("nan")
        self.out = dict(kp=dev(kp), vp=dev(vp), wo=full(-7.0, *s.w.shape, t=torch.float32), o=full(9.0, batch, 16, 128, t=torch.float32))
        self.ws = full(0, self.rc.decode_weighted_workspace_bytes(batch, s.kp.shape[0]), t=torch.uint8)

    def run(self):
        x, o = self.x, self.out
        more = dict(k_new=x["kn"], v_new=x["vn"], weight_in=x["w"], out=o["o"], workspace=self.ws)
        if self.q8:
            self.rc.attend_decode_q8(x["q"], x["pos"], *self.q8, x["rt"], x["res"], o["kp"], o["vp"], x["ht"], x["hist"], weight_out=o["wo"], **more)
        else:
            self.rc.attend_decode_weighted(x["q"], x["pos"], o["kp"], o["vp"], x["rt"], x["res"], x["ht"], x["hist"], o["wo"], **more)


def test_replays_write_everything_again():
    """All calls in one graph, eviction with one block an item and with a cluster; all that they write is put back before each replay, and the inputs
    of the second are other ones."""
    parts = [Pack(1), Pack(2, pt=48), Decode(3, True), Decode(4, False), Evict(5, [700, 100, 431], 250, 30), Evict(6, [9000, 70, 20000, 5000], 4000, 100)]
    fresh = [{k: v.clone() for k, v in p.out.items()} for p in parts]

    def reset():
        for p, f in zip(parts, fresh):
            for k, v in f.items():
                p.out[k].copy_(v)

    def eager():
        reset()
        for p in parts:
            p.run()
        torch.cuda.synchronize()
        want = [{k: v.clone() for k, v in p.out.items()} for p in parts]
        for w, f in zip(want, fresh):
            for k in w:
                assert not torch.equal(raw(w[k]), raw(f[k])), k
        return want

    first = eager()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            for p in parts:
                p.run()
    torch.cuda.synchronize()

    def compare(want):
        reset()
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        for i, (p, w) in enumerate(zip(parts, want)):
            for k in w:
                assert torch.equal(raw(p.out[k]), raw(w[k])), (i, k)

    compare(first)
    for p in parts:                                             # other rows, queries, lengths and weights, in place
        if isinstance(p, Pack):
            p.kc.mul_(-3.0)
            p.lists[0].copy_(1 - p.lists[0])
        elif isinstance(p, Decode):
            p.x["q"].mul_(-0.5)
            p.x["res"].sub_(torch.clamp(p.x["res"], max=7))
        else:
            p.lens.sub_(3)
    for p, f in zip(parts, fresh):
        if isinstance(p, Evict):
            f["w"].copy_(torch.where(f["w"].isnan(), f["w"], f["w"].flip(1).nan_to_num(2.0)))
    second = eager()
    assert not torch.equal(first[2]["o"], second[2]["o"]) and not torch.equal(first[4]["kept"], second[4]["kept"])
    compare(second)
    assert all(p.rc.poll_status() == 0 for p in parts)


def test_streams_that_pack_and_evict_at_once():
    """The last of them packs more rows than its list and its free pages hold, and says so each time."""
    make = [lambda: Pack(11), lambda: Evict(12, [9000, 70, 20000], 4000, 100), lambda: Pack(13, pt=32), lambda: Evict(14, [300] * 60 + [900], 200, 7), lambda: Pack(15, n_requests=40)]
    parts = [m() for m in make]
    want = []
    for p in parts:
        fresh = {k: v.clone() for k, v in p.out.items()}
        p.run()
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in p.out.items()})
        p.fresh, p.code = fresh, p.rc.poll_status()
    assert [p.code for p in parts] == [0, 0, 0, 0, 3]
    streams = [torch.cuda.Stream() for _ in parts]
    for _ in range(5):
        for p in parts:
            for k, v in p.fresh.items():
                p.out[k].copy_(v)
        torch.cuda.synchronize()
        for p, s in zip(parts, streams):
            with torch.cuda.stream(s):
                p.run()
        torch.cuda.synchronize()
        for i, (p, w) in enumerate(zip(parts, want)):
            for k in w:
                assert torch.equal(raw(p.out[k]), raw(w[k])), (i, k)
            assert p.rc.poll_status() == p.code


@pytest.mark.parametrize("wide", [200, 5000])
def test_eviction_with_wide_tables(wide):
    """Blocks to an item and keys in shared memory go by the table's width; the result does not."""
    for lens, budget, recent in (([700, 100, 431], 250, 30), ([300] * 40, 299, 7), ([9000, 70, 20000, 5000], 4000, 100), ([130, 200] * 160, 128, 5)):
        a, b = Evict(21, lens, budget, recent), Evict(21, lens, budget, recent, wide=wide)
        a.run()
        b.run()
        for k in a.out:
            assert torch.equal(raw(a.out[k]), raw(b.out[k])), k
        assert a.rc.poll_status() == 0 and b.rc.poll_status() == 0


@pytest.mark.parametrize("q8", [True, False], ids=["q8", "same"])
def test_a_larger_pool_gives_the_same_bits(q8):
    rc = ctx()
    st = Step(22, 32, 8, 128, "bf16", 5, (0, 900), (1, 700), q8)
    a = st.call(rc)
    n = st.kp.shape[0]
    more = torch.full((333, PT, 128), float("nan"), dtype=torch.bfloat16)
    st.kp, st.vp, st.w = torch.cat([st.kp, more]), torch.cat([st.vp, more]), torch.cat([st.w, more[:, :, 0].float()])
    b = st.call(rc)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1][:n]) and (b[1][n:] == -7).all()
    assert torch.equal(raw(a[2]), raw(b[2][:n])) and torch.equal(raw(a[3]), raw(b[3][:n])) and rc.poll_status() == 0


@pytest.mark.parametrize("q8", [True, False], ids=["q8", "same"])
def test_both_launches_of_the_append(q8):
    """More than four items a multiprocessor append in a launch of their own; the first of them alone do not.  The same rows either way."""
    rc = ctx(16, 4)
    st = Step(23, 16, 4, 128, "bf16", 160, (0, 200), (1, 200), q8)
    few = copy.copy(st)
    b, items = 100, 400
    few.batch, few.q, few.pos, few.kn, few.vn = b, st.q[:b], st.pos[:b], st.kn[:b], st.vn[:b]
    few.rt, few.res, few.ht, few.hist = st.rt[:items], st.res[:items], st.ht[:items], st.hist[:items]
    many, some = st.call(rc), few.call(rc)
    last = st.hist - 1
    page, slot = (torch.from_numpy(x.astype(np.int64)) for x in (st.ht[np.arange(len(last)), last // PT], last % PT))
    for pool, part, old in ((many[2], some[2], st.kp), (many[3], some[3], st.vp)):
        new = pool.cpu()[page, slot]
        assert torch.equal(raw(new[:items]), raw(part.cpu()[page[:items], slot[:items]]))
        assert torch.equal(raw(part.cpu()[page[items:], slot[items:]]), raw(old[page[items:], slot[items:]]))
        assert not torch.equal(new, old[page, slot])
    # probabilities are rounded to eight bits against other running maxima: half a step each, on both sides
    assert (many[0][:b] - some[0]).abs().max() <= 2 * 1.01 * U["bf16"] * float(st.vp[~st.vp.isnan()].abs().max() if not q8 else 8.0)
    assert rc.poll_status() == 0


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 128), ("f32", 64)])
def test_packing_turns_its_rings_over(dtype, d):
    """Three times and more: some 200 pages to a block (of 296, or 148 where a block takes an SM), where a ring holds 32 of a block's half."""
    rng = np.random.default_rng(31)
    g, blocks = 2, 148 if (dtype, d) == ("f32", 128) else 296
    length = rng.integers(0, 3000, 30)
    slot = np.concatenate([[0], np.cumsum(length)[:-1]]).astype(np.int32)
    pool = int(length.sum())
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    kc, vc = (dev(wl.normal(i, (g, pool, d), t) * 3) for i in (1, 2))
    keep = (rng.random(pool) < 0.6).astype(np.uint8)
    lists, rows = [], 0
    while rows < blocks * 200 * 64:
        lists.append(rng.integers(0, 30, 25))
        rows += int(1.2 * 0.6 * length[lists[-1]].sum())
    flat = np.concatenate(lists)
    off = np.cumsum([0] + [25] * len(lists)).astype(np.int32)
    vis = (rng.random((g, len(flat))) < 0.6).astype(np.uint8)
    routes = [r for b in base.compact_routes(keep, off, slot[flat], length[flat], vis) for r in b]
    lens = np.array([len(r) for r in routes])
    n_pages = -(-lens // PT)
    total = int(n_pages.sum())
    assert total > blocks * 190
    free = rng.permutation(total + 5).astype(np.int32)
    cap, width = int(lens.sum()), int(n_pages.max()) + 1
    cu, idx, table, out_len = full(-7, len(lens) + 1), full(-7, cap), full(-7, len(lens), width), full(-7, len(lens))
    k8, v8 = (full(0x55, total + 5, PT, d, t=torch.uint8) for _ in range(2))
    ks, vs = (full(-7.0, total + 5, t=torch.float32) for _ in range(2))
    rc = ReCache(g, g, d, 1e4, dtype, max_pos=64)
    rc.compact_routes_q8(kc, vc, dev(keep), dev(off), dev(slot[flat]), dev(length[flat].astype(np.int32)), dev(vis), cu, idx, k8, v8, ks, vs, table, dev(free), route_len=out_len)
    assert rc.poll_status() == 0
    assert np.array_equal(cu.cpu().numpy(), np.concatenate([[0], np.cumsum(lens)])) and np.array_equal(out_len.cpu().numpy(), lens)
    assert np.array_equal(idx.cpu().numpy(), np.concatenate(routes))
    want_table = np.full((len(lens), width), -1, np.int32)
    place = np.zeros((total, PT), np.int64)                     # rows of each page in turn; behind a route's end -1
    at = 0
    for r, n in enumerate(n_pages):
        want_table[r, :n] = free[at:at + n]
        p = np.full(n * PT, -1, np.int64)
        p[:lens[r]] = routes[r] + (r % g) * pool
        place[at:at + n] = p.reshape(n, PT)
        at += n
    assert np.array_equal(table.cpu().numpy(), want_table)
    place, ids = dev(place), dev(free[:total].astype(np.int64))
    there = place >= 0
    for cache, p8, sc in ((kc, k8, ks), (vc, v8, vs)):
        for a in range(0, total, 8192):
            m = there[a:a + 8192]
            x = torch.where(m[:, :, None], cache.view(g * pool, d)[place[a:a + 8192].clamp(min=0)].double(), 0.0)
            f, e = torch.frexp(x.abs().amax((1, 2)))            # 448 = 0.875 * 2^9
            scale = torch.ldexp(torch.ones_like(f), e - 9 + (f > 0.875).int())
            got = p8[ids[a:a + 8192]]
            assert torch.equal(sc[ids[a:a + 8192]].double(), scale)
            want = (x / scale[:, None, None]).float().to(torch.float8_e4m3fn).view(torch.uint8)
            assert torch.equal(got[m], want[m]) and (got[~m] == 0x55).all()
        assert (p8[dev(free[total:].astype(np.int64))] == 0x55).all() and (sc[dev(free[total:].astype(np.int64))] == -7).all()
