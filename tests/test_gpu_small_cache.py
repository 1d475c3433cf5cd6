"""8-bit pages, attention weights and eviction as a serving loop uses them together, and what surrounds the calls: graphs,
streams, far offsets, refusals and device status codes."""
import numpy as np
import pytest
import torch

from oracle import recache_oracle as base
from oracle import small_cache as orc
from paper_2608_19662_b200 import ReCache, ReCacheError, workloads as wl

from pipeline import dev, f64
from small_cache import U, Step, tables

pytestmark = pytest.mark.gpu

PT = 64


def ctx(hq=32, g=8, d=128, dtype="bf16", pt=64):
    return ReCache(hq, g, d, 1e4, dtype, max_pos=16384, page_tokens=pt)


def test_a_conversation_over_packed_resources_with_eviction():
    """Resources are packed into 8-bit pages; every step appends a token and adds to the weights of the conversation's rows; past a budget the
    conversation is cut back, and the next steps run over what is left.  Each step against the oracle over the pages as they are."""
    hq, g, d, batch, budget, recent = 16, 4, 128, 3, 150, 20
    rc = ctx(hq, g)
    rng = np.random.default_rng(3)
    sh = wl.Shape(hq, g, d, 1e4, "bf16")
    length = rng.integers(100, 400, 6)
    slot = np.concatenate([[0], np.cumsum(length)[:-1]]).astype(np.int32)
    pool = int(length.sum())
    kc, vc = (wl.normal(s, (g, pool, d), sh.torch_dtype) for s in (1, 2))
    keep = (rng.random(pool) < 0.5).astype(np.uint8)
    res_off, vis = np.array([0, 2, 4, 6], np.int32), (rng.random((g, 6)) < 0.7).astype(np.uint8)
    n8 = 64
    k8, v8 = (torch.full((n8, PT, d), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.full((n8,), float("nan"), device="cuda") for _ in range(2))
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    r_cu, r_len, r_idx, r_table = z(batch * g + 1), z(batch * g), z(pool * g), z(batch * g, 16)
    rc.compact_routes_q8(dev(kc), dev(vc), dev(keep), dev(res_off), dev(slot), dev(length.astype(np.int32)), dev(vis), r_cu, r_idx, k8, v8, ks, vs, r_table,
                         dev(rng.permutation(n8).astype(np.int32)), route_len=r_len)
    res_len, rt = r_len.cpu().numpy(), r_table.cpu().numpy()
    rows = base.compact_routes(keep, res_off, slot, length, vis)
    assert np.array_equal(res_len, [len(rows[b][k]) for b in range(batch) for k in range(g)])
    # conversation: a pool with free pages, every item starts with some rows
    items, n_pages, width = batch * g, 120, 4
    free = list(rng.permutation(n_pages).astype(np.int32))
    hist = np.repeat(rng.integers(100, 140, batch), g).astype(np.int32)
    ht = np.full((items, width), -1, np.int32)
    for it in range(items):
        for p in range(-(-int(hist[it]) // PT)):
            ht[it, p] = free.pop()
    kp, vp = (dev(wl.normal(s, (n_pages, PT, d), sh.torch_dtype)) for s in (3, 4))
    w = torch.zeros((n_pages, PT), device="cuda")
    pos = np.full(batch, 2000, np.int32)
    k8f, v8f = f64(k8.float()), f64(v8.float())
    want_w = [np.zeros(int(n)) for n in hist]
    for step in range(25):
        hist = hist + 1
        for it in range(items):
            if (hist[it] - 1) % PT == 0:
                ht[it, (hist[it] - 1) // PT] = free.pop()
        pos = pos + 1
        q, kn, vn = (wl.normal(100 * step + i, (batch, h, d), sh.torch_dtype) for i, h in enumerate((hq, g, g)))
        o = rc.attend_decode_q8(dev(q), dev(pos), k8, v8, ks, vs, r_table, r_len, kp, vp, dev(ht), dev(hist), k_new=dev(kn), v_new=dev(vn), weight_in=w, weight_out=w,
                                out_dtype=torch.float32)
        ref, got = orc.attend_decode(f64(q), pos, (k8f, v8f, f64(ks), f64(vs)), f64(kp), f64(vp), rt, res_len, ht, hist, 1e4, PT, storage="bf16")
        # probabilities meet bf16 values in bf16; a rotated query element next to a border of bf16 may be a step off, which moves a score by up to
        # 2^-7 |q||k| / sqrt(d) < 0.012 for one of |q|, |k| <= 4: one such element a head
        vmax = max(np.abs(f64(vp)).max(), 8.0)
        assert np.abs(f64(o) - ref).max() <= (U["bf16"] + 2 * 0.012) * vmax
        for it in range(items):
            want_w[it] = np.append(want_w[it], 0.0) + got[it][int(res_len[it]):]
            pg, sl = orc.rows_of(ht[it], int(hist[it]), PT)
            have = f64(w)[pg, sl]
            assert (np.abs(have - want_w[it]) <= 0.025 * want_w[it] + 1e-6).all()
            want_w[it] = have                                  # (the sums go on from what the pages hold)
        if hist.max() > budget:
            new_table, new_len, kept = z(items, -(-budget // PT)), z(items), z(items, budget)
            before_k, before_w = f64(kp), f64(w)
            rc.evict_rows(kp, vp, w, dev(ht), dev(hist), budget, recent, dev(np.array(free, np.int32)), new_table, new_len, kept)
            nt, nl, kt = new_table.cpu().numpy(), new_len.cpu().numpy(), kept.cpu().numpy()
            after_k, after_w = f64(kp), f64(w)
            for it in range(items):
                keeps = orc.keep_rows(list(want_w[it]), budget, recent)
                assert nl[it] == len(keeps) and np.array_equal(kt[it, :nl[it]], keeps)
                old, new = orc.rows_of(ht[it], int(hist[it]), PT), orc.rows_of(nt[it], int(nl[it]), PT)
                assert np.array_equal(after_k[new[0], new[1]], before_k[old[0][keeps], old[1][keeps]])
                assert np.array_equal(after_w[new[0], new[1]], before_w[old[0][keeps], old[1][keeps]])
                if hist[it] > budget:
                    for p in nt[it][:-(-budget // PT)]:
                        free.remove(p)
                    free.extend(ht[it][:-(-int(hist[it]) // PT)])
                    ht[it] = -1
                    ht[it, :nt.shape[1]] = nt[it]
                want_w[it] = want_w[it][keeps]
            hist = nl.copy()
    assert (hist <= budget).all() and rc.poll_status() == 0


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_weights_in_place_are_those_apart(dtype, d):
    rc = ctx(8, 2, d, dtype)
    st = Step(21, 8, 2, d, dtype, 4, (0, 300), (1, 300), False)
    _, want, _, _ = st.call(rc)
    w = dev(st.w)
    rc.attend_decode_weighted(dev(st.q), dev(st.pos), dev(st.kp), dev(st.vp), dev(st.rt), dev(st.res), dev(st.ht), dev(st.hist), w, weight_in=w, k_new=dev(st.kn), v_new=dev(st.vn),
                              out_dtype=torch.float32)
    seen = want != -7.0
    assert torch.equal(w[seen], want[seen]) and torch.equal(w[~seen], dev(st.w)[~seen])


def test_the_same_inputs_give_the_same_bits_whatever_the_room():
    """Twice, with wider tables, with a larger pool and on the two launch shapes of the append."""
    rc = ctx(32, 8)
    for q8 in (True, False):
        st = Step(22, 32, 8, 128, "bf16", 5, (0, 900), (1, 700), q8)
        a = st.call(rc)
        b = st.call(rc)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        st.rt = np.concatenate([st.rt, np.full((40, 50), -1, np.int32)], 1)
        st.ht = np.concatenate([st.ht, np.full((40, 50), -1, np.int32)], 1)
        c = st.call(rc)
        assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


def test_replays_from_a_graph():
    rc = ctx(16, 4)
    a, b = Step(31, 16, 4, 128, "bf16", 6, (0, 500), (1, 400), True), Step(32, 16, 4, 128, "bf16", 6, (0, 500), (1, 400), False)
    ws = [torch.empty(rc.decode_weighted_workspace_bytes(6, x.kp.shape[0]), dtype=torch.uint8, device="cuda") for x in (a, b)]
    lens = np.array([700, 100, 431], np.int32)
    t = tables(np.random.default_rng(1), -(-lens // PT))
    n = int(t.max()) + 1
    ek, ev = (dev(wl.normal(s, (n + 12, PT, 128), torch.bfloat16)) for s in (5, 6))
    ew = torch.rand((n + 12, PT), device="cuda")
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    free, out = dev(np.arange(n, n + 12, dtype=np.int32)), (z(3, 4), z(3), z(3, 250))
    dt, dl = dev(t), dev(lens)
    kw = {}
    for x in (a, b):
        kw[x] = {k: dev(getattr(x, k)) for k in ("q", "pos", "rt", "res", "kp", "vp", "ht", "hist", "kn", "vn", "w")}
        kw[x]["wo"] = torch.zeros_like(kw[x]["w"])
        kw[x]["o"] = torch.zeros((6, 16, 128), device="cuda")
    k8, v8, ks, vs = (dev(x) for x in (a.k8, a.v8, a.ks, a.vs))

    def step():
        p = kw[a]
        rc.attend_decode_q8(p["q"], p["pos"], k8, v8, ks, vs, p["rt"], p["res"], p["kp"], p["vp"], p["ht"], p["hist"], k_new=p["kn"], v_new=p["vn"], weight_in=p["w"],
                            weight_out=p["wo"], out=p["o"], workspace=ws[0])
        p = kw[b]
        rc.attend_decode_weighted(p["q"], p["pos"], p["kp"], p["vp"], p["rt"], p["res"], p["ht"], p["hist"], p["wo"], weight_in=p["w"], k_new=p["kn"], v_new=p["vn"], out=p["o"],
                                  workspace=ws[1])
        rc.evict_rows(ek, ev, ew, dt, dl, 250, 30, free, *out)

    watched = [kw[a]["o"], kw[a]["wo"], kw[b]["o"], kw[b]["wo"], *out, ek, ew]
    step()
    torch.cuda.synchronize()
    want = [x.clone() for x in watched]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    for x in watched[:-2]:
        x.zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(watched, want)) and rc.poll_status() == 0


def test_two_streams_with_workspaces_of_their_own():
    rc = ctx(32, 8)
    steps = [Step(41 + i, 32, 8, 128, "bf16", 8, (200, 900), (100, 700), bool(i & 1)) for i in range(4)]
    want = [s.call(rc) for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    ws = [torch.empty(rc.decode_weighted_workspace_bytes(8, s.kp.shape[0]), dtype=torch.uint8, device="cuda") for s in steps]
    pools = [(dev(s.kp), dev(s.vp)) for s in steps]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, stream, w, p in zip(steps, streams, ws, pools):
            with torch.cuda.stream(stream):
                got.append(s.call(rc, pools=p, workspace=w))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_eight_bit_pages_that_several_items_list():
    """Pages that are only read: two items with the same pages, and one item with a page twice."""
    rc = ctx(16, 4)
    st = Step(53, 16, 4, 128, "bf16", 3, np.full(12, 200), (50, 200), True)
    st.rt[5] = st.rt[2]
    st.rt[9, 1] = st.rt[9, 0]
    st.check(rc, U["bf16"])


def test_a_page_that_is_listed_again_leaves_the_rest_right():
    """With weights: the attention, and the weights of all other pages."""
    rc = ctx(16, 4)
    st = Step(54, 16, 4, 128, "bf16", 3, np.full(12, 192), (50, 200), False)
    st.rt[5, 0] = st.rt[2, 0]
    st.rt[9, 1] = st.rt[9, 0]
    again = {int(st.rt[2, 0]), int(st.rt[9, 0])}
    o, w, kp, vp = st.call(rc)
    ref, got = st.oracle(kp, vp)
    ob, rel = st.bounds(kp, vp, ref, got, torch.float32, U["bf16"])
    assert (np.abs(f64(o) - ref) <= ob).all()
    w, listed = f64(w), np.zeros(st.w.shape[0], bool)
    for it in range(12):
        pg, sl = st.rows(it)
        prior = f64(st.w)[pg, sl]
        prior[-1] = 0.0
        own = ~np.isin(pg, list(again))
        # as in Step.check: the probability's relative error, one fp32 rounding for each of the additions
        bound = rel[it] * got[it] + 10 * U["f32"] * (prior + got[it]) + 2.0 ** -120
        assert (np.abs(w[pg, sl] - prior - got[it]) <= bound)[own].all()
        listed[pg] = True
    assert (w[~listed] == -7.0).all() and rc.poll_status() == 0


@pytest.mark.parametrize("q8,spread", [(True, 1.0), (True, 4.0), (False, 1.0)])
def test_a_long_cache(q8, spread):
    """An item of 150 thousand rows: flat scores, and scores of which a few rows have nearly all."""
    rc = ctx(8, 1)
    st = Step(52, 8, 1, 128, "bf16", 1, (150_000, 150_000), (33, 33), q8, pos=0, spread=spread)
    st.check(rc, U["bf16"])


def test_more_pages_than_a_routes_table_holds():
    """The pages behind the table's end are packed, as the copying compaction fills them, and reported."""
    g, d = 1, 128
    rc = ctx(2, g)
    kc = wl.normal(3, (g, 300, d), torch.bfloat16)
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    k8, v8, ks, vs, table = z(6, PT, d, t=torch.uint8), z(6, PT, d, t=torch.uint8), z(6, t=torch.float32), z(6, t=torch.float32), z(1, 2)
    rc.compact_routes_q8(dev(kc), dev(kc), torch.ones(300, dtype=torch.uint8, device="cuda"), i32(0, 1), i32(0), i32(300), torch.ones((g, 1), dtype=torch.uint8, device="cuda"),
                         z(2), z(300), k8, v8, ks, vs, table, i32(5, 4, 3, 2, 1, 0))
    assert rc.poll_status() == 4 and table.tolist() == [[5, 4]] and (ks[1:] > 0).all() and ks[0] == 0


@pytest.mark.parametrize("q8", [True, False], ids=["q8", "same"])
def test_pages_past_two_to_the_31_elements(q8):
    """The item's pages lie at the far end of pools of more than 2^31 elements."""
    rc = ctx(8, 1)
    st = Step(51, 8, 1, 128, "bf16", 2, (150, 250), (100, 200), q8)
    near, nw, kp, vp = st.call(rc)
    shift = 290_000
    far = shift + st.kp.shape[0]
    big = [torch.empty((far, PT, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for x, y in zip(big, (st.kp, st.vp)):
        x[shift:] = dev(y)
    w_in, w_out = torch.zeros((far, PT), device="cuda"), torch.full((far, PT), -7.0, device="cuda")
    w_in[shift:] = dev(st.w)
    ht = dev(np.where(st.ht >= 0, st.ht + shift, -1).astype(np.int32))
    new = dict(k_new=dev(st.kn), v_new=dev(st.vn), out_dtype=torch.float32)
    if q8:
        k8, v8 = (torch.empty((far, PT, 128), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
        ks, vs = torch.empty(far, device="cuda"), torch.empty(far, device="cuda")
        n8 = st.k8.shape[0]
        for x, y in ((k8, st.k8), (v8, st.v8)):
            x.view(torch.uint8)[far - n8:] = dev(y.view(torch.uint8))
        ks[far - n8:], vs[far - n8:] = dev(st.ks), dev(st.vs)
        rt = dev(np.where(st.rt >= 0, st.rt + far - n8, -1).astype(np.int32))
        o = rc.attend_decode_q8(dev(st.q), dev(st.pos), k8, v8, ks, vs, rt, dev(st.res), *big, ht, dev(st.hist), weight_in=w_in, weight_out=w_out, **new)
    else:
        rt = dev(np.where(st.rt >= 0, st.rt + shift, -1).astype(np.int32))
        o = rc.attend_decode_weighted(dev(st.q), dev(st.pos), *big, rt, dev(st.res), ht, dev(st.hist), w_out, weight_in=w_in, **new)
    assert torch.equal(o, near) and torch.equal(w_out[shift:], nw) and (w_out[:shift] == -7).all()
    assert torch.equal(big[0][shift:].view(torch.int16), kp.view(torch.int16)) and rc.poll_status() == 0
    if not q8:                                                  # and eviction from there to the pool's start
        z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        nt, nl, kept = z(2, 1), z(2), z(2, 64)
        rc.evict_rows(*big, w_out, ht, dev(st.hist), 64, 9, dev(np.array([7, 3], np.int32)), nt, nl, kept)
        for it, pg in ((0, 7), (1, 3)):
            p, s = orc.rows_of(st.ht[it], int(st.hist[it]), PT)
            keeps = orc.keep_rows([float(x) for x in f64(nw)[p, s]], 64, 9)
            assert np.array_equal(kept[it].cpu().numpy(), keeps)
            assert torch.equal(big[1][pg], vp[torch.from_numpy(p[keeps]).cuda().long(), torch.from_numpy(s[keeps]).cuda().long()])
        assert rc.poll_status() == 0


def test_packing_from_a_cache_past_two_to_the_31_elements():
    g, d, pool = 2, 128, 9_000_000
    rc = ctx(4, g)
    kc, vc = (torch.zeros((g, pool, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows = wl.normal(9, (g, 100, d), torch.bfloat16)
    kc[:, pool - 100:], vc[:, pool - 100:] = dev(rows), -dev(rows)
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device="cuda")
    k8, v8, ks, vs = z(4, PT, d, t=torch.uint8), z(4, PT, d, t=torch.uint8), z(4, t=torch.float32), z(4, t=torch.float32)
    table, idx, i32 = z(g, 2), z(200), lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    rc.compact_routes_q8(kc, vc, torch.ones(pool, dtype=torch.uint8, device="cuda"), i32(0, 1), i32(pool - 100), i32(100), torch.ones((g, 1), dtype=torch.uint8, device="cuda"),
                         z(g + 1), idx, k8, v8, ks, vs, table, i32(2, 0, 3, 1))
    for k in range(g):
        for p, pg in enumerate(table[k].tolist()):
            want, s = orc.pack_page(f64(rows)[k, p * PT:(p + 1) * PT])
            assert ks[pg] == s and np.array_equal(f64(k8.view(torch.float8_e4m3fn).float())[pg, :len(want)], want)
            assert np.array_equal(f64(v8.view(torch.float8_e4m3fn).float())[pg, :len(want)], -want)
    assert idx[0] == pool - 100 and rc.poll_status() == 0


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("q8", [True, False], ids=["q8", "same"])
def test_what_the_device_reports(dtype, d, q8):
    rc = ctx(8, 2, d, dtype)
    fresh = lambda: Step(61, 8, 2, d, dtype, 3, (100, 200), (70, 100), q8)
    want = fresh().call(rc)[0]
    assert rc.poll_status() == 0
    for breaks, code, item in ((lambda s: s.rt.__setitem__((3, 1), 1 << 25), 4, 3), (lambda s: s.rt.__setitem__((2, 0), -1), 4, 2), (lambda s: s.ht.__setitem__((0, 1), -7), 4, 0),
                               (lambda s: s.hist.__setitem__(5, 0), 4, 5), (lambda s: s.res.__setitem__(1, 64 * s.rt.shape[1] + 1), 4, 1),
                               (lambda s: s.hist.__setitem__(4, 64 * s.ht.shape[1] + 9), 4, 4), (lambda s: s.res.__setitem__(4, -5), 0, 4),
                               (lambda s: s.pos.__setitem__(1, 1 << 20), 6, (2, 3)), (lambda s: s.pos.__setitem__(2, -1), 6, (4, 5))):
        s = fresh()
        breaks(s)
        o = s.call(rc)[0]
        assert rc.poll_status() == code and rc.poll_status() == 0
        for it in range(6):                                    # the other items are not touched by it
            if it != item and (not isinstance(item, tuple) or it not in item):
                assert torch.allclose(o[it // 2, it % 2 * 4:it % 2 * 4 + 4], want[it // 2, it % 2 * 4:it % 2 * 4 + 4], rtol=0, atol=2.0 ** -7 * 6)


def test_an_item_without_rows_gives_zeros():
    for dtype, d in (("bf16", 128), ("f32", 64)):
        for q8 in (True, False):
            rc = ctx(8, 2, d, dtype)
            s = Step(62, 8, 2, d, dtype, 2, (0, 0), (3, 9), q8)
            s.hist[1] = 0
            o, w, _, _ = s.call(rc, append=False)
            assert rc.poll_status() == 4 and (o[0, 4:] == 0).all() and torch.isfinite(o).all()


def test_refusals_of_the_decode_calls():
    rc = ctx(8, 2)
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device="cuda")
    bf, f8, f4 = torch.bfloat16, torch.float8_e4m3fn, torch.float32
    a = dict(q=z(3, 8, 128, t=bf), q_pos=z(3), k_pages8=z(4, 64, 128, t=f8), v_pages8=z(4, 64, 128, t=f8), k_scale=z(4, t=f4), v_scale=z(4, t=f4), res_page_table=z(6, 2),
             res_len=z(6), k_pages=z(9, 64, 128, t=bf), v_pages=z(9, 64, 128, t=bf), hist_page_table=z(6, 3), hist_len=torch.ones(6, dtype=torch.int32, device="cuda"))
    rc.attend_decode_q8(**a)
    bad = dict(q=[z(3, 8, 128, t=f4), z(3, 4, 128, t=bf), z(3, 8, 64, t=bf), z(2, 8, 128, t=bf)], q_pos=[z(4), z(3, t=torch.int64)], k_pages8=[z(4, 64, 128, t=bf), z(5, 64, 128, t=f8), z(4, 32, 128, t=f8)],
               k_scale=[z(3, t=f4), z(4, t=bf)], v_scale=[z(5, t=f4)], res_page_table=[z(5, 2), z(12)], res_len=[z(5)], k_pages=[z(9, 64, 128, t=f4), z(8, 64, 128, t=bf), z(9, 16, 128, t=bf)],
               hist_page_table=[z(7, 3)], hist_len=[z(7)], k_new=[z(3, 2, 128, t=bf)], weight_out=[z(9, 63, t=f4), z(9, 64, t=bf)], out=[z(3, 8, 127, t=bf), z(3, 8, 128, t=torch.float16)],
               out_dtype=[torch.float16])
    for name, values in bad.items():
        for x in values:
            with pytest.raises((ValueError, TypeError)):
                rc.attend_decode_q8(**{**a, name: x})
    with pytest.raises(ValueError):
        rc.attend_decode_q8(**a, k_new=z(3, 2, 128, t=bf), v_new=z(3, 1, 128, t=bf))
    with pytest.raises(ReCacheError, match="weight_in without weight_out"):
        rc.attend_decode_q8(**a, weight_in=z(9, 64, t=f4))
    with pytest.raises(ReCacheError, match="workspace too small"):
        rc.attend_decode_q8(**a, workspace=z(64, t=torch.uint8))
    with pytest.raises(ReCacheError, match="null 8-bit pages"):
        rc.attend_decode_q8(**{**a, "k_pages8": z(0, 64, 128, t=f8), "v_pages8": z(0, 64, 128, t=f8), "k_scale": z(0, t=f4), "v_scale": z(0, t=f4)})
    with pytest.raises(AssertionError):
        rc.attend_decode_q8(**{**a, "q": a["q"].cpu()})
    # no resource part at all, and no sequence
    rc.attend_decode_q8(**{**a, "k_pages8": z(0, 64, 128, t=f8), "v_pages8": z(0, 64, 128, t=f8), "k_scale": z(0, t=f4), "v_scale": z(0, t=f4), "res_page_table": z(6, 0)})
    rc.attend_decode_q8(**{**a, "q": z(0, 8, 128, t=bf), "q_pos": z(0), "res_page_table": z(0, 2), "res_len": z(0), "hist_page_table": z(0, 3), "hist_len": z(0)})
    for k in ("k_pages8", "v_pages8", "k_scale", "v_scale"):
        del a[k]
    rc.attend_decode_weighted(**a, weight_out=z(9, 64, t=f4))
    for x in (z(9, 63, t=f4), z(9, 64, t=bf)):
        with pytest.raises((ValueError, TypeError)):
            rc.attend_decode_weighted(**a, weight_out=x)
    with pytest.raises(ReCacheError, match="null weight_out"):
        rc.attend_decode_weighted(**a, weight_out=None)
    wide = dict(q=z(16, 8, 128, t=bf), q_pos=z(16), res_page_table=torch.empty((32, (1 << 25) - 2), dtype=torch.int32, device="cuda"), res_len=z(32), hist_page_table=z(32, 3),
                hist_len=torch.ones(32, dtype=torch.int32, device="cuda"))
    with pytest.raises(ReCacheError, match="2\\^30 entries"):
        rc.attend_decode_weighted(**{**a, **wide}, weight_out=z(9, 64, t=f4))
    ws = torch.empty(rc.decode_weighted_workspace_bytes(3, 9) - 256, dtype=torch.uint8, device="cuda")
    with pytest.raises(ReCacheError, match="workspace too small"):
        rc.attend_decode_weighted(**a, weight_out=z(9, 64, t=f4), workspace=ws)
    torch.cuda.synchronize()
    assert rc.poll_status() == 0


@pytest.mark.parametrize("seed", range(12))
def test_drawn_shapes(seed):
    rng = np.random.default_rng([seed, 77])
    dtype = "f32" if seed % 4 == 3 else "bf16"
    d = 128 if seed % 3 else int(rng.choice([64, 128]))
    g = int(rng.choice([1, 2, 3, 8]))
    s = int(rng.integers(1, 9))
    pt = 64 if seed % 5 else int(rng.choice([16, 32, 64, 80]))
    rc = ctx(g * s, g, d, dtype, pt)
    lo, hi = sorted(int(x) for x in np.exp(rng.uniform(0, 6.5, 2)))
    h0, h1 = sorted(max(1, int(x)) for x in np.exp(rng.uniform(0, 6, 2)))
    st = Step(200 + seed, g * s, g, d, dtype, int(rng.integers(1, 12)), (lo - 1, hi), (h0, h1), bool(seed & 1), pt)
    st.check(rc, U["bf16"] if dtype == "bf16" else 0.0, append=bool(rng.integers(2)), w_in=["prior", "none"][int(rng.integers(2))])


@pytest.mark.parametrize("dtype,d,pt", [("bf16", 128, 64), ("bf16", 64, 16), ("f32", 64, 64)])
def test_tables_for_more_rows_than_are_numbered_are_refused(dtype, d, pt):
    """The rows of both parts of an item are numbered together."""
    rc = ctx(2, 1, d, dtype, pt)
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device="cuda")
    st, most = rc.torch_dtype, 2 ** 30 // pt
    wide = torch.full((1, most), -1, dtype=torch.int32, device="cuda")
    a = dict(q=z(1, 2, d, t=st), q_pos=z(1), k_pages=z(3, pt, d, t=st), v_pages=z(3, pt, d, t=st), res_len=z(1), hist_len=torch.ones(1, dtype=torch.int32, device="cuda"))
    q8 = dict(k_pages8=z(2, pt, d, t=torch.float8_e4m3fn), v_pages8=z(2, pt, d, t=torch.float8_e4m3fn), k_scale=z(2, t=torch.float32), v_scale=z(2, t=torch.float32))
    for res, hist in ((wide, z(1, 1)), (z(1, 1), wide), (wide[:, :most // 2 + 1], wide[:, :most // 2])):
        with pytest.raises(ReCacheError, match="2\\^30 rows"):
            rc.attend_decode_weighted(**a, res_page_table=res, hist_page_table=hist, weight_out=z(3, pt, t=torch.float32))
        with pytest.raises(ReCacheError, match="2\\^30 rows"):
            rc.attend_decode_q8(**a, **q8, res_page_table=res, hist_page_table=hist)
    rc.attend_decode_weighted(**a, res_page_table=wide[:, :most - 1], hist_page_table=z(1, 1), weight_out=z(3, pt, t=torch.float32))
    rc.attend_decode_q8(**a, **q8, res_page_table=wide[:, :most - 1], hist_page_table=z(1, 1))
    assert rc.poll_status() == 0
