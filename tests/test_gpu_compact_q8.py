"""Compaction into 8-bit pages: values, scales, indices, page tables and status codes, bit for bit against the oracle."""
import numpy as np
import pytest
import torch

from oracle import small_cache as orc
from oracle import recache_oracle as base
from paper_2608_19662_b200 import ReCache, workloads as wl

from pipeline import dev, f64

pytestmark = pytest.mark.gpu


def run(rc, kc, vc, keep, lists, slot, length, vis, capacity=None, pages=None, max_pages=None, free=None, pt=64):
    """lists: resources listed by each request, as indices into slot / length."""
    g, pool, d = kc.shape
    flat = [r for l in lists for r in l]
    res_off = np.cumsum([0] + [len(l) for l in lists]).astype(np.int32)
    res_slot, res_len = np.array([slot[r] for r in flat], np.int32), np.array([length[r] for r in flat], np.int32)
    rows = base.compact_routes(keep, res_off, res_slot, res_len, vis)
    lens = [len(rows[b][k]) for b in range(len(lists)) for k in range(g)]
    need = int(sum(-(-n // pt) for n in lens))
    pages = need + 2 if pages is None else pages
    max_pages = max(1, max(-(-n // pt) for n in lens)) if max_pages is None else max_pages
    free = np.random.default_rng(7).permutation(pages).astype(np.int32) if free is None else np.asarray(free, np.int32)
    capacity = sum(lens) + 3 if capacity is None else capacity
    z = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")
    out = dict(cu=z(len(lens) + 1), idx=z(max(capacity, 1)), len=z(len(lens)), table=z(len(lens), max_pages),
               k8=torch.full((pages, pt, d), 0x55, dtype=torch.uint8, device="cuda"), v8=torch.full((pages, pt, d), 0x55, dtype=torch.uint8, device="cuda"),
               ks=torch.full((pages,), -7.0, device="cuda"), vs=torch.full((pages,), -7.0, device="cuda"))
    rc.compact_routes_q8(dev(kc), dev(vc), dev(keep), dev(res_off), dev(res_slot), dev(res_len), dev(vis), out["cu"], out["idx"], out["k8"], out["v8"], out["ks"],
                         out["vs"], out["table"], dev(free), route_len=out["len"])
    return {k: v.cpu() for k, v in out.items()}, rows, lens, free


def check(out, rows, lens, free, kc, vc, pt=64):
    g = kc.shape[0]
    cu = np.concatenate([[0], np.cumsum(lens)])
    assert np.array_equal(out["cu"].numpy(), cu) and np.array_equal(out["len"].numpy(), lens)
    want = {x: np.full(out[x + "8"].shape, np.nan) for x in "kv"}
    scale = {x: np.full(len(out["ks"]), -7.0) for x in "kv"}
    touched = np.zeros(out["k8"].shape[:2], bool)
    at = 0
    for r, n in enumerate(lens):
        idx = rows[r // g][r % g]
        assert np.array_equal(out["idx"].numpy()[cu[r]:cu[r + 1]], idx)
        n_pages = -(-n // pt)
        assert np.array_equal(out["table"].numpy()[r], np.concatenate([free[at:at + n_pages], np.full(out["table"].shape[1] - n_pages, -1)]))
        for p in range(n_pages):
            part = idx[p * pt:(p + 1) * pt]
            pg = free[at + p]
            touched[pg, :len(part)] = True
            for x, cache in (("k", kc), ("v", vc)):
                want[x][pg, :len(part)], scale[x][pg] = orc.pack_page(f64(cache)[r % g][part])
        at += n_pages
    for x in "kv":
        assert np.array_equal(f64(out[x + "s"]), scale[x])
        raw = out[x + "8"]
        got = f64(raw.view(torch.float8_e4m3fn).float())
        assert np.array_equal(got[touched], want[x][touched], equal_nan=True)
        assert (raw.numpy()[~touched] == 0x55).all()       # slots behind a route's end, pages of no route
    assert (out["idx"].numpy()[cu[-1]:] == -7).all()


@pytest.mark.parametrize("dtype,d,pt", [("bf16", 128, 64), ("bf16", 64, 64), ("f32", 128, 64), ("f32", 64, 16), ("bf16", 128, 48)])
@pytest.mark.parametrize("hq,g", [(8, 2), (8, 8)])
def test_pages_match_the_oracle(dtype, d, pt, hq, g):
    rng = np.random.default_rng([d, pt, g])
    sh = wl.Shape(hq, g, d, 1e4, dtype)
    length = rng.integers(0, 200, 9)
    length[3] = 2200
    slot = np.concatenate([[0], np.cumsum(length)[:-1]])
    pool = int(length.sum())
    kc, vc = (wl.normal(s, (g, pool, d), sh.torch_dtype) * 3 for s in (1, 2))
    keep = (rng.random(pool) < 0.4).astype(np.uint8)
    lists = [[0, 1, 2, 3], [], [4, 3, 8], [5], [6, 7]]
    vis = (rng.random((g, sum(map(len, lists)))) < 0.6).astype(np.uint8)
    vis[0, :] = 1
    rc = ReCache(hq, g, d, 1e4, dtype, max_pos=256, page_tokens=pt)
    got = run(rc, kc, vc, keep, lists, slot, length, vis, pt=pt)
    assert rc.poll_status() == 0
    check(*got, kc, vc, pt=pt)


def test_odd_values():
    """Pages of zeros, of tiny and huge values, with infinities and NaN, and values on every border between two codes."""
    g, d = 1, 128
    kc = torch.zeros((g, 64 * 6, d), dtype=torch.bfloat16)
    kc[0, 64:128] = torch.randn(64, d, generator=torch.Generator().manual_seed(1)) * 1e-38
    kc[0, 128:192] = torch.randn(64, d, generator=torch.Generator().manual_seed(2)) * 1e37
    kc[0, 192:256] = torch.randn(64, d, generator=torch.Generator().manual_seed(3))
    kc[0, 200, 5], kc[0, 201, 6], kc[0, 202, 7] = float("inf"), float("-inf"), float("nan")
    ties = torch.arange(64 * d, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()       # bit patterns 0 ..: all tiny, and
    kc[0, 256:320] = torch.where(torch.isfinite(ties), ties, torch.zeros(())).reshape(64, d).bfloat16()
    kc[0, 320:384] = (torch.arange(64 * d).reshape(64, d) % 3585 / 8.0).bfloat16()                   # 0 .. 448 in eighths
    vc = -kc.flip(1)
    rc = ReCache(2, 1, d, 1e4, "bf16", max_pos=256)
    got = run(rc, kc, vc, np.ones(384, np.uint8), [[0]], [0], [384], np.ones((1, 1), np.uint8))
    assert rc.poll_status() == 0
    check(*got, kc, vc)


def test_many_routes_and_no_rows():
    rng = np.random.default_rng(9)
    g, d, n = 8, 128, 400
    length = rng.integers(0, 30, n)
    slot = np.concatenate([[0], np.cumsum(length)[:-1]])
    pool = int(length.sum())
    kc, vc = (wl.normal(s, (g, pool, d), torch.bfloat16) for s in (3, 4))
    keep = (rng.random(pool) < 0.5).astype(np.uint8)
    lists = [list(rng.integers(0, n, int(rng.integers(0, 6)))) for _ in range(300)]
    vis = (rng.random((g, sum(map(len, lists)))) < 0.3).astype(np.uint8)
    rc = ReCache(32, g, d, 1e4, "bf16", max_pos=256)
    check(*run(rc, kc, vc, keep, lists, slot, length, vis), kc, vc)
    none = run(rc, kc, vc, np.zeros(pool, np.uint8), [[0, 1], [2]], slot, length, np.ones((g, 3), np.uint8))
    check(*none, kc, vc)
    assert rc.poll_status() == 0


def test_what_the_device_reports():
    g, d = 2, 128
    kc, vc = (wl.normal(s, (g, 300, d), torch.bfloat16) for s in (5, 6))
    keep, vis = np.ones(300, np.uint8), np.ones((g, 1), np.uint8)
    rc = ReCache(4, g, d, 1e4, "bf16", max_pos=256)
    out, _, _, free = run(rc, kc, vc, keep, [[0]], [0], [300], vis, pages=10, free=list(range(7)))     # ten pages wanted, seven free
    assert rc.poll_status() == 5
    assert (out["table"][1].numpy() == [5, 6, -1, -1, -1]).all() and (out["ks"][7:] == -7).all() and (out["ks"][:7] > 0).all()
    out, _, _, _ = run(rc, kc, vc, keep, [[0]], [0], [300], vis, capacity=350, pages=10)               # index list too short
    assert rc.poll_status() == 3 and (out["idx"] >= 0).all()
    out, _, _, _ = run(rc, kc, vc, keep, [[0]], [0], [300], vis, pages=10, free=[0, 1, 2, 99, 4, -3, 6, 7, 8, 9])
    assert rc.poll_status() == 4 and out["table"][0, 3] == -1 and out["table"][1, 0] == -1
    assert rc.poll_status() == 0


def test_refusals():
    g, d = 2, 128
    rc = ReCache(4, g, d, 1e4, "bf16", max_pos=256)
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device="cuda")
    a = dict(k_cache=z(g, 8, d, t=torch.bfloat16), v_cache=z(g, 8, d, t=torch.bfloat16), keep=z(8, t=torch.uint8), res_off=z(2), res_slot=z(1), res_len=z(1),
             vis=z(g, 1, t=torch.uint8), route_cu=z(g + 1), route_idx=z(16), k_pages8=z(4, 64, d, t=torch.uint8), v_pages8=z(4, 64, d, t=torch.uint8),
             k_scale=z(4, t=torch.float32), v_scale=z(4, t=torch.float32), page_table=z(g, 2), free_pages=z(4))
    rc.compact_routes_q8(**a)
    bad = [("k_cache", z(g, 8, d, t=torch.float32)), ("v_cache", z(g, 9, d, t=torch.bfloat16)), ("keep", z(7, t=torch.uint8)), ("keep", z(8)),
           ("res_len", z(2)), ("res_off", z(2, t=torch.int64)), ("vis", z(g, 2, t=torch.uint8)), ("route_cu", z(g)), ("k_pages8", z(4, 64, d, t=torch.int8)),
           ("k_pages8", z(4, 32, d, t=torch.uint8)), ("v_pages8", z(5, 64, d, t=torch.uint8)), ("k_scale", z(3, t=torch.float32)),
           ("v_scale", z(4, t=torch.float64)), ("page_table", z(g + 1, 2)), ("page_table", z(g)), ("route_len", z(1)), ("k_cache", z(1, 8, d, t=torch.bfloat16))]
    for name, t in bad:
        with pytest.raises((ValueError, TypeError)):
            rc.compact_routes_q8(**{**a, name: t})
    with pytest.raises(AssertionError):
        rc.compact_routes_q8(**{**a, "keep": a["keep"].cpu()})
    with pytest.raises(RuntimeError, match="workspace too small"):
        rc.compact_routes_q8(**a, workspace=z(16, t=torch.uint8))
    assert rc.poll_status() == 0
