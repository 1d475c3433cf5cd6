"""Eviction by weight against a sort in plain Python: which rows stay, where they go, and what is left alone."""
import math

import numpy as np
import pytest
import torch

from oracle import small_cache as orc
from paper_2608_19662_b200 import ReCache

from pipeline import dev
from small_cache import tables

pytestmark = pytest.mark.gpu


class Pool:
    def __init__(self, seed, lens, budget, d=128, dtype=torch.bfloat16, pt=64, spare=None, weights=None):
        rng = np.random.default_rng([seed, 3])
        self.lens, self.budget, self.pt = np.asarray(lens, np.int32), budget, pt
        counts = -(-self.lens // pt)
        self.new = -(-budget // pt)
        over = int((self.lens > budget).sum())
        self.table = tables(rng, counts)
        n = int(counts.sum())
        fresh = over * self.new + 3 if spare is None else spare
        self.free = (n + rng.permutation(fresh)).astype(np.int32)
        gen = torch.Generator().manual_seed(seed)
        self.k, self.v = (torch.randn((n + fresh, pt, d), generator=gen).to(dtype) for _ in range(2))
        w = rng.choice([0.0, 0.25, 1.0], (n + fresh, pt)) if weights == "ties" else np.exp(2 * rng.standard_normal((n + fresh, pt)))
        self.w = torch.from_numpy(w.astype(np.float32))
        if weights == "odd":
            flat = self.w.view(-1)
            at = rng.permutation(flat.numel())
            for i, x in enumerate([math.nan, -math.nan, math.inf, -math.inf, -0.0, 0.0, -1.0, 1e-45, 3.4e38]):
                flat[torch.from_numpy(at[i::23].copy())] = x

    def weights_of(self, it):
        pg, sl = orc.rows_of(self.table[it], int(self.lens[it]), self.pt)
        return [float(x) for x in self.w.numpy()[pg, sl]]

    def call(self, rc, recent, wide=0, free=None):
        z = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")
        out = dict(k=dev(self.k), v=dev(self.v), w=dev(self.w), table=z(len(self.lens), self.new + wide), len=z(len(self.lens)), kept=z(len(self.lens), self.budget))
        rc.evict_rows(out["k"], out["v"], out["w"], dev(self.table), dev(self.lens), self.budget, recent, dev(self.free if free is None else free), out["table"], out["len"],
                      out["kept"])
        return {k: v.cpu() for k, v in out.items()}

    def check(self, out, recent):
        k, v, w = self.k.clone(), self.v.clone(), self.w.clone()
        evicting = 0
        for it, n in enumerate(self.lens):
            keep = orc.keep_rows(self.weights_of(it), self.budget, recent)
            assert out["len"][it] == len(keep)
            kept = out["kept"][it].numpy()
            assert np.array_equal(kept[:len(keep)], keep), (it, n)
            assert (kept[len(keep):] == -7).all()
            n_pages = -(-len(keep) // self.pt)
            if n > self.budget:
                pages = self.free[evicting * self.new:(evicting + 1) * self.new]
                evicting += 1
                src, dst = orc.rows_of(self.table[it], int(n), self.pt), orc.rows_of(pages, len(keep), self.pt)
                for x in (k, v, w):
                    x[dst[0], dst[1]] = x[src[0][keep], src[1][keep]]
            else:
                pages = self.table[it][:n_pages]
            assert np.array_equal(out["table"][it, :n_pages].numpy(), pages)
            assert (out["table"][it, n_pages:] == -7).all()
        for name, x in (("k", k), ("v", v), ("w", w)):
            raw = torch.int16 if x.dtype == torch.bfloat16 else torch.int32
            assert torch.equal(out[name].view(raw), x.view(raw)), name


CASES = [
    # lengths, budget, recent
    ([1, 2, 3, 0], 1, 0), ([1, 2, 3, 0], 1, 1), ([65, 64, 63], 64, 64), ([65, 64, 200], 64, 0), ([1088], 1024, 64), ([130, 4000, 5, 2048, 2049], 2047, 100),
    ([4097, 8193, 4095], 4096, 4095), ([70000, 3], 5000, 333), ([300] * 40, 299, 7), (list(range(50, 550)), 200, 10),
]


@pytest.mark.parametrize("weights", ["spread", "ties", "odd"])
@pytest.mark.parametrize("lens,budget,recent", CASES, ids=lambda x: str(x)[:24].replace(" ", ""))
def test_matches_a_sort(lens, budget, recent, weights):
    rc = ReCache(8, 2, 128, 1e4, "bf16", max_pos=256)
    p = Pool(len(lens) + budget, lens, budget, weights=weights)
    p.check(p.call(rc, recent, wide=2), recent)
    assert rc.poll_status() == 0


@pytest.mark.parametrize("recent", [0, 700])
def test_more_rows_than_a_block_keeps_keys_of(recent):
    """Many items, so a block each, one of them longer than its shared memory holds keys."""
    rc = ReCache(2, 1, 64, 1e4, "bf16", max_pos=256)
    lens = [3, 70, 21700] + [int(x) for x in np.random.default_rng(4).integers(0, 130, 320)] + [20481]
    p = Pool(9, lens, 1000, d=64, weights="odd")
    p.check(p.call(rc, recent), recent)
    assert rc.poll_status() == 0


@pytest.mark.parametrize("dtype,d,pt", [("f32", 64, 64), ("f32", 128, 16), ("bf16", 64, 48), ("bf16", 64, 50)])
def test_other_shapes(dtype, d, pt):
    rc = ReCache(8, 2, d, 1e4, dtype, max_pos=256, page_tokens=pt)
    p = Pool(5, [700, 20, 333, 500], 300, d=d, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, pt=pt)
    p.check(p.call(rc, 31), 31)
    assert rc.poll_status() == 0


def test_weights_that_are_not_16_byte_aligned():
    rc = ReCache(8, 2, 128, 1e4, "bf16", max_pos=256)
    p = Pool(6, [700, 20, 333, 5000], 300)
    whole = torch.empty(p.w.numel() + 1, device="cuda")
    whole[1:] = dev(p.w).reshape(-1)
    z = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")
    out = dict(k=dev(p.k), v=dev(p.v), w=whole[1:].view(p.w.shape), table=z(4, p.new), len=z(4), kept=z(4, 300))
    rc.evict_rows(out["k"], out["v"], out["w"], dev(p.table), dev(p.lens), 300, 50, dev(p.free), out["table"], out["len"], out["kept"])
    p.check({k: v.cpu() for k, v in out.items()}, 50)
    assert rc.poll_status() == 0


def test_what_the_device_reports():
    rc = ReCache(8, 2, 128, 1e4, "bf16", max_pos=256)
    p = Pool(5, [700, 20, 333, 500], 300, spare=40)
    full = p.call(rc, 31)
    assert rc.poll_status() == 0
    out = p.call(rc, 31, free=p.free[:7])                       # three items want five pages each
    assert rc.poll_status() == 5
    assert (out["table"][0].numpy() == p.free[:5]).all() and (out["table"][2].numpy() == [p.free[5], p.free[6], -1, -1, -1]).all() and (out["table"][3] == -1).all()
    assert torch.equal(out["kept"], full["kept"]) and torch.equal(out["len"], full["len"])
    for pg in p.free[7:]:
        assert torch.equal(out["k"][pg], p.k[pg])
    bad = p.free.copy()
    bad[1], bad[6] = -5, 1 << 20
    out = p.call(rc, 31, free=bad)
    assert rc.poll_status() == 4 and out["table"][0, 1] == -1 and out["table"][2, 1] == -1
    p.table[2, 1] = 1 << 20                                     # a page that is none: its 64 rows are the first to go
    out = p.call(rc, 31)
    assert rc.poll_status() == 4
    p.table[2, 1] = p.table[2, 0]
    want = orc.keep_rows([math.nan if 64 <= i < 128 else x for i, x in enumerate(p.weights_of(2))], 300, 31)
    assert np.array_equal(out["kept"][2].numpy(), want)
    p.lens[1] = 20 + 64 * p.table.shape[1]                      # longer than its table: read as what the table holds
    p.table[1] = p.table[0, 0]
    out = p.call(rc, 31)
    assert rc.poll_status() == 4 and out["len"][1] == 300


def test_refusals():
    rc = ReCache(4, 2, 128, 1e4, "bf16", max_pos=256)
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device="cuda")
    a = dict(k_pages=z(4, 64, 128, t=torch.bfloat16), v_pages=z(4, 64, 128, t=torch.bfloat16), weight=z(4, 64, t=torch.float32), page_table=z(2, 2), row_len=z(2),
             budget=70, n_recent=3, free_pages=z(0), new_table=z(2, 2), new_len=z(2), kept=z(2, 70))
    rc.evict_rows(**a)
    for name, x in [("k_pages", z(4, 64, 128, t=torch.float32)), ("v_pages", z(5, 64, 128, t=torch.bfloat16)), ("k_pages", z(4, 32, 128, t=torch.bfloat16)),
                    ("weight", z(4, 64)), ("weight", z(3, 64, t=torch.float32)), ("page_table", z(3, 2)), ("row_len", z(2, t=torch.int64)), ("budget", 0), ("budget", -1),
                    ("n_recent", 71), ("n_recent", -1), ("new_len", z(1)), ("kept", z(2, 69)), ("new_table", z(1, 2))]:
        with pytest.raises((ValueError, TypeError)):
            rc.evict_rows(**{**a, name: x})
    with pytest.raises(RuntimeError, match="too few pages"):
        rc.evict_rows(**{**a, "new_table": z(2, 1)})
    with pytest.raises(RuntimeError, match="must not be"):
        rc.evict_rows(**{**a, "new_table": a["page_table"]})
    with pytest.raises(RuntimeError, match="must not be"):
        rc.evict_rows(**{**a, "new_len": a["row_len"]})
    rc.evict_rows(**{**a, "page_table": z(0, 2), "row_len": z(0), "new_table": z(0, 2), "new_len": z(0), "kept": z(0, 70)})
    assert rc.poll_status() == 0


def test_tables_for_more_rows_than_are_numbered_are_refused():
    rc = ReCache(4, 2, 128, 1e4, "bf16", max_pos=256, page_tokens=8)
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device="cuda")
    a = dict(k_pages=z(4, 8, 128, t=torch.bfloat16), v_pages=z(4, 8, 128, t=torch.bfloat16), weight=z(4, 8, t=torch.float32), row_len=z(1), budget=70, n_recent=3,
             free_pages=z(0), new_len=z(1), kept=z(1, 70))
    most = 2 ** 30 // 8
    wide = torch.empty((1, 2 ** 31 // 8 - 1), dtype=torch.int32, device="cuda")
    for tables in (dict(page_table=wide, new_table=z(1, 9)), dict(page_table=wide[:, :most + 1], new_table=z(1, 9)), dict(page_table=z(1, 2), new_table=wide[:, :most + 1])):
        with pytest.raises(RuntimeError, match="2\\^30 rows"):
            rc.evict_rows(**a, **tables)
    rc.evict_rows(**a, page_table=wide[:, :most], new_table=wide[:, most:most + 9])
    assert rc.poll_status() == 0
