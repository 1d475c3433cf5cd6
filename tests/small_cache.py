"""Helpers for the tests of 8-bit pages, attention weights and eviction: inputs with poisoned slots, and what the
results may be off by."""
import numpy as np
import torch

from oracle import recache_oracle as base
from oracle import small_cache as orc
from paper_2608_19662_b200 import workloads as wl

from pipeline import dev, f64

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}     # half a step, relative


def tables(rng, counts, first=0, width=None):
    """Shuffled pages first .. first + sum - 1, one run of each item in its row; -1 behind."""
    ids = first + rng.permutation(int(counts.sum())).astype(np.int32)
    out = np.full((len(counts), max(1, int(counts.max())) if width is None else width), -1, np.int32)
    at = 0
    for it, n in enumerate(counts):
        out[it, :n] = ids[at:at + n]
        at += int(n)
    return out


class Step:
    """Inputs of one decode step; slots of no row hold NaN."""

    def __init__(self, seed, hq, g, d, dtype, batch, res, hist, q8, pt=64, pos=None, spread=1.0, scales=None):
        rng = np.random.default_rng([seed, 41])
        self.sh, self.pt, self.q8, self.batch = wl.Shape(hq, g, d, 1e4, dtype), pt, q8, batch
        items = batch * g
        self.res = np.asarray(res, np.int32) if np.ndim(res) and len(np.atleast_1d(res)) == items else rng.integers(res[0], res[1] + 1, items).astype(np.int32)
        self.hist = np.repeat(rng.integers(hist[0], hist[1] + 1, batch), g).astype(np.int32)
        rp, hp = -(-self.res // pt), -(-self.hist // pt)
        n8 = int(rp.sum())
        self.rt = tables(rng, rp)
        self.ht = tables(rng, hp, 0 if q8 else n8)
        n = int(hp.sum()) + (0 if q8 else n8)
        td = self.sh.torch_dtype
        self.q = wl.normal(seed * 7 + 1, (batch, hq, d), td) * spread
        self.kn, self.vn = (wl.normal(seed * 7 + i, (batch, g, d), td) for i in (2, 3))
        self.kp, self.vp = (wl.normal(seed * 7 + i, (n, pt, d), td) for i in (4, 5))
        self.k8 = self.v8 = self.ks = self.vs = None
        if q8:
            pages = [wl.normal(seed * 7 + i, (max(n8, 1), pt, d), torch.float32) for i in (6, 7)]
            ks = np.array([orc.page_scale(f64(p)) for p in pages[0]])
            vs = np.array([orc.page_scale(f64(p)) for p in pages[1]])
            self.k8, self.v8 = (torch.from_numpy(np.stack([orc.round_e4m3(f64(p) / s) for p, s in zip(x, sc)])).to(torch.float8_e4m3fn)
                                for x, sc in zip(pages, (ks, vs)))
            if scales is not None:                         # scales of no power of two: the call takes any
                ks, vs = ks * rng.uniform(*scales, ks.shape), vs * rng.uniform(*scales, vs.shape)
            self.ks, self.vs = (torch.from_numpy(s.astype(np.float32)) for s in (ks, vs))
        self.poison()
        self.w = torch.from_numpy(rng.uniform(0, 3, (n, pt)).astype(np.float32))
        self.pos = (rng.integers(0, 9000, batch).astype(np.int32) if pos is None else np.full(batch, pos, np.int32))

    def poison(self):
        for table, lens, pools in ((self.rt, self.res, (self.k8, self.v8) if self.q8 else (self.kp, self.vp)), (self.ht, self.hist, (self.kp, self.vp))):
            for it, n in enumerate(lens):
                if n % self.pt:
                    for p in pools:
                        if p.dtype == torch.float8_e4m3fn:
                            p.view(torch.uint8)[table[it, n // self.pt], n % self.pt:] = 0x7F
                        else:
                            p[table[it, n // self.pt], n % self.pt:] = float("nan")

    def rows(self, it):
        """Pool rows (page, slot) of the item's rows that have a weight: resource rows if they lie in the pool, history rows."""
        r = [orc.rows_of(self.ht[it], int(self.hist[it]), self.pt)]
        if not self.q8:
            r.insert(0, orc.rows_of(self.rt[it], int(self.res[it]), self.pt))
        return np.concatenate([x[0] for x in r]), np.concatenate([x[1] for x in r])

    def call(self, rc, out_dtype=torch.float32, append=True, weights=True, w_in="prior", pools=None, **more):
        """(o, weight_out or None, k_pages, v_pages after the call)."""
        kp, vp = pools if pools is not None else (dev(self.kp), dev(self.vp))
        new = dict(k_new=dev(self.kn), v_new=dev(self.vn)) if append else {}
        wo = torch.full(self.w.shape, -7.0, device="cuda") if weights else None
        wi = {"prior": dev(self.w), "none": None}[w_in] if weights else None
        if self.q8:
            o = rc.attend_decode_q8(dev(self.q), dev(self.pos), dev(self.k8), dev(self.v8), dev(self.ks), dev(self.vs), dev(self.rt), dev(self.res), kp, vp,
                                    dev(self.ht), dev(self.hist), weight_in=wi, weight_out=wo, out_dtype=out_dtype, **new, **more)
        else:
            o = rc.attend_decode_weighted(dev(self.q), dev(self.pos), kp, vp, dev(self.rt), dev(self.res), dev(self.ht), dev(self.hist), wo,
                                          weight_in=wi, out_dtype=out_dtype, **new, **more)
        return o, wo, kp, vp

    def oracle(self, kp, vp):
        """(o, probabilities per item) over the pages as the call left them."""
        first = None if not self.q8 else tuple(f64(x.float()) for x in (self.k8, self.v8, self.ks, self.vs))
        return orc.attend_decode(f64(self.q), self.pos, first, f64(kp), f64(vp), self.rt, self.res, self.ht, self.hist, self.sh.rope_theta, self.pt,
                                 storage=self.sh.dtype)

    def score_slack(self, kmax):
        """How far a score may be off, per (sequence, query head): the fp32 product sums, and one step of the storage type for every rotated
        query element that lies so near to a border that fp32 and fp64 rotations may round it differently.  kmax: largest |key element|."""
        d = self.sh.head_dim
        x = f64(self.q)
        y = base.rope(x, self.pos, self.sh.rope_theta)
        half = d // 2
        pair = np.abs(x[..., :half]) + np.abs(x[..., half:])
        err = 4 * U["f32"] * np.concatenate([pair, pair], -1)          # two products, one sum, the table's own rounding
        bits = 24 if self.sh.dtype == "f32" else 8
        _, e = np.frexp(np.where(y == 0, 1.0, y))
        step = np.ldexp(1.0, e - bits)
        frac = np.abs(y) / step
        near = np.abs(frac - np.floor(frac) - 0.5) * step <= err
        moved = np.where(near, step, 0.0) if self.sh.dtype == "bf16" else err + step
        flips = moved.sum(-1) * kmax / np.sqrt(d)
        size = np.abs(base.round_storage(y, self.sh.dtype)).sum(-1) * kmax / np.sqrt(d)
        return flips + (d + 8) * U["f32"] * size                        # d products summed, scaled by constants and a page's scale

    def bounds(self, kp, vp, ref, got, out_dtype, p_step):
        """(bound on |o|'s error [B][Hq][1 or d], relative bound on a probability summed over heads, per item).  p_step: half a step of the type in
        which probabilities meet the values."""
        live = lambda pool, table, lens: [f64(pool)[orc.rows_of(table[it], int(n), self.pt)] for it, n in enumerate(lens) if n]
        if self.q8:
            k8, v8 = (f64(a.float()) * f64(b)[:, None, None] for a, b in ((self.k8, self.ks), (self.v8, self.vs)))
            ks, vs = live(k8, self.rt, self.res), live(v8, self.rt, self.res)
        else:
            ks, vs = live(kp, self.rt, self.res), live(vp, self.rt, self.res)
        ks, vs = ks + live(kp, self.ht, self.hist), vs + live(vp, self.ht, self.hist)
        kmax, vmax = max(np.abs(x).max() for x in ks), max(np.abs(x).max() for x in vs)
        slack = self.score_slack(kmax)                                  # [B][Hq]
        rel = np.expm1(2 * slack) + 2.0 ** -20                          # of a probability: its own score and the sum's; exponentials good to 2^-21
        o_bound = (rel + p_step)[..., None] * vmax + (U["bf16"] * np.abs(ref) if out_dtype == torch.bfloat16 else 0.0) + 1e-6 * vmax
        g = self.sh.n_kv_heads
        return o_bound, rel.reshape(self.batch * g, -1).max(axis=1)

    def check(self, rc, p_step, out_dtype=torch.float32, append=True, weights=True, w_in="prior"):
        o, wo, kp, vp = self.call(rc, out_dtype, append, weights, w_in)
        last = (self.hist - 1)
        page, slot = self.ht[np.arange(len(last)), last // self.pt], last % self.pt
        want_k, want_v = f64(self.kp), f64(self.vp)
        if append:
            base.append_decode_kv(want_k, want_v, self.ht, self.hist, f64(self.kn), f64(self.vn), self.pos, self.sh.rope_theta, self.pt, storage=self.sh.dtype)
        gk, gv = f64(kp), f64(vp)
        assert np.array_equal(gv, want_v, equal_nan=True)
        new = np.zeros(gk.shape[:2], bool)
        new[page, slot] = append
        assert np.array_equal(gk[~new], want_k[~new], equal_nan=True)
        step = 2.0 ** -7 if self.sh.dtype == "bf16" else 2.0 ** -22     # neighbours of the storage type; fp32: rounding of the rotation itself
        assert (np.abs(gk[new] - want_k[new]) <= step * np.abs(want_k[new]) + 4e-6).all()
        ref, got = self.oracle(kp, vp)
        ob, rel = self.bounds(kp, vp, ref, got, out_dtype, p_step)
        err = np.abs(f64(o) - ref)
        assert o.dtype == out_dtype and (err <= ob).all(), (err.max(), ob[err > ob][:3] if ob.shape == err.shape else ob.max(), err[(err > ob)][:3])
        if weights:
            w = f64(wo)
            seen = np.zeros(w.shape, bool)
            for it in range(len(self.res)):
                pg, sl = self.rows(it)
                mine = got[it][-len(pg):] if len(pg) else got[it][:0]
                prior = f64(self.w)[pg, sl] if w_in == "prior" else np.zeros(len(pg))
                if append:
                    prior[-1] = 0.0
                # the probability's relative error, one fp32 rounding for each of the additions; 2^-120: an exponential that is no longer normal
                bound = rel[it] * mine + 10 * U["f32"] * (prior + mine) + 2.0 ** -120
                assert (np.abs(w[pg, sl] - prior - mine) <= bound).all(), (it, np.abs(w[pg, sl] - prior - mine).max(), bound.min())
                seen[pg, sl] = True
            assert (w[~seen] == -7.0).all()
        assert rc.poll_status() == 0
        return o, wo
