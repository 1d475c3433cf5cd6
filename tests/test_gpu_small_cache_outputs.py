"""Outputs of decode over 8-bit pages and with weights, held as tightly as their rounding allows: over a long cache whose scores are flat, the values
cancel, and a bound made from the largest of them is wider than the output."""
import math

import numpy as np
import pytest
import torch

from oracle import recache_oracle as base
from oracle import small_cache as orc
from paper_2608_19662_b200 import ReCache

from pipeline import f64
from small_cache import U, Step

pytestmark = pytest.mark.gpu


def ctx(hq=32, g=8, d=128, dtype="bf16", pt=64):
    return ReCache(hq, g, d, 1e4, dtype, max_pos=16384, page_tokens=pt)


def hold(st, o, kp, vp, out_dtype=torch.float32, rounded=True):
    """|o|'s error against the sum's own statistics.  Returns (largest error / bound, mean bound, rms of o).

    A probability meets its value rounded: half a step of f16 (8-bit rows) or bf16 relative to itself, up or down alike, so n of them add up to more than
    6 sqrt(sum (step p |v|)^2) once in 3e7 outputs (Hoeffding), and never to more than sum step p |v|.  A score is off by the fp32 sums over the head dimension
    (tensor cores cut sums off where fp32 arithmetic rounds: 2^-23 for each of d + 8 steps) and, where a query element lies next to a border of bf16, by a step of
    it (Step.score_slack's part of that); a probability by twice that, with exponentials good to 2^-20.  Sums over rows: fewer than 512 cut-off steps deep.  f16
    probabilities below 2^-29 of the largest are off by 2^-40 of it: n of them, times the largest value.  rounded: not so in the kernel of the other shapes, whose
    probabilities stay in fp32."""
    sh, g = st.sh, st.sh.n_kv_heads
    s, d = sh.n_q_heads // g, sh.head_dim
    kp, vp = f64(kp), f64(vp)
    qh = base.round_storage(base.rope(f64(st.q), st.pos, sh.rope_theta), sh.dtype)
    o, worst, bounds, power = f64(o), 0.0, [], []
    for it in range(st.batch * g):
        i, kg = divmod(it, g)
        ph, sl = orc.rows_of(st.ht[it], int(st.hist[it]), st.pt)
        pr, sr = orc.rows_of(st.rt[it], int(st.res[it]), st.pt)
        if st.q8:
            kf, vf = (f64(a.float())[pr, sr] * f64(b)[pr][:, None] for a, b in ((st.k8, st.ks), (st.v8, st.vs)))
        else:
            kf, vf = kp[pr, sr], vp[pr, sr]
        k, v = np.concatenate([kf, kp[ph, sl]]), np.concatenate([vf, vp[ph, sl]])
        step = np.concatenate([np.full(len(kf), U["f16"] if st.q8 else U["bf16"]), np.full(len(ph), U["bf16"])])[:, None] * rounded
        q = qh[i, kg * s:(kg + 1) * s]
        sc = k @ q.T / math.sqrt(d)
        p = np.exp(sc - sc.max(0))
        p /= p.sum(0)
        fp = (d + 8) * 2.0 ** -23 * (np.abs(k) @ np.abs(q).T).max(0) / math.sqrt(d)
        kmax, vmax = np.abs(k).max(), np.abs(v).max()
        flips = np.maximum(0.0, st.score_slack(kmax)[i, kg * s:(kg + 1) * s] - (d + 8) * U["f32"] * np.abs(q).sum(1) * kmax / math.sqrt(d))
        rel = np.expm1(2 * (fp + flips)) + 2.0 ** -20 + 2.0 ** -14
        for h in range(s):
            pv = p[:, h:h + 1] * np.abs(v)
            rounding = np.minimum((step * pv).sum(0), 6 * np.sqrt(((step * pv) ** 2).sum(0)))
            ref = p[:, h] @ v
            bound = rounding + rel[h] * pv.sum(0) + len(v) * 2.0 ** -40 * vmax + (U["bf16"] * np.abs(ref) if out_dtype == torch.bfloat16 else 0.0)
            worst = max(worst, float((np.abs(o[i, kg * s + h] - ref) / bound).max()))
            bounds.append(bound.mean())
            power.append(np.sqrt((ref ** 2).mean()))
    return worst, float(np.mean(bounds)), float(np.mean(power))


@pytest.mark.parametrize("n", [1400, 18_000, 150_000])
@pytest.mark.parametrize("q8,spread", [(True, 1.0), (True, 4.0), (False, 1.0), (False, 4.0)])
def test_outputs_over_long_caches(n, q8, spread):
    """The bound is a fraction of the output itself, whose values cancel more the longer a flat cache is."""
    rc = ctx(8, 1)
    st = Step(71, 8, 1, 128, "bf16", 1, (n, n), (33, 33), q8, pos=0, spread=spread)
    o, _, kp, vp = st.call(rc)
    worst, bound, rms = hold(st, o, kp, vp)
    assert bound < rms / 8, (bound, rms)
    assert worst <= 1.0, (worst, bound, rms)
    assert rc.poll_status() == 0


@pytest.mark.parametrize("hq,g", [(8, 8), (4, 2), (9, 3), (32, 8), (10, 2), (7, 1), (16, 2)])
@pytest.mark.parametrize("q8", [True, False], ids=["q8", "same"])
def test_outputs_of_a_ragged_batch(hq, g, q8):
    rc = ctx(hq, g)
    st = Step(72 + hq, hq, g, 128, "bf16", 5, (0, 1500), (1, 900), q8)
    o, _, kp, vp = st.call(rc)
    worst, bound, rms = hold(st, o, kp, vp)
    assert worst <= 1.0, (worst, bound, rms)
    o, _, kp, vp = st.call(rc, out_dtype=torch.bfloat16)
    worst, bound, rms = hold(st, o, kp, vp, torch.bfloat16)
    assert worst <= 1.0, (worst, bound, rms)
    assert rc.poll_status() == 0


@pytest.mark.parametrize("dtype,d,pt", [("bf16", 64, 64), ("bf16", 128, 16), ("bf16", 64, 80), ("f32", 128, 64), ("f32", 64, 32)])
@pytest.mark.parametrize("hq,g", [(8, 8), (10, 2), (8, 1)])
@pytest.mark.parametrize("q8", [True, False], ids=["q8", "same"])
def test_outputs_of_other_shapes(dtype, d, pt, hq, g, q8):
    rc = ctx(hq, g, d, dtype, pt)
    st = Step(90 + hq, hq, g, d, dtype, 3, (0, 1500), (1, 900), q8, pt)
    o, _, kp, vp = st.call(rc)
    worst, bound, rms = hold(st, o, kp, vp, rounded=False)
    assert worst <= 1.0, (worst, bound, rms)
    assert rc.poll_status() == 0
