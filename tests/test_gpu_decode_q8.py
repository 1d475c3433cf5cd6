"""Decode over 8-bit pages and decode with attention weights against the fp64 oracle: types, head layouts, lengths from one
row on, pages that end inside a tile, poisoned slots, and the appended token."""
import numpy as np
import pytest
import torch

from paper_2608_19662_b200 import ReCache

from small_cache import U, Step

pytestmark = pytest.mark.gpu


def ctx(hq, g, d, dtype, pt=64, max_pos=16384):
    return ReCache(hq, g, d, 1e4, dtype, max_pos=max_pos, page_tokens=pt)


CASES = [
    # hq, g, d, dtype, page tokens, batch, resource rows, history rows
    (8, 8, 128, "bf16", 64, 1, (0, 0), (1, 1)),
    (32, 8, 128, "bf16", 64, 1, (1, 1), (1, 1)),
    (32, 8, 128, "bf16", 64, 1, (700, 760), (700, 700)),
    (16, 8, 128, "bf16", 64, 5, (0, 200), (1, 300)),
    (24, 8, 128, "bf16", 64, 4, (60, 70), (31, 34)),
    (40, 8, 128, "bf16", 64, 3, (127, 129), (63, 66)),
    (64, 8, 128, "bf16", 64, 3, (0, 900), (1, 900)),
    (7, 1, 128, "bf16", 64, 2, (5000, 6000), (95, 97)),
    (4, 1, 128, "bf16", 64, 1, (64 * 150, 64 * 150), (64 * 140, 64 * 140)),
    (12, 2, 128, "bf16", 64, 70, (0, 130), (1, 130)),
    (16, 8, 128, "bf16", 64, 90, (0, 64), (1, 200)),
    (8, 2, 64, "bf16", 64, 3, (0, 300), (1, 200)),
    (4, 2, 128, "bf16", 16, 3, (0, 100), (1, 90)),
    (4, 2, 64, "f32", 64, 3, (0, 300), (1, 200)),
    (8, 1, 128, "f32", 48, 2, (0, 200), (1, 200)),
]


@pytest.mark.parametrize("q8", [True, False], ids=["q8", "same"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_matches_the_oracle_and_appends(case, q8):
    hq, g, d, dtype, pt, batch, res, hist = case
    rc = ctx(hq, g, d, dtype, pt)
    step = Step(hq + d + batch, hq, g, d, dtype, batch, res, hist, q8, pt)
    step.check(rc, U["bf16"] if dtype == "bf16" else 0.0)


@pytest.mark.parametrize("q8", [True, False], ids=["q8", "same"])
def test_bf16_results_no_append_no_prior(q8):
    rc = ctx(32, 8, 128, "bf16")
    step = Step(3, 32, 8, 128, "bf16", 6, (0, 500), (1, 500), q8)
    step.check(rc, U["bf16"], out_dtype=torch.bfloat16, append=False, w_in="none")
    step.check(rc, U["bf16"], weights=not q8)


@pytest.mark.parametrize("scales", [(0.01, 1.9), (1e-12, 1e-9), (50.0, 400.0)])
def test_scales_of_any_size(scales):
    rc = ctx(16, 4, 128, "bf16")
    step = Step(11, 16, 4, 128, "bf16", 3, (100, 700), (1, 100), True, scales=scales)
    step.check(rc, U["bf16"])


@pytest.mark.parametrize("spread", [1e-30, 8.0, 1e4])
@pytest.mark.parametrize("q8", [True, False], ids=["q8", "same"])
def test_queries_of_any_size(q8, spread):
    """Scores that are all alike, that rescale from page to page, and that leave one row with everything."""
    rc = ctx(16, 4, 128, "bf16")
    step = Step(12, 16, 4, 128, "bf16", 3, (100, 700), (1, 100), q8, pos=0, spread=spread)
    if spread < 1e3:
        step.check(rc, U["bf16"])
        return
    o, w, kp, vp = step.call(rc)
    ref, got = step.oracle(kp, vp)
    assert torch.isfinite(o).all() and np.isfinite(np.asarray(w.cpu())).all()
    assert np.median(np.abs(o.double().cpu().numpy() - ref)) < 2.0 ** -8


def test_nan_and_infinite_rows_stay_in_their_item():
    rc = ctx(16, 4, 128, "bf16")
    step = Step(13, 16, 4, 128, "bf16", 3, (100, 300), (70, 100), True)
    clean, wc, _, _ = step.call(rc)
    step.k8.view(torch.uint8)[step.rt[5, 1], 3, 7] = 0x7F
    step.vp[step.ht[6, 0], 2, 9] = float("inf")
    o, w, _, _ = step.call(rc)
    assert torch.isnan(o[1, 4:8]).all()                # item 5: sequence 1, group 1: a NaN score
    assert (o[1, 8:12, 9] == float("inf")).all()       # item 6: an infinite value under a positive probability
    keep = torch.ones_like(o, dtype=torch.bool)
    keep[1, 4:8] = False
    keep[1, 8:12, 9] = False
    assert torch.equal(o[keep], clean[keep])
    assert rc.poll_status() == 0
