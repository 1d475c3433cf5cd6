"""Timed cases of the operators that make the decode cache smaller, through the package's public calls.

  pack    compact_routes_q8: the visible, kept rows of cached resources go into 64-token pages of 8-bit
          values (e4m3) with one power-of-two scale for a page's keys and one for its values
  decode8 attend_decode_q8: one token for every running sequence; its resource rows lie in 8-bit pages, its
          conversation in pages of the storage type, to which the call appends the current token
  weigh   attend_decode_weighted: one token for every running sequence over pages of the storage type, and the
          attention that every row got is added to the row's weight
  evict   evict_rows: items longer than a budget keep their last rows and, of the others, those with
          the greatest weights, copied to fresh pages

Lengths follow from the case alone (`mix` seeds them), so that the work of a case is known; tensors,
keep masks, routes and page orders follow from the seed.  Activations and cached rows are N(0,1), as
normalised projections are.
"""
import functools
import math

import numpy as np
import torch

own = False            # True: the framework's kernels; False: the same in elementary torch operations

PAGE = 64              # tokens of a page
HEADS_KV, DIM = 8, 128
THETA = 1.0e6
MAX_POS = 131072       # rows of the rotary table: the longest context served
KEPT, ROUTED = 0.30, 0.25   # share of a resource's tokens that the masks keep; share of the resources that a KV group sees
E4M3_MAX = 448.0


def _case(kind, name=None, hq=32, **sizes):
    case = {"kind": kind, "hq": hq, **sizes}
    return {"name": name, **case} if name else case


def listed():
    return [
        # one user's first turn over a handful of tools: its routes are packed before the first decode step
        _case("pack", "pack-one-request", batch=1, res=8, lo=200, hi=800, mix=2),
        # a batch of first turns over ordinary tools
        _case("pack", "pack-batch", batch=16, res=16, lo=150, hi=1200, mix=3),
        # a full server is refilled: the routes of all its sequences
        _case("pack", "pack-full-server", batch=64, res=16, lo=500, hi=700, mix=4),
        # one user alone, a decode step of some ten microseconds
        _case("decode8", "decode8-one-sequence", batch=1, res_lo=720, res_hi=720, hist_lo=700, hist_hi=700, mix=5),
        # ragged long tool results and short conversations, eight query heads to a KV head
        _case("decode8", "decode8-ragged", hq=64, batch=16, res_lo=500, res_hi=6000, hist_lo=30, hist_hi=2000, mix=6),
        # the steady decode of a full server over long resources
        _case("decode8", "decode8-full-server", batch=64, res_lo=4096, res_hi=4096, hist_lo=1024, hist_hi=1024, mix=7),
        # one user alone, weights kept
        _case("weigh", "weigh-one-sequence", batch=1, res_lo=720, res_hi=720, hist_lo=1500, hist_hi=1500, mix=8),
        # ragged running conversations, two query heads to a KV head
        _case("weigh", "weigh-ragged", hq=16, batch=16, res_lo=300, res_hi=900, hist_lo=300, hist_hi=4000, mix=9),
        # the steady decode of a full server
        _case("weigh", "weigh-full-server", batch=64, res_lo=720, res_hi=720, hist_lo=2048, hist_hi=2048, mix=10),
        # one conversation has grown a page past its budget
        _case("evict", "evict-one-sequence", batch=1, lo=1088, hi=1088, budget=1024, recent=64, mix=11),
        # ragged conversations of a full server come back to a common budget; the short ones stay
        _case("evict", "evict-full-server", batch=64, lo=1500, hi=4500, budget=2048, recent=256, mix=12),
        # a few very long documents
        _case("evict", "evict-long", batch=4, lo=40000, hi=90000, budget=16384, recent=1024, mix=13),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(rng, lo, hi):
    """A range of lengths inside [lo, hi]."""
    a, b = _log(rng, lo, hi), _log(rng, lo, hi)
    return min(a, b), max(a, b)


def draw(rng):
    kind = rng.choice(["pack", "pack", "decode8", "decode8", "decode8", "weigh", "weigh", "weigh", "evict", "evict"])
    mix, batch = rng.randrange(1 << 16), _log(rng, 1, 64)
    most = {c["name"]: work(c)["bytes"] for c in listed()}      # a drawn case costs no more than its kind's largest
    if kind == "pack":
        lo, hi = _span(rng, 60, 2000)
        case = _case("pack", hq=rng.choice([16, 32, 32, 64]), batch=batch, res=_log(rng, 1, 32), lo=lo, hi=hi, mix=mix)
        limit = most["pack-full-server"]
    elif kind == "evict":
        lo, hi = _span(rng, 100, 60000 if batch <= 8 else 6000)
        case = _case("evict", hq=32, batch=batch, lo=lo, hi=hi, mix=mix)
        longest = int(_evict_lengths(case).max())
        case["budget"] = _log(rng, longest // 8, longest - 1)
        case["recent"] = rng.randrange(0, case["budget"] + 1) if rng.random() < 0.8 else 0
        limit = most["evict-full-server"]
    else:
        hq = rng.choice([8, 16, 24, 32, 32, 40, 64])
        long = 60000 if batch <= 2 else 8000
        res_lo, res_hi = _span(rng, 40, long) if rng.random() < 0.9 else (0, 0)
        h_lo, h_hi = _span(rng, 1, 4096)
        case = _case(kind, hq=hq, batch=batch, res_lo=res_lo, res_hi=res_hi, hist_lo=h_lo, hist_hi=h_hi, mix=mix)
        limit = most["decode8-full-server" if kind == "decode8" else "weigh-full-server"]
    while case["batch"] > 1 and work(case)["bytes"] > limit:
        case["batch"] = max(1, case["batch"] * 3 // 4)
    return case


# ---------------------------------------------------------------- sizes of a case --
@functools.lru_cache(maxsize=64)
def _lengths(mix, batch, *spans):
    """One array of lengths for each (low, high, columns)."""
    rng = np.random.default_rng([mix, 19662])
    return tuple(rng.integers(lo, hi + 1, (batch, n)).astype(np.int64) for lo, hi, n in spans)


def _pack_lengths(case):
    return _lengths(case["mix"], case["batch"], (case["lo"], case["hi"], case["res"]))[0]


def _decode_lengths(case):
    """(resource rows, conversation rows), one of each for every item = sequence x KV group."""
    res, hist = _lengths(case["mix"], case["batch"], (case["res_lo"], case["res_hi"], HEADS_KV), (case["hist_lo"], case["hist_hi"], 1))
    return res.reshape(-1), np.repeat(hist.reshape(-1), HEADS_KV)


def _evict_lengths(case):
    return np.repeat(_lengths(case["mix"], case["batch"], (case["lo"], case["hi"], 1))[0].reshape(-1), HEADS_KV)


def _visible(n_res):
    return max(1, int(math.floor(ROUTED * n_res + 0.5)))


def work(case):
    row = DIM * 2                                         # bytes of one key or value row in bf16
    if case["kind"] == "pack":
        res = _pack_lengths(case)
        rows = float((res.mean(1) * _visible(res.shape[1])).sum()) * KEPT * HEADS_KV
        return {"bytes": float(res.sum()) + rows * (2 * row + row + 4), "flops": 2 * 2 * DIM * rows}
    if case["kind"] == "evict":
        n = _evict_lengths(case)
        over = n[n > case["budget"]]
        return {"bytes": 4.0 * n.size * 2 + 4.0 * float(over.sum()) + float(over.size) * case["budget"] * (4 * row + 8), "flops": float(over.sum())}
    res, hist = _decode_lengths(case)
    io = case["batch"] * (2 * case["hq"] + 4 * HEADS_KV) * row          # q, k, v in, o and the appended row out
    flops = 4.0 * DIM * (case["hq"] // HEADS_KV) * float(res.sum() + hist.sum())
    if case["kind"] == "decode8":
        return {"bytes": float(res.sum()) * row + float(((res + PAGE - 1) // PAGE).sum()) * 8 + float(hist.sum()) * 2 * row + io, "flops": flops}
    return {"bytes": float(res.sum() + hist.sum()) * (2 * row + 8) + io, "flops": flops}


# ------------------------------------------------------------------------ inputs --
class _Draw:
    """Seeded tensors on the device, and index arrays from the same seed."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(int(seed))
        self.np = np.random.default_rng([int(seed), 1])

    def normal(self, *shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=self.gen, dtype=dtype, device="cuda")

    @staticmethod
    def ints(a, dtype=np.int32):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def _zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def _power(e):
    """2^e in fp32, for exponents of normal numbers."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _pages_of(rows):
    return (rows + PAGE - 1) // PAGE


def _tables(counts, ids, width):
    """Page tables padded with -1; each item takes the next ids."""
    out = np.full((len(counts), int(width)), -1, np.int32)
    out[np.arange(out.shape[1])[None, :] < counts[:, None]] = ids[:int(counts.sum())]
    return _Draw.ints(out)


def _keep(rng, total):
    """About 30 % of the tokens, as field spans of 4-32 tokens."""
    n = total // 40 + 2
    spans, gaps = rng.integers(4, 33, n), rng.integers(10, 75, n)
    flags = np.repeat(np.tile(np.array([0, 1], np.uint8), n), np.stack([gaps, spans], 1).reshape(-1))
    return np.resize(flags, total)


def _prepare_pack(case, dr):
    res = _pack_lengths(case)
    batch, n, g = res.shape[0], res.shape[1], HEADS_KV
    flat = res.reshape(-1)
    pool, slot = int(flat.sum()), np.concatenate([[0], np.cumsum(flat)[:-1]])
    keep = _keep(dr.np, pool)
    vis = np.zeros((g, batch, n), np.uint8)
    order = np.argsort(dr.np.random((g, batch, n)), axis=2)[:, :, :_visible(n)]
    np.put_along_axis(vis, order, 1, axis=2)
    room = np.sort(res, axis=1)[:, -_visible(n):].sum(1)         # rows that a route can hold at most: what buffers are sized for
    pages = int(_pages_of(room).sum()) * g
    st = dict(k_cache=dr.normal(g, pool, DIM), v_cache=dr.normal(g, pool, DIM), keep=dr.ints(keep, np.uint8), vis=dr.ints(vis.reshape(g, -1), np.uint8),
              res_off=dr.ints(np.arange(batch + 1) * n), res_slot=dr.ints(slot), res_len=dr.ints(flat), free=dr.ints(dr.np.permutation(pages)),
              route_cu=_zeros(batch * g + 1, dtype=torch.int32), route_len=_zeros(batch * g, dtype=torch.int32),
              route_idx=_zeros(int(room.sum()) * g, dtype=torch.int32), table=_zeros(batch * g, int(_pages_of(room).max()), dtype=torch.int32))
    for x in ("k", "v"):
        st[x + "_pages8"], st[x + "_scale"] = _zeros(pages, PAGE, DIM, dtype=torch.float8_e4m3fn), _zeros(pages, dtype=torch.float32)
    return st


def _prepare_decode(case, dr):
    res, hist = _decode_lengths(case)
    hq, g, batch = case["hq"], HEADS_KV, case["batch"]
    st = dict(q=dr.normal(batch, hq, DIM), k_new=dr.normal(batch, g, DIM), v_new=dr.normal(batch, g, DIM), q_pos=dr.ints((res.reshape(batch, g).max(1) * 4 + hist[::g]) % MAX_POS),
              res_len=dr.ints(res), hist_len=dr.ints(hist))
    n_res, n_hist = int(_pages_of(res).sum()), int(_pages_of(hist).sum())
    widths = max(1, int(_pages_of(res).max())), int(_pages_of(hist).max())
    if case["kind"] == "decode8":
        st["res_table"] = _tables(_pages_of(res), dr.np.permutation(max(n_res, 1)), widths[0])
        st["hist_table"] = _tables(_pages_of(hist), dr.np.permutation(n_hist), widths[1])
        for x in ("k", "v"):
            rows = dr.normal(max(n_res, 1), PAGE, DIM)
            _, e = torch.frexp(rows.float().abs().amax((1, 2)) / E4M3_MAX)
            scale = _power(e)
            st[x + "_pages8"], st[x + "_scale"] = (rows.float() / scale[:, None, None]).to(torch.float8_e4m3fn), scale
        st["k_pages"], st["v_pages"] = dr.normal(n_hist, PAGE, DIM), dr.normal(n_hist, PAGE, DIM)
    else:
        ids = dr.np.permutation(n_res + n_hist)
        st["res_table"], st["hist_table"] = _tables(_pages_of(res), ids[:n_res], widths[0]), _tables(_pages_of(hist), ids[n_res:], widths[1])
        st["k_pages"], st["v_pages"] = dr.normal(n_res + n_hist, PAGE, DIM), dr.normal(n_res + n_hist, PAGE, DIM)
        # what some hundred earlier steps have left
        st["weight_in"] = torch.rand((n_res + n_hist, PAGE), generator=dr.gen, device="cuda").square() * 0.2
        st["weight_out"] = _zeros(n_res + n_hist, PAGE, dtype=torch.float32)
    return st


def _prepare_evict(case, dr):
    n = _evict_lengths(case)
    counts, new = _pages_of(n), int(_pages_of(np.int64(case["budget"])))
    old, fresh = int(counts.sum()), int((n > case["budget"]).sum()) * new
    ids = dr.np.permutation(old + fresh)
    # sums of probabilities: a few rows have most of it, and some nothing at all
    weight = torch.exp(2 * dr.normal(old + fresh, PAGE, dtype=torch.float32)) * 1e-2
    weight[torch.rand(weight.shape, generator=dr.gen, device="cuda") < 0.05] = 0.0
    return dict(k_pages=dr.normal(old + fresh, PAGE, DIM), v_pages=dr.normal(old + fresh, PAGE, DIM), weight=weight, table=_tables(counts, ids, int(counts.max())),
                row_len=dr.ints(n), free=dr.ints(ids[old:]), new_table=torch.full((n.size, new), -1, dtype=torch.int32, device="cuda"),
                new_len=_zeros(n.size, dtype=torch.int32), kept=torch.full((n.size, case["budget"]), -1, dtype=torch.int32, device="cuda"))


def prepare(case, seed):
    dr = _Draw(seed)
    make = {"pack": _prepare_pack, "evict": _prepare_evict}.get(case["kind"], _prepare_decode)
    return {"case": dict(case), **make(case, dr)}


# -------------------------------------------------------------- the plain forms --
def _rotate(x, pos):
    """Rows x [n][heads][128] at positions pos [n]: element i pairs with i + 64; the result is a tensor of the storage type again.
    One rounding after the second product, so that a value next to a border of the storage type falls on the same side
    wherever the rotation is done with fused multiply-adds: hence the 64-bit products."""
    inv = THETA ** (-torch.arange(0, DIM, 2, dtype=torch.float64, device=x.device) / DIM)
    angle = pos.double()[:, None, None] * inv
    c, s = angle.cos().float().double(), angle.sin().float().double()
    lo, hi = x[..., :DIM // 2].double(), x[..., DIM // 2:].double()
    out = torch.cat([lo * c - (hi * s).float().double(), hi * c + (lo * s).float().double()], -1)
    return out.float().to(torch.bfloat16)


def _rows(table, lengths):
    """Pool rows [items][longest] of page tables (0 where there is none), and which of them there are."""
    at = torch.arange(max(1, int(table.shape[1]) * PAGE), device=table.device)
    there = at[None, :] < lengths[:, None]
    if table.shape[1] == 0:
        return torch.zeros_like(there, dtype=torch.int64), there
    rows = table.long()[:, at // PAGE] * PAGE + at % PAGE
    return torch.where(there, rows, torch.zeros_like(rows)), there


def _append(st):
    """The current token's key and value become the last row of each item's conversation."""
    g, b = HEADS_KV, st["q"].shape[0]
    last = st["hist_len"].long() - 1
    page = st["hist_table"].long().gather(1, (last // PAGE)[:, None])[:, 0]
    st["k_pages"][page, last % PAGE] = _rotate(st["k_new"], st["q_pos"]).reshape(b * g, DIM)
    st["v_pages"][page, last % PAGE] = st["v_new"].reshape(b * g, DIM)
    return page, last % PAGE


def _probabilities(q, keys, there):
    """Softmax over the rows that are there, [items][heads of the group][rows]."""
    s = torch.matmul(q, keys.transpose(1, 2)) / math.sqrt(DIM)
    s = s.masked_fill(~there[:, None, :], float("-inf"))
    p = torch.exp(s - s.amax(-1, keepdim=True))
    return p / p.sum(-1, keepdim=True)


def _queries(st, hq):
    b = st["q"].shape[0]
    return _rotate(st["q"], st["q_pos"]).float().reshape(b * HEADS_KV, hq // HEADS_KV, DIM)


def _plain_decode8(st, hq):
    _append(st)
    res, res_there = _rows(st["res_table"], st["res_len"])
    hist, hist_there = _rows(st["hist_table"], st["hist_len"])

    def all_rows(x):
        part = st[x + "_pages8"].reshape(-1, DIM).view(torch.uint8)[res].view(torch.float8_e4m3fn).float()
        part = part * st[x + "_scale"][res // PAGE][..., None]
        return torch.cat([torch.where(res_there[..., None], part, 0.0), torch.where(hist_there[..., None], st[x + "_pages"].reshape(-1, DIM)[hist].float(), 0.0)], 1)

    p = _probabilities(_queries(st, hq), all_rows("k"), torch.cat([res_there, hist_there], 1))
    o = torch.matmul(p, all_rows("v")).reshape(-1, hq, DIM).to(torch.bfloat16)
    return {"o": o, "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _plain_weigh(st, hq):
    page, slot = _append(st)
    res, res_there = _rows(st["res_table"], st["res_len"])
    hist, hist_there = _rows(st["hist_table"], st["hist_len"])
    rows, there = torch.cat([res, hist], 1), torch.cat([res_there, hist_there], 1)
    p = _probabilities(_queries(st, hq), torch.where(there[..., None], st["k_pages"].reshape(-1, DIM)[rows].float(), 0.0), there)
    o = torch.matmul(p, torch.where(there[..., None], st["v_pages"].reshape(-1, DIM)[rows].float(), 0.0)).reshape(-1, hq, DIM).to(torch.bfloat16)
    before = st["weight_in"].clone()
    before[page, slot] = 0.0                       # the appended token has no weight yet
    weight = st["weight_out"].reshape(-1)
    weight[rows[there]] = (before.reshape(-1)[rows] + p.sum(1))[there]
    return {"o": o, "weight": st["weight_out"], "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _plain_pack(st):
    g, device = HEADS_KV, st["keep"].device
    n_req, n_listed = st["res_off"].numel() - 1, st["res_len"].numel()
    # every (group, token of a listed resource), those that are visible and kept, by route
    res = torch.repeat_interleave(torch.arange(n_listed, device=device), st["res_len"].long())
    first = torch.cumsum(st["res_len"].long(), 0) - st["res_len"].long()
    row = st["res_slot"].long()[res] + torch.arange(res.numel(), device=device) - first[res]
    seen = (st["vis"][:, res] != 0) & (st["keep"][row] != 0)[None, :]
    group, token = torch.nonzero(seen, as_tuple=True)
    request = torch.searchsorted(st["res_off"].long(), res[token], right=True) - 1
    route, order = torch.sort(request * g + group, stable=True)
    row, group = row[token][order], group[order]
    lens = torch.bincount(route, minlength=n_req * g)
    ends = torch.cumsum(lens, 0)
    st["route_len"].copy_(lens)
    st["route_cu"][0] = 0
    st["route_cu"][1:] = ends
    st["route_idx"][:row.numel()] = row.to(torch.int32)
    # pages: each route takes the next ones of the free list
    rank = torch.arange(row.numel(), device=device) - (ends - lens)[route]
    n_pages = (lens + PAGE - 1) // PAGE
    first_page = torch.cumsum(n_pages, 0) - n_pages
    at = torch.arange(st["table"].shape[1], device=device)
    there = at[None, :] < n_pages[:, None]
    ids = st["free"][torch.clamp(first_page[:, None] + at, max=st["free"].numel() - 1)]
    st["table"].copy_(torch.where(there, ids, -1))
    page = st["free"].long()[first_page[route] + rank // PAGE]
    for x in ("k", "v"):
        rows = st[x + "_cache"][group, row].float()
        most = torch.zeros_like(st[x + "_scale"]).scatter_reduce(0, page, rows.abs().amax(1), "amax")
        m, e = torch.frexp(most)                                   # most = m 2^e with m in [1/2, 1); 448 = 7/8 2^9
        e = torch.where(most > 0, torch.clamp(e - 9 + (m > 0.875).int(), min=-126), 0)
        scale = _power(e)
        used = st["free"].long()[:int(n_pages.sum())]
        st[x + "_scale"][used] = scale[used]
        st[x + "_pages8"].view(torch.uint8)[page, rank % PAGE] = (rows / scale[page][:, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return _packed(st)


def _packed(st):
    return {k: st[k] for k in ("k_pages8", "v_pages8", "k_scale", "v_scale", "route_cu", "route_len", "route_idx", "table")}


def _plain_evict(st, budget, recent):
    device, lens = st["row_len"].device, st["row_len"].long()
    over = lens > budget
    rows, there = _rows(st["table"], lens)
    at = torch.arange(rows.shape[1], device=device)
    candidate = there & (at[None, :] < lens[:, None] - recent)
    # by weight, the earlier row first among equals; the last rows stay whatever their weight
    rank = torch.where(candidate, st["weight"].reshape(-1)[rows], float("-inf"))
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices
    place = torch.empty_like(order).scatter_(1, order, at[None, :].expand_as(order))
    stays = there & (~candidate | (place < budget - recent) | ~over[:, None])
    item, old = torch.nonzero(stays, as_tuple=True)
    new_len = torch.where(over, budget, lens)
    new = torch.arange(item.numel(), device=device) - (torch.cumsum(new_len, 0) - new_len)[item]
    st["kept"][item, new] = old.to(torch.int32)
    st["new_len"].copy_(new_len)
    n_new = st["new_table"].shape[1]
    fresh = ((torch.cumsum(over.long(), 0) - 1) * n_new)[:, None] + torch.arange(n_new, device=device)
    mine = torch.arange(n_new, device=device)[None, :] < ((new_len + PAGE - 1) // PAGE)[:, None]
    pages = torch.where(over[:, None], st["free"][torch.clamp(fresh, 0, max(0, st["free"].numel() - 1))] if st["free"].numel() else -1,
                        torch.nn.functional.pad(st["table"], (0, max(0, n_new - st["table"].shape[1])), value=-1)[:, :n_new])
    st["new_table"].copy_(torch.where(mine, pages, st["new_table"]))
    moved = over[item]
    item, old, new = item[moved], old[moved], new[moved]
    src, dst = rows[item, old], st["new_table"].long()[item, new // PAGE] * PAGE + new % PAGE
    for x in ("k_pages", "v_pages"):
        st[x].reshape(-1, DIM)[dst] = st[x].reshape(-1, DIM)[src]
    st["weight"].reshape(-1)[dst] = st["weight"].reshape(-1)[src]
    return _evicted(st)


def _evicted(st):
    return {k: st[k] for k in ("k_pages", "v_pages", "weight", "new_table", "new_len", "kept")}


# ----------------------------------------------------------- the framework's calls --
@functools.lru_cache(maxsize=8)
def _context(hq):
    """The attention shape's context: made once by a program, like the model's weights."""
    from paper_2608_19662_b200 import ReCache
    return ReCache(hq, HEADS_KV, DIM, THETA, "bf16", max_pos=MAX_POS, page_tokens=PAGE, device=torch.cuda.current_device())


def run(state):
    st, case = state, state["case"]
    kind, hq = case["kind"], case["hq"]
    if not own:
        if kind == "pack":
            return _plain_pack(st)
        if kind == "evict":
            return _plain_evict(st, case["budget"], case["recent"])
        return _plain_decode8(st, hq) if kind == "decode8" else _plain_weigh(st, hq)
    rc = _context(hq)
    if kind == "pack":
        rc.compact_routes_q8(st["k_cache"], st["v_cache"], st["keep"], st["res_off"], st["res_slot"], st["res_len"], st["vis"], st["route_cu"], st["route_idx"],
                             st["k_pages8"], st["v_pages8"], st["k_scale"], st["v_scale"], st["table"], st["free"], route_len=st["route_len"])
        return _packed(st)
    if kind == "evict":
        rc.evict_rows(st["k_pages"], st["v_pages"], st["weight"], st["table"], st["row_len"], case["budget"], case["recent"], st["free"], st["new_table"],
                      st["new_len"], st["kept"])
        return _evicted(st)
    if kind == "decode8":
        o = rc.attend_decode_q8(st["q"], st["q_pos"], st["k_pages8"], st["v_pages8"], st["k_scale"], st["v_scale"], st["res_table"], st["res_len"], st["k_pages"],
                                st["v_pages"], st["hist_table"], st["hist_len"], k_new=st["k_new"], v_new=st["v_new"])
        return {"o": o, "k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    o = rc.attend_decode_weighted(st["q"], st["q_pos"], st["k_pages"], st["v_pages"], st["res_table"], st["res_len"], st["hist_table"], st["hist_len"],
                                  st["weight_out"], weight_in=st["weight_in"], k_new=st["k_new"], v_new=st["v_new"])
    return {"o": o, "weight": st["weight_out"], "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


# ------------------------------------------------------------- in 64 bits, item by item --
def _exact_rotate(x, pos):
    """The rotation as a product of complex numbers, rounded to the storage type (rotated rows are tensors of that type)."""
    n = DIM // 2
    z = torch.complex(x[..., :n].double(), x[..., n:].double())
    angle = torch.tensor([float(pos) * THETA ** (-2.0 * i / DIM) for i in range(n)], dtype=torch.float64, device=x.device)
    z = z * torch.polar(torch.ones_like(angle), angle)
    return torch.cat([z.real, z.imag], -1).to(torch.bfloat16).double()


def _exact_decode(case, st):
    res, hist = _decode_lengths(case)
    s, weigh = case["hq"] // HEADS_KV, case["kind"] == "weigh"
    o = torch.zeros(case["batch"], case["hq"], DIM, dtype=torch.float64, device="cuda")
    kp, vp = st["k_pages"].double(), st["v_pages"].double()
    weight = torch.zeros(st["weight_in"].shape, dtype=torch.float64, device="cuda") if weigh else None
    res_table, hist_table, pos = st["res_table"].cpu().numpy(), st["hist_table"].cpu().numpy(), st["q_pos"].cpu().numpy()
    for it in range(len(res)):
        b, g, n, h = it // HEADS_KV, it % HEADS_KV, int(res[it]), int(hist[it])
        rp, hp = torch.tensor(res_table[it][:-(-n // PAGE)], device="cuda").long(), torch.tensor(hist_table[it][:-(-h // PAGE)], device="cuda").long()
        kp[hp[-1], (h - 1) % PAGE] = _exact_rotate(st["k_new"][b, g], pos[b])
        vp[hp[-1], (h - 1) % PAGE] = st["v_new"][b, g].double()
        if weigh:
            first = [x[rp].reshape(-1, DIM)[:n] for x in (kp, vp)]
        else:
            first = [(st[x + "_pages8"].view(torch.uint8)[rp].view(torch.float8_e4m3fn).double() * st[x + "_scale"][rp].double()[:, None, None]).reshape(-1, DIM)[:n] for x in "kv"]
        keys, values = (torch.cat([f, x[hp].reshape(-1, DIM)[:h]]) for f, x in zip(first, (kp, vp)))
        q = _exact_rotate(st["q"][b, g * s:(g + 1) * s], pos[b])
        p = torch.softmax(q @ keys.T / DIM ** 0.5, -1)
        o[b, g * s:(g + 1) * s] = p @ values
        if weigh:
            got = p.sum(0)
            prior = st["weight_in"].double()
            for pages, part, count in ((rp, got[:n], n), (hp, got[n:], h)):
                slots = (pages[:, None] * PAGE + torch.arange(PAGE, device="cuda")).reshape(-1)[:count]
                weight.reshape(-1)[slots] = part + prior.reshape(-1)[slots]
            weight[hp[-1], (h - 1) % PAGE] = got[-1]
    return {"o": o, **({"weight": weight} if weigh else {}), "k_pages": kp, "v_pages": vp}


def _exact_e4m3(x):
    """The nearest value with three bits after the leading one and exponents from -6 (even last bit among equals)."""
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)
    return np.rint(x / step) * step


def _exact_pack(case, st):
    if work(case)["bytes"] > 1.5e8:                # minutes on the host
        return None
    c = {k: v.cpu().numpy() for k, v in st.items() if isinstance(v, torch.Tensor) and v.dtype in (torch.int32, torch.uint8)}
    cache = [st[x].double().cpu().numpy() for x in ("k_cache", "v_cache")]
    out = {k: np.zeros(tuple(st[k].shape)) for k in ("k_pages8", "v_pages8", "k_scale", "v_scale")}
    free = iter(c["free"])
    for b in range(case["batch"]):
        for g in range(HEADS_KV):
            rows = [np.flatnonzero(c["keep"][s:s + n]) + s for s, n, v in zip(c["res_slot"], c["res_len"], c["vis"][g])][c["res_off"][b]:c["res_off"][b + 1]]
            seen = c["vis"][g][c["res_off"][b]:c["res_off"][b + 1]]
            rows = np.concatenate([r for r, v in zip(rows, seen) if v] + [np.zeros(0, np.int64)]).astype(np.int64)
            for at in range(0, len(rows), PAGE):
                page = next(free)
                for name, x in zip("kv", cache):
                    part = x[g, rows[at:at + PAGE]]
                    top, scale = np.abs(part).max(), 1.0
                    while top > E4M3_MAX * scale:
                        scale *= 2
                    while 0 < top <= E4M3_MAX * scale / 2 and scale > 2.0 ** -126:
                        scale /= 2
                    out[name + "_scale"][page] = scale
                    out[name + "_pages8"][page, :len(part)] = _exact_e4m3(part / scale)
    return {**out, "route_cu": None, "route_len": None, "route_idx": None, "table": None}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "pack":
        return _exact_pack(case, st)
    if case["kind"] == "evict":
        return None                                # copies and whole numbers: nothing is computed
    return _exact_decode(case, st)
