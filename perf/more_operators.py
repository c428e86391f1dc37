"""The operators that serve a language model from a paged cache of codes, as measurable cases.

  attend   Context.cache_attend: one new token of each sequence over its cached keys and values, all of them or those of picked pages
  select   Context.cache_select: the pages of each sequence whose stand-ins score highest against the new token's queries
  extend   Context.cache_extend and cache_copy: pages and slots for a step's new rows, with copies of pages that forks share
  compact  Context.cache_compact and cache_copy: pages in use moved to the front of the cache

A cache for attention has its G key heads first and its G value heads behind them; R query heads share a key head.  D = 128, M = 8 or 16
and K = 256 are the 64- and 128-bit codes of the repository's benchmark; head counts, sequence lengths and pages are generic.
"""
import math

import torch

own = False


def listed():
    return [
        # one step of one short sequence: latency is all there is
        {"name": "attend_short", "op": "attend", "B": 1, "n": 150, "G": 8, "R": 4, "D": 128, "M": 8, "K": 256, "page": 16, "type": "bf16", "scaled": True, "picks": 0},
        # a few sequences, one of them empty, odd head size, odd group, small dictionaries, no scales
        {"name": "attend_odd", "op": "attend", "B": 5, "n": 1237, "G": 3, "R": 5, "D": 80, "M": 5, "K": 200, "page": 24, "type": "fp32", "scaled": False, "picks": 0},
        # a batch of ordinary contexts with the better codes
        {"name": "attend_batch", "op": "attend", "B": 32, "n": 4096, "G": 8, "R": 4, "D": 128, "M": 16, "K": 256, "page": 16, "type": "fp16", "scaled": True, "picks": 0},
        # one long context, many query heads a key head
        {"name": "attend_long", "op": "attend", "B": 1, "n": 131071, "G": 8, "R": 8, "D": 128, "M": 8, "K": 256, "page": 64, "type": "bf16", "scaled": True, "picks": 0},
        # a large batch of long contexts
        {"name": "attend_many", "op": "attend", "B": 64, "n": 16384, "G": 8, "R": 4, "D": 128, "M": 8, "K": 256, "page": 64, "type": "bf16", "scaled": True, "picks": 0},
        # 64 pages of every long context, as a selection leaves them
        {"name": "attend_picked", "op": "attend", "B": 16, "n": 65536, "G": 8, "R": 4, "D": 128, "M": 8, "K": 256, "page": 64, "type": "bf16", "scaled": True, "picks": 64},
        # sixteen pages of one context
        {"name": "select_one", "op": "select", "B": 1, "n": 8000, "G": 8, "R": 4, "D": 128, "M": 8, "K": 256, "page": 64, "type": "bf16", "scaled": True, "picks": 16},
        # 64 of two thousand pages for every sequence of a batch
        {"name": "select_long", "op": "select", "B": 32, "n": 131072, "G": 8, "R": 4, "D": 128, "M": 8, "K": 256, "page": 64, "type": "bf16", "scaled": True, "picks": 64},
        # one row more for every sequence of a batch
        {"name": "extend_step", "op": "extend", "B": 64, "P": 64, "n": 2048, "add": 1, "G": 8, "M": 8, "page": 16, "scaled": True},
        # a step of a beam search: every hypothesis continues one of the last step's, several of them the same
        {"name": "extend_beams", "op": "extend", "B": 256, "P": 256, "n": 4001, "add": 1, "G": 8, "M": 16, "page": 64, "scaled": True, "forks": True},
        # a small cache, an odd page
        {"name": "compact_small", "op": "compact", "B": 7, "n": 500, "G": 2, "M": 5, "page": 24, "scaled": False},
        # a large one half of whose sequences have ended
        {"name": "compact_large", "op": "compact", "B": 128, "n": 8192, "G": 8, "M": 8, "page": 64, "scaled": True},
    ]


def _between(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "select", "extend", "compact"])
    G, M = rng.choice([1, 2, 8, _between(rng, 1, 16)]), rng.choice([8, 8, 16, _between(rng, 2, 16)])
    case = {"op": op, "G": G, "M": M, "page": rng.choice([1, 16, 24, 64, 128] if op == "attend" else [16, 24, 64, 128]), "scaled": rng.random() < 0.75}
    B = case["B"] = _between(rng, 1, 64)
    if op in ("attend", "select"):
        case.update(R=rng.choice([1, 4, 8, _between(rng, 1, 16)]), D=rng.choice([64, 128, 128, 4 * _between(rng, 8, 64)]), K=rng.choice([256, 256, _between(rng, 16, 256)]),
                    type=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
        # products with codewords, and rows x heads x query heads a key head x dictionaries, of the largest listed cases
        case["B"] = B = max(1, min(B, 32 * 8 * 4 * 16 * 256 * 128 // (G * case["R"] * M * case["K"] * case["D"])))
        most = (64 * 16384 * 8 * 4 * 8) // (B * G * max(case["R"], 4) * max(M, 8))
        case["n"] = _between(rng, 1, max(1, min(131072, most)))
        case["picks"] = 0
        if op == "select":                                          # there is something to choose
            case["n"] = max(case["n"], 50 * case["page"])
            case["picks"] = _between(rng, 6, min(128, case["n"] // (4 * case["page"])))
        elif rng.random() < 0.3:
            case.update(picks=_between(rng, 1, 64), page=max(case["page"], 16))
    elif op == "extend":
        forks = rng.random() < 0.5
        case.update(n=_between(rng, 1, 8192), add=rng.choice([1, 1, _between(rng, 1, 100)]), P=B, forks=forks)
    else:
        case["n"] = _between(rng, 1, max(1, min(8192, 128 * 8192 * 8 * 8 // (B * G * max(M, 8)))))
    return case


def _lengths(case):
    """The sequences' lengths: from n evenly down to about half of it, the last of several short ones empty."""
    B, n = case.get("P", case["B"]), case["n"]
    lens = [n - (n // 2) * b // max(1, B - 1) for b in range(B)]
    if case["op"] != "select" and B > 2 and n < 2000:
        lens[-1] = 0
    return lens


def _parents(case):
    """Which of the P sequences each of the B new ones continues."""
    B, P = case["B"], case["P"]
    return [(i * i + i // 3) % P for i in range(B)] if case.get("forks") else list(range(B))


# ---- inputs ---------------------------------------------------------------------------------------------------------------

_TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def _codes(shape, K, g, dev):
    """Codes as greedy encoding gives them: the first dictionaries' first codewords are met more often."""
    u = torch.rand(shape, generator=g, device=dev)
    u[..., :2] *= u[..., :2]
    return (u * K).clamp_(max=K - 1).to(torch.uint8)


def _tables(pages_of, g, dev, more):
    """Tables of sequences of so many pages, scattered over a pool that is `more` times as large; and the pool's size."""
    need = sum(pages_of)
    pool = int(need * more) + 1
    pages = torch.randperm(pool, generator=g, device=dev)[:need].int()
    tables = torch.zeros((len(pages_of), max(1, max(pages_of))), dtype=torch.int32, device=dev)
    at = 0
    for b, p in enumerate(pages_of):
        tables[b, :p] = pages[at:at + p]
        at += p
    return tables, pool


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    op, G, M, page = case["op"], case["G"], case["M"], case["page"]
    s = {"case": case}
    lens = _lengths(case)
    up = lambda x: (x + page - 1) // page
    if op in ("attend", "select"):
        B, R, D, K, dt = case["B"], case["R"], case["D"], case["K"], _TYPES[case["type"]]
        H = 2 * G if op == "attend" else G
        fall = 0.75 ** torch.arange(M, device=dev)[None, :, None, None]
        s["C"] = 0.6 * fall * torch.randn((H, M, K, D), generator=g, device=dev)
        # the queries lie in the output of a projection that gives keys and values too
        wide = torch.randn((B, G * R + 2 * G, D), generator=g, device=dev).to(dt)
        s["Q"] = wide[:, :G * R]
        s["tables"], pool = _tables([up(x) for x in lens], g, dev, 1.25)
        s["lengths"] = torch.tensor(lens, dtype=torch.int32, device=dev)
        rows = pool * page if op == "attend" else pool             # select: one stand-in a page
        s["codes"] = _codes((rows, H, M), K, g, dev)
        s["scale"] = torch.exp(0.3 * torch.randn((rows, H), generator=g, device=dev)) if case["scaled"] else None
        if op == "attend":
            s["out"] = torch.zeros((B, G * R, D), dtype=dt, device=dev)
            s["picked"] = None
            if case["picks"]:                                       # a different choice of pages a head, ascending, the last page among them
                order = torch.rand((B, G, s["tables"].shape[1]), generator=g, device=dev)
                j = torch.arange(s["tables"].shape[1], device=dev)
                live = torch.tensor([up(x) for x in lens], device=dev)[:, None, None]
                order = torch.where(j < live, order, -1.0)
                order = torch.where(j == live - 1, 2.0, order)
                k = min(case["picks"], order.shape[2])
                best = order.topk(k, dim=2)
                picked = torch.where(best.values < 0, 2 ** 30, best.indices).sort(2).values
                s["picked"] = torch.full((B, G, case["picks"]), -1, dtype=torch.int32, device=dev)
                s["picked"][:, :, :k] = torch.where(picked == 2 ** 30, -1, picked).int()
        else:
            s["picked"] = torch.zeros((B, G, case["picks"]), dtype=torch.int32, device=dev)
    else:
        B = case["B"]
        s["tables0"], pool = _tables([up(x + case.get("add", 0)) for x in lens], g, dev, 1.5 if op == "extend" else 2.0)
        if op == "compact":                                         # every other sequence continues the first half of the one before it
            for b in range(1, B, 2):
                half = up(min(lens[b - 1], lens[b])) // 2
                s["tables0"][b, :half] = s["tables0"][b - 1, :half]
        else:
            pool += 2 * B * (1 + up(case["add"]))
            s["parents"] = torch.tensor(_parents(case), device=dev)
            s["starts"] = case["add"] * torch.arange(B + 1, dtype=torch.int32, device=dev)
            s["slots"] = torch.zeros((B * case["add"],), dtype=torch.int64, device=dev)
        s["pool"] = pool
        s["lengths0"] = torch.tensor(lens, dtype=torch.int32, device=dev)
        s["tables"] = torch.zeros((B, s["tables0"].shape[1]), dtype=torch.int32, device=dev)
        s["lengths"] = torch.zeros((B,), dtype=torch.int32, device=dev)
        s["codes"] = torch.randint(0, 256, (pool * page, 2 * G, M), generator=g, device=dev, dtype=torch.uint8)
        s["scale"] = torch.rand((pool * page, 2 * G), generator=g, device=dev) if case["scaled"] else None
        n = B if op == "extend" else pool // 2
        s["src"], s["dst"] = (torch.zeros((n,), dtype=torch.int32, device=dev) for _ in range(2))
        s["rows"] = torch.zeros((n,), dtype=torch.int32, device=dev) if op == "extend" else None
        s["used"] = torch.zeros((1,), dtype=torch.int32, device=dev)
    if own:
        from paper_1509_05194_amd import hclae
        if op in ("attend", "select"):
            s["ctx"] = hclae.Context(case["B"], case["D"], M, case["K"])
            s["ctx"].cache_begin(s["C"])
        else:                                                       # pages are moved whatever the dictionaries are
            s["ctx"] = hclae.Context(case["B"] * case.get("add", 1), 4, M, 1)
            s["ctx"].cache_begin(torch.zeros((2 * G, M, 1, 4), device=dev))
    return s


# ---- the calls, and their plain forms -------------------------------------------------------------------------------------

def run(s):
    return _RUN[s["case"]["op"]](s)


def _decode(C, ids, heads):
    """Sums of codewords: ids [n][heads][M] of the heads of C."""
    x = C[heads, 0, ids[:, :, 0]]
    for m in range(1, C.shape[1]):
        x = x + C[heads, m, ids[:, :, m]]
    return x


def _run_attend(s):
    c, Q, C, codes, scale, out = s["case"], s["Q"], s["C"], s["codes"], s["scale"], s["out"]
    G, R, D, page = c["G"], c["R"], c["D"], c["page"]
    factor = 1.0 / math.sqrt(D)
    if own:
        s["ctx"].cache_attend(Q, codes, scale, s["tables"], s["lengths"], page, out, factor=factor, picked=s["picked"])
        return out
    heads = torch.arange(G, device=Q.device)
    for b in range(c["B"]):
        n = s["lengths"][b]
        if s["picked"] is None:
            t = torch.arange(s["tables"].shape[1] * page, device=Q.device)[:, None].expand(-1, G)
            t = t[:c["n"]]
        else:
            t = (s["picked"][b].long()[:, :, None] * page + torch.arange(page, device=Q.device)).reshape(G, -1).T
        there = (t >= 0) & (t < n)
        t = t.clamp(min=0, max=s["tables"].shape[1] * page - 1)
        slot = s["tables"][b].long()[t // page] * page + t % page       # [n][G]
        k = _decode(C, codes[slot, heads].long(), heads)
        v = _decode(C, codes[slot, heads + G].long(), heads + G)
        if scale is not None:
            k = k * scale[slot, heads][:, :, None]
            v = v * scale[slot, heads + G][:, :, None]
        q = Q[b].float().reshape(G, R, D)
        x = factor * torch.bmm(q, k.permute(1, 2, 0).contiguous())      # [G][R][n]
        x = torch.where(there.T[:, None, :], x, -math.inf)
        top = x.amax(2, keepdim=True)
        p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
        total = p.sum(2, keepdim=True)
        y = torch.bmm(p, v.transpose(0, 1).contiguous()) / torch.where(total == 0, 1.0, total)
        out[b] = y.reshape(G * R, D).to(out.dtype)
    return out


def _run_select(s):
    c, Q, C, codes, scale = s["case"], s["Q"], s["C"], s["codes"], s["scale"]
    G, R, D, M, page, k = c["G"], c["R"], c["D"], c["M"], c["page"], c["picks"]
    if own:
        s["ctx"].cache_select(Q, codes, scale, s["tables"], s["lengths"], page, s["picked"], first=1 if k > 1 else 0, recent=1)
        return s["picked"]
    heads = torch.arange(G, device=Q.device)
    first = 1 if k > 1 else 0
    for b in range(c["B"]):
        j = torch.arange(s["tables"].shape[1], device=Q.device)
        P = (s["lengths"][b] + page - 1) // page
        q = Q[b].double().reshape(G, R, D).sum(1)
        T = torch.bmm(C.double().reshape(G, -1, D), q[:, :, None]).reshape(G, M, -1)      # in 64 bits: which page is better
        ids = codes[s["tables"][b].long()].long()                        # [pages][G][M]
        x = T[heads, 0, ids[:, :, 0]]
        for m in range(1, M):
            x = x + T[heads, m, ids[:, :, m]]
        if scale is not None:
            x = x * scale[s["tables"][b].long()].double()
        x = torch.where(((j < first) | (j >= P - 1))[:, None], math.inf, x)
        x = torch.where((j >= P)[:, None], -math.inf, x)
        best = torch.sort(x, dim=0, descending=True, stable=True).indices[:k]             # the lowest index of equals first
        best = torch.where(best < P, best, 2 ** 30).sort(0).values
        s["picked"][b] = -1
        s["picked"][b, :, :best.shape[0]] = torch.where(best == 2 ** 30, -1, best).T.int()
    return s["picked"]


def _use(tables, lengths, page, pool):
    """How many entries of the tables name each page, and which entries do."""
    j = torch.arange(tables.shape[1], device=tables.device)
    live = j[None] < ((lengths + page - 1) // page)[:, None]
    used = torch.zeros((pool + 1,), dtype=torch.int64, device=tables.device)
    used.index_add_(0, torch.where(live, tables, pool).long().flatten(), torch.ones_like(tables, dtype=torch.int64).flatten())
    return used[:pool], live


def _copy(s, src, dst, rows):
    """Rows of pages copied: entries with a negative source copy nothing."""
    page = s["case"]["page"]
    codes, scale = s["codes"], s["scale"]
    i = torch.nonzero(src >= 0).flatten()
    off = torch.arange(page, device=src.device)
    fr, to = (src[i].long()[:, None] * page + off).flatten(), (dst[i].long()[:, None] * page + off).flatten()
    if rows is not None:
        keep = (off[None] < rows[i][:, None]).flatten()
        fr, to = fr[keep], to[keep]
    codes[to] = codes[fr]
    if scale is not None:
        scale[to] = scale[fr]


def _run_extend(s):
    c = s["case"]
    page, pool, tables, lengths, starts = c["page"], s["pool"], s["tables"], s["lengths"], s["starts"]
    src, dst, rows, slots = s["src"], s["dst"], s["rows"], s["slots"]
    # the fork: a hypothesis continues a row of the tables; a step that is taken back sets the lengths back
    if c.get("forks"):
        torch.index_select(s["tables0"], 0, s["parents"], out=tables)
        torch.index_select(s["lengths0"], 0, s["parents"], out=lengths)
    else:
        tables.copy_(s["tables0"])
        lengths.copy_(s["lengths0"])
    outs = [tables, lengths, slots, src, dst, rows, s["codes"]] + ([s["scale"]] if s["scale"] is not None else [])
    if own:
        s["ctx"].cache_extend(tables, lengths, starts, page, pool, slots, src, dst, rows)
        s["ctx"].cache_copy(s["codes"], s["scale"], page, src, dst, rows)
        return outs
    B, most = tables.shape
    used, _ = _use(tables, lengths, page, pool)
    add = (starts[1:] - starts[:-1]).clamp(min=0)
    old, new = (lengths + page - 1) // page, (lengths + add + page - 1) // page
    last = (lengths // page).clamp(max=most - 1).long()
    at = tables.gather(1, last[:, None])[:, 0]
    copy = (add > 0) & (lengths % page > 0) & (used[at.clamp(min=0, max=pool - 1).long()] > 1)
    need = torch.where(new <= most, new - old + copy, 0)
    upto = need.cumsum(0)
    free = torch.nonzero(used == 0).flatten()
    ok = (add > 0) & (new <= most) & ((need == 0) | (upto <= free.shape[0]))
    free = torch.nn.functional.pad(free, (0, 1))
    begin = upto - need
    take = lambda i: free[i.clamp(min=0, max=free.shape[0] - 1)].int()
    copy = copy & ok
    dst.copy_(torch.where(copy, take(begin), -1))
    src.copy_(torch.where(copy, at, -1))
    rows.copy_(torch.where(copy, lengths % page, 0))
    j = torch.arange(most, device=tables.device)[None]
    fresh = ok[:, None] & (j >= old[:, None]) & (j < new[:, None])
    tables.copy_(torch.where(fresh, take(begin[:, None] + copy[:, None] + j - old[:, None]), tables))
    tables.copy_(torch.where(copy[:, None] & (j == last[:, None]), dst[:, None], tables))
    t = torch.arange(slots.shape[0], device=tables.device, dtype=torch.int32)
    b = (torch.searchsorted(starts, t, right=True) - 1).clamp(min=0, max=B - 1)
    pos = lengths[b] + t - starts[b]
    p = tables[b, (pos // page).clamp(max=most - 1).long()].long()
    slots.copy_(torch.where(ok[b], p * page + pos % page, -1))
    lengths.add_(torch.where(ok, add, 0))
    _copy(s, src, dst, rows)
    return outs


def _run_compact(s):
    c = s["case"]
    page, pool, tables, lengths, src, dst = c["page"], s["pool"], s["tables"], s["lengths"], s["src"], s["dst"]
    tables.copy_(s["tables0"])                                       # the tables as the last steps left them
    lengths.copy_(s["lengths0"])
    outs = [tables, src, dst, s["used"], s["codes"]] + ([s["scale"]] if s["scale"] is not None else [])
    if own:
        s["ctx"].cache_compact(tables, lengths, page, pool, src, dst, s["used"])
        s["ctx"].cache_copy(s["codes"], s["scale"], page, src, dst)
        return outs
    used, live = _use(tables, lengths, page, pool)
    n = (used > 0).sum()
    p = torch.arange(pool, device=tables.device)
    to = torch.nonzero((used == 0) & (p < n)).flatten()
    fr = torch.nonzero((used > 0) & (p >= n)).flatten()
    src.fill_(-1)
    dst.fill_(-1)
    src[:fr.shape[0]] = fr.int()
    dst[:to.shape[0]] = to.int()
    where = p.clone()
    where[fr] = to
    tables.copy_(torch.where(live, where[torch.where(live, tables, 0).long()].int(), tables))
    s["used"].copy_(n)
    _copy(s, src, dst, None)
    return outs


_RUN = {"attend": _run_attend, "select": _run_select, "extend": _run_extend, "compact": _run_compact}


def work(case):
    """Every input read and every output written once; of the dictionaries the codewords that a call can need at most."""
    G, M, page = case["G"], case["M"], case["page"]
    row = M + (4 if case["scaled"] else 0)
    lens = _lengths(case)
    pages = sum((x + page - 1) // page for x in lens)
    if case["op"] in ("attend", "select"):
        B, R, D, K = case["B"], case["R"], case["D"], case["K"]
        e = 4 if case["type"] == "fp32" else 2
        if case["op"] == "select":
            return {"bytes": pages * G * row + 4 * pages + B * G * R * D * e + 4 * B * G * case["picks"] + 4 * G * M * K * D, "flops": 2 * B * G * M * K * D + pages * G * M}
        rows = [min(x, case["picks"] * page) for x in lens] if case["picks"] else lens
        n = sum(rows)
        words = 8 * G * M * min(K, n) * D
        return {"bytes": n * 2 * G * row + 4 * (sum((x + page - 1) // page for x in rows) + B) + 2 * B * G * R * D * e + words,
                "flops": 4 * n * G * R * M + sum(4 * G * R * M * min(K, x) * D for x in rows)}
    if case["op"] == "extend":
        parents, add = _parents(case), case["add"]
        shared = [p for p in parents if parents.count(p) > 1 and lens[p] % page]
        entries = sum((lens[p] + page - 1) // page for p in parents)
        return {"bytes": 4 * entries + 16 * case["B"] + 8 * case["B"] * add + sum(2 * (lens[p] % page) * 2 * G * row for p in shared), "flops": entries}
    return {"bytes": 8 * pages + pages * page * 2 * G * row, "flops": pages}     # about half of the pages move: each read and written


# ---- the same in 64 bits --------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    page = case["page"]
    if case["op"] == "attend":
        G, R, D = case["G"], case["R"], case["D"]
        out = s["out"].double()
        C = s["C"].double()
        for b, n in enumerate(s["lengths"].tolist()):
            for h in range(G):
                if s["picked"] is None:
                    t = torch.arange(n, device=out.device)
                else:
                    j = s["picked"][b, h]
                    t = torch.cat([torch.arange(x * page, min(n, (x + 1) * page), device=out.device) for x in j[j >= 0].tolist()] + [torch.zeros(0, dtype=torch.int64, device=out.device)])
                if len(t) == 0:
                    continue
                slot = s["tables"][b].long()[t // page] * page + t % page
                k = torch.zeros((len(t), D), dtype=torch.float64, device=out.device)
                v = torch.zeros_like(k)
                for m in range(case["M"]):
                    k += C[h, m].index_select(0, s["codes"][slot, h, m].long())
                    v += C[h + G, m].index_select(0, s["codes"][slot, h + G, m].long())
                if case["scaled"]:
                    k *= s["scale"][slot, h].double()[:, None]
                    v *= s["scale"][slot, h + G].double()[:, None]
                q = s["Q"][b, h * R:(h + 1) * R].double()
                p = torch.softmax(q @ k.T / math.sqrt(D), 1)
                out[b, h * R:(h + 1) * R] = p @ v
        return out
    if case["op"] == "select":
        G, R, D, k = case["G"], case["R"], case["D"], case["picks"]
        C = s["C"].double()
        picked = torch.full_like(s["picked"], -1)
        for b, n in enumerate(s["lengths"].tolist()):
            P = (n + page - 1) // page
            own_pages = s["tables"][b, :P].long()
            for h in range(G):
                q = s["Q"][b, h * R:(h + 1) * R].double().sum(0)
                x = torch.zeros((P, D), dtype=torch.float64, device=C.device)
                for m in range(case["M"]):
                    x += C[h, m].index_select(0, s["codes"][own_pages, h, m].long())
                if case["scaled"]:
                    x *= s["scale"][own_pages, h].double()[:, None]
                score = (x * q).sum(1).tolist()
                keep = sorted(range(P), key=lambda j: (not ((j == 0 and k > 1) or j == P - 1), -score[j], j))[:k]
                picked[b, h, :len(keep)] = torch.tensor(sorted(keep), dtype=torch.int32, device=C.device)
        return picked
    codes, scale = s["codes"], s["scale"]
    lens = _lengths(case)
    pool, rows_of = s["pool"], s["tables0"].tolist()
    up = lambda x: (x + page - 1) // page
    if case["op"] == "extend":
        parents = _parents(case)
        rows_of, lens = [list(rows_of[p]) for p in parents], [lens[p] for p in parents]
        users = {}
        for r, n in zip(rows_of, lens):
            for p in r[:up(n)]:
                users[p] = users.get(p, 0) + 1
        free = [p for p in range(pool) if p not in users]
        slots, moves = [], []
        add, most, asked = case["add"], len(rows_of[0]), 0
        for b, (r, n) in enumerate(zip(rows_of, lens)):
            split = n % page > 0 and users[r[n // page]] > 1
            need = up(n + add) - up(n) + split
            if up(n + add) > most:
                slots += [-1] * add
                moves.append((-1, -1, 0))
                continue
            asked += need
            if need and asked > len(free):
                slots += [-1] * add
                moves.append((-1, -1, 0))
                continue
            mine = free[asked - need:asked]
            if split:
                moves.append((r[n // page], mine[0], n % page))
                r[n // page] = mine.pop(0)
            else:
                moves.append((-1, -1, 0))
            for j in range(up(n), up(n + add)):
                r[j] = mine.pop(0)
            slots += [r[t // page] * page + t % page for t in range(n, n + add)]
            lens[b] = n + add
        for a, d, k in moves:
            if a >= 0:
                codes[d * page:d * page + k] = codes[a * page:a * page + k]
                if scale is not None:
                    scale[d * page:d * page + k] = scale[a * page:a * page + k]
        whole = lambda x, like: torch.tensor(x, dtype=like.dtype, device=like.device)
        outs = [whole(rows_of, s["tables"]), whole(lens, s["lengths"]), whole(slots, s["slots"])]
        outs += [whole([m[i] for m in moves], s["src"]) for i in range(3)]
        return outs + [codes] + ([scale] if scale is not None else [])
    in_use = sorted({p for r, n in zip(rows_of, lens) for p in r[:up(n)]})
    n = len(in_use)
    there = set(in_use)
    holes = [p for p in range(n) if p not in there]
    movers = [p for p in in_use if p >= n]
    to = dict(zip(movers, holes))
    for r, x in zip(rows_of, lens):
        r[:up(x)] = [to.get(p, p) for p in r[:up(x)]]
    for a, d in to.items():
        codes[d * page:(d + 1) * page] = codes[a * page:(a + 1) * page]
        if scale is not None:
            scale[d * page:(d + 1) * page] = scale[a * page:(a + 1) * page]
    pad = [-1] * (len(s["src"]) - len(movers))
    whole = lambda x, like: torch.tensor(x, dtype=like.dtype, device=like.device)
    return [whole(rows_of, s["tables"]), whole(movers + pad, s["src"]), whole(holes + pad, s["dst"]), whole([n], s["used"]), codes] + ([scale] if scale is not None else [])
