"""The operators that write and read vectors as codes of additive dictionaries inside a language model, as measurable cases.

  write   Context.cache_write: the rows of H heads, as a layer hands them over, quantised into the slots of a paged cache
  read    Context.cache_read: the cached rows of a batch of sequences read back through their page tables
  lookup  Context.lookup: rows of a table that is kept as codes, scaled; without row numbers, the decoding of all of it
  grad    Context.lookup_grad: the gradient of a lookup with respect to the dictionaries

D = 128, M = 8 or 16 and K = 256 are the 64- and 128-bit codes of the repository's benchmark, D = 960 its long rows, D = 4096 the
longest rows the library takes, a million rows its base set; head counts, sequence lengths and pages are generic.
"""
import math

import torch

own = False


def listed():
    return [
        # one step of one sequence: keys and values of eight heads; latency is all there is
        {"name": "write_token", "op": "write", "n": 1, "H": 16, "D": 128, "M": 8, "K": 256, "page": 16, "type": "bf16", "scaled": True},
        # one step of a batch of sequences, with the better codes
        {"name": "write_batch", "op": "write", "n": 64, "H": 16, "D": 128, "M": 16, "K": 256, "page": 16, "type": "fp16", "scaled": True},
        # a chunk of a prompt with an odd head size and small dictionaries, rows quantised as they are
        {"name": "write_odd", "op": "write", "n": 1237, "H": 5, "D": 80, "M": 5, "K": 200, "page": 24, "type": "fp32", "scaled": False},
        # a whole prompt
        {"name": "write_prompt", "op": "write", "n": 8192, "H": 16, "D": 128, "M": 8, "K": 256, "page": 64, "type": "bf16", "scaled": True},
        # a few short sequences
        {"name": "read_short", "op": "read", "n": 150, "B": 4, "H": 16, "D": 128, "M": 8, "K": 256, "page": 16, "type": "bf16", "scaled": True},
        # long rows of few heads, better codes, odd lengths
        {"name": "read_odd", "op": "read", "n": 5003, "B": 7, "H": 3, "D": 192, "M": 16, "K": 256, "page": 24, "type": "fp32", "scaled": False},
        # a batch of long contexts
        {"name": "read_long", "op": "read", "n": 32768, "B": 9, "H": 16, "D": 128, "M": 8, "K": 256, "page": 64, "type": "bf16", "scaled": True},
        # the embeddings of one step of a batch
        {"name": "lookup_step", "op": "lookup", "T": 64, "V": 100003, "D": 4096, "M": 8, "K": 256, "type": "bf16", "all": False},
        # the embeddings of a training batch
        {"name": "lookup_batch", "op": "lookup", "T": 16384, "V": 100003, "D": 4096, "M": 8, "K": 256, "type": "bf16", "all": False},
        # a base set of a million 64-bit codes decoded
        {"name": "decode_base", "op": "lookup", "T": 1000000, "V": 1000000, "D": 128, "M": 8, "K": 256, "type": "fp32", "all": True},
        # the gradient of a short batch of long rows, an odd count
        {"name": "grad_short", "op": "grad", "T": 509, "V": 20011, "D": 960, "M": 8, "K": 256, "type": "fp32", "all": False},
        # the gradient of a training batch: frequent rows come thousands of times
        {"name": "grad_batch", "op": "grad", "T": 16384, "V": 100003, "D": 4096, "M": 8, "K": 256, "type": "bf16", "all": False},
    ]


def _between(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["write", "write", "read", "read", "lookup", "lookup", "grad", "grad"])
    case = {"op": op, "type": rng.choice(["bf16", "bf16", "fp16", "fp32"])}
    M = rng.choice([8, 8, 16, _between(rng, 1, 16)])
    K = rng.choice([256, 256, _between(rng, 16, 256)])
    if op in ("write", "read"):
        D = rng.choice([64, 128, 128, 4 * _between(rng, 8, 64)])
        H = rng.choice([1, 2, 8, 16, _between(rng, 1, 16)])
        most = 8192 * 16 * 8 * 256 * 128 // (H * M * max(K, 64) * D) if op == "write" else 32768 * 16 * 8 * 128 // (H * max(M, 8) * D)
        n = _between(rng, 1, min(most, 8192 if op == "write" else 32768))
        case.update(n=n, H=H, D=D, M=M, K=K, page=rng.choice([1, 16, 24, 64, 256]), scaled=rng.random() < 0.75)
        if op == "read":
            case["B"] = _between(rng, 1, max(1, min(64, n)))
        return case
    D = rng.choice([128, 960, 4096, 4 * _between(rng, 16, 1024)])
    most = (128 << 20) if op == "lookup" else (64 << 20)
    T = _between(rng, 1, min(1000000, most * 8 // (max(M, 8) * D)))
    case.update(T=T, D=D, M=M, K=K, all=rng.random() < 0.25)
    case["V"] = T if case["all"] else _between(rng, 1000, 200000)
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------------------

_TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def _head_rows(n, H, D, g, shape):
    """Rows as keys and values have them: a few directions carry most of it, channels of different size, some far off zero."""
    basis, size, offset = shape
    z = torch.randn((H, n, basis.shape[1]), generator=g, device=basis.device)
    x = torch.bmm(z, basis) + 0.5 * torch.randn((H, n, D), generator=g, device=basis.device)
    return (x * size + offset).transpose(0, 1)                       # [n][H][D]


def _head_shape(H, D, g, dev):
    basis = torch.randn((H, 12, D), generator=g, device=dev) / 4
    size = torch.exp(0.4 * torch.randn((H, 1, D), generator=g, device=dev))
    offset = 2.0 * torch.randn((H, 1, D), generator=g, device=dev) * (torch.rand((H, 1, D), generator=g, device=dev) < 0.05)
    return basis, size, offset


def _head_dictionaries(H, M, K, D, g, shape, scaled):
    """M dictionaries a head, each from what the ones before it leave of a sample of rows."""
    x = _head_rows(2 * K + 64, H, D, g, shape).transpose(0, 1).contiguous()
    if scaled:
        x = x / x.abs().amax(2, keepdim=True)
    C = torch.empty((H, M, K, D), device=x.device)
    for m in range(M):
        pick = torch.randperm(x.shape[1], generator=g, device=x.device)[:K]
        c = 0.9 * x[:, pick] + 0.1 * x.std() * torch.randn((H, K, D), generator=g, device=x.device)
        C[:, m] = c
        s = torch.bmm(x, c.transpose(1, 2).contiguous()) - 0.5 * (c * c).sum(2)[:, None]
        x = x - c.gather(1, s.argmax(2)[:, :, None].expand(-1, -1, D))
    return C


def _pages(n_tokens, page, g, dev):
    """Page numbers for the tokens of one sequence after another, scattered over a pool that has a quarter more; and the pool's size."""
    need = sum((n + page - 1) // page for n in n_tokens)
    pool = need + need // 4 + 1
    return torch.randperm(pool, generator=g, device=dev)[:need], pool


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    D, M, K, dt = case["D"], case["M"], case["K"], _TYPES[case["type"]]
    s = {"case": case}
    if case["op"] in ("write", "read"):
        n, H, page = case["n"], case["H"], case["page"]
        shape = _head_shape(H, D, g, dev)
        C = _head_dictionaries(H, M, K, D, g, shape, case["scaled"])
    if case["op"] == "write":
        # the rows lie in the output of a larger projection, as many columns again beside them
        wide = torch.zeros((n, 2 * H, D), dtype=dt, device=dev)
        wide[:, :H] = _head_rows(n, H, D, g, shape).to(dt)
        pages, pool = _pages([n], page, g, dev)
        t = torch.arange(n, device=dev)
        slots = pages[t // page] * page + t % page
        slots[torch.rand((n,), generator=g, device=dev) < 0.03] = -1    # padding of the batch
        s.update(C=C, X=wide[:, :H], slots=slots, n_slots=pool * page)
        # one slot more than the cache has, for what is not kept
        s["codes"] = torch.zeros((pool * page + 1, H, M), dtype=torch.uint8, device=dev)
        s["scale"] = torch.zeros((pool * page + 1, H), device=dev) if case["scaled"] else None
    elif case["op"] == "read":
        B = case["B"]
        cut = torch.sort(torch.randint(0, n + 1, (B - 1,), generator=g, device=dev)).values.tolist()
        ends = cut + [n]
        lens = [e - b for b, e in zip([0] + cut, ends)]
        pages, pool = _pages(lens, page, g, dev)
        tables = torch.zeros((B, max((x + page - 1) // page for x in lens)), dtype=torch.int32, device=dev)
        at = 0
        for b, x in enumerate(lens):
            p = (x + page - 1) // page
            tables[b, :p] = pages[at:at + p].int()
            at += p
        s.update(C=C, tables=tables, starts=torch.tensor([0] + ends, dtype=torch.int32, device=dev))
        s["codes"] = torch.randint(0, K, (pool * page, H, M), generator=g, device=dev, dtype=torch.uint8)
        s["scale"] = torch.exp(torch.randn((pool * page, H), generator=g, device=dev)) if case["scaled"] else None
        s["out"] = torch.zeros((n + 5, H, D), dtype=dt, device=dev)      # a few rows more than the sequences have
    else:
        T, V = case["T"], case["V"]
        fall = 0.7 ** torch.arange(M, device=dev)[:, None, None]
        s["C"] = 0.02 * fall * torch.randn((M, K, D), generator=g, device=dev)
        s["codes"] = torch.randint(0, K, (V, M), generator=g, device=dev, dtype=torch.uint8)
        s["rows"] = None
        s["a"] = math.sqrt(D) if not case["all"] else 1.0
        if not case["all"]:                                             # row r about as often as 1 / (r + 1), some padding
            r = torch.exp(torch.rand((T,), generator=g, device=dev, dtype=torch.float64) * math.log(V)).long().clamp_(1, V) - 1
            r[torch.rand((T,), generator=g, device=dev) < 0.01] = -1
            s["rows"] = r
        if case["op"] == "lookup":
            s["out"] = torch.zeros((T, D), dtype=dt, device=dev)
        else:
            s["dout"] = (torch.randn((T, D), generator=g, device=dev) / T).to(dt) if dt != torch.float16 else torch.randn((T, D), generator=g, device=dev).to(dt)
            s["dC"] = torch.zeros((M, K, D), device=dev)
    if own:
        from paper_1509_05194_amd import hclae
        s["ctx"] = hclae.Context(case["n"] + 5 if "n" in case else case["T"], D, M, K)
        if case["op"] in ("write", "read"):
            s["ctx"].cache_begin(s["C"])
    return s


# ---- the calls, and their plain forms -------------------------------------------------------------------------------------

def run(s):
    return _RUN[s["case"]["op"]](s)


def _run_write(s):
    X, C, slots, n_slots = s["X"], s["C"], s["slots"], s["n_slots"]
    codes, scale = s["codes"][:n_slots], s["scale"][:n_slots] if s["scale"] is not None else None
    if own:
        s["ctx"].cache_write(X, slots, codes, scale)
        return (codes, scale) if scale is not None else codes
    H, M, _, D = C.shape
    r = X.transpose(0, 1).float()                                    # [H][n][D]
    to = torch.where(slots < 0, n_slots, slots)
    if scale is not None:
        top = r.abs().amax(2)
        r = torch.where(top[:, :, None] > 0, r / top[:, :, None], 0.0)
        s["scale"][to] = top.T
    ids = torch.empty((H, r.shape[1], M), dtype=torch.uint8, device=r.device)
    for m in range(M):                                               # which codeword is nearest: in 64 bits
        c = C[:, m].double()
        d = (c * c).sum(2)[:, None] - 2 * torch.bmm(r.double(), c.transpose(1, 2).contiguous())
        k = d.argmin(2)
        ids[:, :, m] = k.to(torch.uint8)
        r = r - C[:, m].gather(1, k[:, :, None].expand(-1, -1, D))
    s["codes"][to] = ids.transpose(0, 1)
    return (codes, scale) if scale is not None else codes


def _run_read(s):
    out, C, tables, starts, page = s["out"], s["C"], s["tables"], s["starts"], s["case"]["page"]
    if own:
        s["ctx"].cache_read(s["codes"], s["scale"], tables, starts, page, out)
        return out
    slot = _slots_of(tables, starts, page, s["case"]["n"])
    ids = s["codes"][slot].long()                                    # [n][H][M]
    heads = torch.arange(C.shape[0], device=out.device)
    x = C[heads, 0, ids[:, :, 0]]
    for m in range(1, C.shape[1]):
        x = x + C[heads, m, ids[:, :, m]]
    if s["scale"] is not None:
        x = x * s["scale"][slot][:, :, None]
    out[:x.shape[0]] = x.to(out.dtype)
    return out


def _slots_of(tables, starts, page, n):
    t = torch.arange(n, device=tables.device, dtype=torch.int32)
    b = torch.searchsorted(starts, t, right=True) - 1
    pos = t - starts[b]
    return tables[b, (pos // page).long()].long() * page + pos % page


def _run_lookup(s):
    C, codes, rows, out, a = s["C"], s["codes"], s["rows"], s["out"], s["a"]
    if own:
        s["ctx"].lookup(codes, C, out, rows=rows, scale=a)
        return out
    ids = codes.long() if rows is None else codes[rows.clamp(min=0)].long()
    x = C[0][ids[:, 0]]
    for m in range(1, C.shape[0]):
        x = x + C[m][ids[:, m]]
    x = x * a
    if rows is not None:
        x = torch.where(rows[:, None] < 0, 0.0, x)
    return x.to(out.dtype)


def _run_grad(s):
    codes, rows, dout, dC, a = s["codes"], s["rows"], s["dout"], s["dC"], s["a"]
    if own:
        s["ctx"].lookup_grad(codes, dout, dC, rows=rows, scale=a)
        return dC
    ids = codes.long() if rows is None else codes[rows.clamp(min=0)].long()
    x = dout.float() * a
    if rows is not None:
        x = torch.where(rows[:, None] < 0, 0.0, x)
    d = torch.zeros_like(dC)
    for m in range(dC.shape[0]):
        d[m].index_add_(0, ids[:, m], x)
    return d


_RUN = {"write": _run_write, "read": _run_read, "lookup": _run_lookup, "grad": _run_grad}


def work(case):
    """Every input read and every output written once, of the dictionaries the codewords that a call can need at most."""
    D, M, K = case["D"], case["M"], case["K"]
    e = 4 if case["type"] == "fp32" else 2
    if case["op"] == "write":
        n, H = case["n"], case["H"]
        return {"bytes": n * H * (D * e + M + (4 if case["scaled"] else 0)) + 8 * n + 4 * H * M * K * D, "flops": 2 * n * H * M * K * D}
    if case["op"] == "read":
        n, H = case["n"], case["H"]
        words = 4 * H * M * min(K, n) * D
        return {"bytes": n * H * (D * e + M + (4 if case["scaled"] else 0)) + 4 * (n // case["page"] + case["B"]) + words, "flops": n * H * M * D}
    T = case["T"]
    small = T * (D * e + M + (0 if case["all"] else 8))
    words = 4 * M * (min(K, T) if case["op"] == "lookup" else K) * D
    return {"bytes": small + words, "flops": T * M * D}


# ---- the same in 64 bits --------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    C = s["C"].double()
    if case["op"] == "write":
        # rows are held in 32 bits from one dictionary to the next: so the operator is defined; every distance in 64
        X, slots, n_slots = s["X"], s["slots"], s["n_slots"]
        if case["n"] * case["H"] * case["M"] * case["K"] * case["D"] > 2 ** 36:
            return None
        codes = s["codes"][:n_slots].clone()
        scale = s["scale"][:n_slots].double() if case["scaled"] else None
        live = torch.nonzero(slots >= 0).flatten()
        step = max(1, (1 << 25) // (case["K"] * case["D"]))
        for h in range(case["H"]):
            for at in live.split(step):
                r = X[at, h].float()
                if scale is not None:
                    top = r.abs().amax(1, keepdim=True)
                    scale[slots[at], h] = top[:, 0].double()
                    r = torch.where(top > 0, r / top, torch.zeros_like(r))
                for m in range(case["M"]):
                    k = ((r.double()[:, None] - C[h, m][None]) ** 2).sum(2).min(1).indices
                    codes[slots[at], h, m] = k.to(torch.uint8)
                    r = r - s["C"][h, m][k]
        return (codes, scale) if scale is not None else codes
    if case["op"] == "read":
        out = s["out"].double()
        at = 0
        starts, tables, page = s["starts"].tolist(), s["tables"].long(), case["page"]
        for b in range(case["B"]):
            t = torch.arange(starts[b + 1] - starts[b], device=out.device)
            slot = tables[b][t // page] * page + t % page
            for h in range(case["H"]):
                x = torch.zeros((len(t), case["D"]), dtype=torch.float64, device=out.device)
                for m in range(case["M"]):
                    x += C[h, m].index_select(0, s["codes"][slot, h, m].long())
                out[at:at + len(t), h] = x * (s["scale"][slot, h].double()[:, None] if case["scaled"] else 1.0)
            at += len(t)
        return out
    rows = s["rows"] if s["rows"] is not None else torch.arange(case["T"], device=C.device)
    live = torch.nonzero(rows >= 0).flatten()
    ids = s["codes"].index_select(0, rows[live]).long()
    if case["op"] == "lookup":
        out = torch.zeros((case["T"], case["D"]), dtype=torch.float64, device=C.device)
        for m in range(case["M"]):
            out.index_add_(0, live, C[m].index_select(0, ids[:, m]))
        return out.mul_(s["a"])
    d = torch.zeros_like(C)
    x = s["dout"].double().index_select(0, live)
    for m in range(case["M"]):
        d[m].index_add_(0, ids[:, m], x)
    return d.mul_(s["a"])
