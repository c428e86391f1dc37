"""Coded caches and coded tables (hclae_cache_begin / write / read, hclae_lookup, hclae_lookup_grad) against plain 64-bit forms.

Tolerances: a decoded element is a sum of M fp32 values in some order, times one or two factors, rounded once to its type: off by at
most (M + 3) 2^-24 sum |c_m| |factor| and half a step of the type.  An element of a gradient is a sum of n values: (n + 2) 2^-24 of
the sum of their magnitudes.  Codes are decisions on rows that are held in fp32 by definition, in 64 bits: equal."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
U32 = 2.0 ** -24


def half_step(t):
    """Half a step of a type, relative, and the same of its smallest numbers."""
    return torch.finfo(t).eps / 2, torch.finfo(t).tiny * torch.finfo(t).eps / 2


def quantise(x, C, scaled):
    """codes [n][M] and scales [n] of the fp32 rows x of one head: rows in fp32, distances in 64 bits."""
    with np.errstate(all="ignore"):
        g = np.abs(x).max(1)
        bad = ~np.isfinite(x).all(1)
        g = np.where(bad, np.float32(np.nan), g)
        r = np.where(bad[:, None], np.float32(0), x)
        if scaled:
            r = np.where((g > 0)[:, None] & ~bad[:, None], r / g[:, None], r).astype(np.float32)
    codes = np.zeros((len(x), C.shape[0]), np.uint8)
    for m in range(C.shape[0]):
        c = C[m].astype(np.float64)
        for i in range(len(r)):
            k = int(((r[i].astype(np.float64) - c) ** 2).sum(1).argmin())
            codes[i, m] = k
            r[i] = r[i] - C[m][k]
    return codes, g


def heads(n, H, D, M, K, seed, spread=1.0):
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((n, H, D)) * spread).astype(np.float32)
    C = np.stack([np.stack([rng.standard_normal((K, D)) * spread * 0.5 ** (m + 1) for m in range(M)]) for _ in range(H)]).astype(np.float32)
    return x, C


def placed(x, layout):
    """The rows [n][H][D] as a view of a larger array."""
    n, H, D = x.shape
    if layout == "tight":
        return x.contiguous()
    if layout == "wide":                                   # beside other columns, as in the output of a projection
        w = torch.full((n, 2 * H + 1, D), 7.0, dtype=x.dtype, device=x.device)
        w[:, H:2 * H] = x
        return w[:, H:2 * H]
    w = torch.full((H, n, D + 4), 7.0, dtype=x.dtype, device=x.device)     # a head after another
    w[:, :, :D] = x.transpose(0, 1)
    return w[:, :, :D].transpose(0, 1)


WRITE = [
    (1, 1, 4, 1, 1, "fp32", True, "tight"), (1, 8, 128, 8, 256, "bf16", True, "wide"), (2, 3, 64, 16, 256, "fp16", True, "heads"),
    (3, 2, 256, 3, 256, "bf16", True, "wide"), (33, 5, 80, 5, 200, "fp32", False, "heads"), (70, 3, 36, 4, 20, "fp16", True, "wide"),
    (130, 2, 132, 2, 130, "bf16", False, "tight"), (300, 1, 128, 4, 256, "bf16", True, "wide"), (65, 4, 192, 2, 64, "fp32", True, "heads"),
    (257, 2, 64, 3, 256, "fp32", False, "wide"), (515, 1, 124, 2, 100, "fp16", True, "heads"), (40, 16, 20, 2, 33, "bf16", True, "tight"),
    # more rows, sixteen a block
    (2100, 1, 64, 2, 20, "bf16", True, "wide"), (1101, 2, 60, 2, 60, "fp16", True, "heads"), (2200, 1, 36, 2, 100, "fp32", False, "tight"),
    (700, 3, 64, 2, 256, "bf16", True, "wide"), (2500, 1, 128, 2, 30, "fp32", True, "tight"), (1200, 2, 100, 2, 64, "bf16", True, "heads"),
    (2300, 1, 128, 2, 128, "fp16", True, "wide"), (3001, 1, 128, 3, 256, "bf16", False, "tight"), (2100, 1, 200, 2, 32, "bf16", True, "wide"),
    (1100, 2, 256, 2, 64, "fp32", False, "heads"), (2100, 1, 160, 2, 120, "fp16", True, "tight"), (700, 4, 256, 2, 256, "bf16", True, "wide"),
    (2089, 1, 196, 2, 201, "fp32", True, "heads"), (2060, 1, 4, 2, 1, "fp32", True, "tight"), (301, 9, 12, 3, 2, "fp32", False, "tight"),
    # more than 4096 rows, in tiles: every size of dictionary (blocks of 32, 64, 128, 256) and row (64, 128, 256)
    (4200, 1, 64, 2, 20, "bf16", True, "wide"), (1403, 3, 60, 2, 60, "fp16", True, "heads"), (4099, 1, 36, 2, 100, "fp32", False, "tight"),
    (1400, 3, 64, 2, 256, "bf16", True, "wide"), (4130, 1, 128, 2, 30, "fp32", True, "tight"), (2103, 2, 100, 2, 64, "bf16", True, "heads"),
    (4150, 1, 128, 2, 128, "fp16", True, "wide"), (1033, 4, 124, 3, 256, "bf16", False, "tight"), (4097, 1, 200, 2, 32, "bf16", True, "wide"),
    (2060, 2, 256, 2, 64, "fp32", False, "heads"), (4111, 1, 160, 2, 120, "fp16", True, "tight"), (1050, 4, 256, 2, 256, "bf16", True, "wide"),
    (4112, 1, 196, 2, 201, "fp32", True, "heads"), (4160, 1, 4, 2, 1, "fp32", True, "tight"), (601, 9, 12, 3, 2, "fp32", False, "tight"),
]


@pytest.mark.parametrize("n,H,D,M,K,kind,scaled,layout", WRITE)
def test_write(n, H, D, M, K, kind, scaled, layout):
    from paper_1509_05194_amd import hclae
    x, C = heads(n, H, D, M, K, n * 7 + D)
    x = torch.from_numpy(x).to(TYPES[kind])
    if n > 2:
        x[1] = 0                                           # padding of a batch
        x[2, 0, D // 2] = float("nan")
    if n > 30:
        x[5, H - 1, 0] = float("inf")
        x[6, :, 1] = -float("inf")
        C[:, :, min(3, K - 1)] = C[:, :, 0]                # equal codewords: the lowest index
        x[7] = torch.from_numpy(C[:, 0, 0]).to(x.dtype)
    n_slots = n + 11
    rng = np.random.default_rng(n)
    slots = rng.permutation(n_slots)[:n].astype(np.int64)
    if n > 30:
        slots[[3, 9, 20]] = [-1, n_slots, 2 ** 40]
    codes = torch.full((n_slots, H, M), 251, dtype=torch.uint8, device="cuda")
    scale = torch.full((n_slots, H), -3.0, device="cuda") if scaled else None
    ctx = hclae.Context(n, D, M, K)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    ctx.cache_write(placed(x.cuda(), layout), torch.from_numpy(slots).cuda(), codes, scale)
    torch.cuda.synchronize()
    want = np.full((n_slots, H, M), 251, np.uint8)
    want_g = np.full((n_slots, H), -3.0, np.float32)
    keep = (slots >= 0) & (slots < n_slots)
    for h in range(H):
        c, g = quantise(x[:, h].float().numpy(), C[h], scaled)
        want[slots[keep], h] = c[keep]
        want_g[slots[keep], h] = g[keep]
    differ = np.argwhere(codes.cpu().numpy() != want)
    assert len(differ) == 0, differ[:5]
    if scaled:
        assert np.array_equal(scale.cpu().numpy(), want_g, equal_nan=True)
    ctx.close()


@pytest.mark.parametrize("spread", [1e-30, 1e-18, 1e15, 1e30])
@pytest.mark.parametrize("n,K,D", [(5, 256, 64), (200, 90, 128), (1100, 256, 128), (1200, 70, 132), (2100, 256, 128), (2080, 70, 132),
                                   (2090, 30, 64)])
def test_write_unusual_magnitudes(spread, n, K, D):
    """Rows quantised as they are, whose squares leave the range of fp32."""
    from paper_1509_05194_amd import hclae
    x, C = heads(n, 2, D, 2, K, 5, spread)
    ctx = hclae.Context(n, D, 2, K)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    codes = torch.zeros((n, 2, 2), dtype=torch.uint8, device="cuda")
    ctx.cache_write(torch.from_numpy(x).cuda(), torch.arange(n, device="cuda"), codes)
    for h in range(2):
        assert np.array_equal(codes[:, h].cpu().numpy(), quantise(x[:, h].copy(), C[h], False)[0])
    ctx.close()


@pytest.mark.parametrize("n,K,D,what", [(1500, 256, 128, "far"), (1500, 256, 128, "equal"), (1100, 200, 64, "zeros"), (1100, 64, 200, "equal"),
                                        (1300, 256, 256, "far"), (2100, 256, 128, "far"), (2070, 256, 128, "equal"), (2100, 200, 64, "zeros"), (2060, 64, 200, "equal"),
                                        (2200, 256, 256, "far"), (60, 256, 128, "far"), (60, 256, 128, "equal"), (60, 70, 64, "zeros")])
def test_write_with_many_near_ties(n, K, D, what):
    """Rows far from the origin compared with what tells them apart, dictionaries of equal codewords, and of zeros."""
    from paper_1509_05194_amd import hclae
    x, C = heads(n, 2, D, 3, K, 8)
    if what == "far":
        x, C[:, 0] = x + np.float32(300), C[:, 0] + np.float32(300)
    elif what == "equal":
        C[:, 1] = C[:, 1, np.random.default_rng(0).integers(0, 5, K)]
    else:
        C[:, 1:] = 0
    ctx = hclae.Context(n, D, 3, K)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    codes = torch.zeros((n, 2, 3), dtype=torch.uint8, device="cuda")
    ctx.cache_write(torch.from_numpy(x).cuda(), torch.arange(n, device="cuda"), codes)
    for h in range(2):
        assert np.array_equal(codes[:, h].cpu().numpy(), quantise(x[:, h].copy(), C[h], False)[0])
    ctx.close()


@pytest.mark.parametrize("D,K", [(64, 20), (60, 60), (36, 100), (64, 256), (128, 30), (100, 64), (128, 128), (124, 255), (200, 32), (256, 64), (160, 120),
                                 (256, 256)])
def test_write_of_very_many_rows_is_that_of_its_parts(D, K):
    """Calls that fill the device with tiles; parts of 500 rows of a head, and a sample of rows in 64 bits."""
    from paper_1509_05194_amd import hclae
    H, M, n = 3, 3, 11333 if D <= 128 else 6007
    x, C = heads(n, H, D, M, K, D + K)
    x[17], x[n - 1, 1, D - 1] = 0, np.nan
    X, slots = torch.from_numpy(x).cuda(), torch.randperm(n, generator=torch.Generator().manual_seed(1)).cuda()
    slots[5] = n
    ctx = hclae.Context(n, D, M, K)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    got, want = (torch.full((n, H, M), 251, dtype=torch.uint8, device="cuda") for _ in range(2))
    g, want_g = (torch.full((n, H), -3.0, device="cuda") for _ in range(2))
    ctx.cache_write(X, slots, got, g)
    for i in range(0, n, 500):
        ctx.cache_write(X[i:i + 500], slots[i:i + 500], want, want_g)
    assert torch.equal(got, want) and torch.equal(g.nan_to_num(-1), want_g.nan_to_num(-1))
    at = np.concatenate([[0, 17, n - 1], np.random.default_rng(0).integers(6, n, 60)])
    for h in range(H):
        codes, scales = quantise(x[at, h].copy(), C[h], True)
        where = slots.cpu().numpy()[at]
        assert np.array_equal(got[:, h].cpu().numpy()[where], codes)
        assert np.array_equal(g[:, h].cpu().numpy()[where], scales, equal_nan=True)
    ctx.close()


def test_write_gives_the_codes_of_the_encoder():
    """One head, no scales: the codes of hclae_encode, whichever kernels took the rows."""
    from paper_1509_05194_amd import hclae
    for n, D, M, K in ((9, 128, 8, 256), (700, 128, 8, 256), (20000, 64, 4, 256), (9000, 128, 3, 100)):
        x, C = heads(n, 1, D, M, K, n)
        X = torch.from_numpy(x[:, 0]).cuda()
        Cg = torch.from_numpy(C).cuda()
        ctx = hclae.Context(n, D, M, K)
        want, r = torch.zeros((n, M), dtype=torch.uint8, device="cuda"), torch.empty_like(X)
        ctx.encode(X, Cg[0], want, r)
        ctx.cache_begin(Cg)
        codes = torch.zeros((n, 1, M), dtype=torch.uint8, device="cuda")
        ctx.cache_write(X[:, None], torch.arange(n, device="cuda"), codes)
        assert torch.equal(codes[:, 0], want), (n, D, M, K, int((codes[:, 0] != want).sum()))
        ctx.close()


def decoded(ids, C, factor):
    """In 64 bits: sum_m C[m][ids[:, m]] * factor, and the sum of magnitudes."""
    s = np.zeros((len(ids), C.shape[2]))
    a = np.zeros_like(s)
    for m in range(C.shape[0]):
        v = C[m][np.minimum(ids[:, m], C.shape[1] - 1)].astype(np.float64)
        s += v
        a += np.abs(v)
    f = np.asarray(factor, np.float64).reshape(-1, 1)
    return s * f, a * np.abs(f)


def close_to(got, want, mag, M, t):
    rel, least = half_step(t)
    tol = (1 + 2.0 ** -8) * (np.abs(want) * rel + (M + 3) * U32 * mag) + least
    off = np.abs(got.double().cpu().numpy() - want)
    bad = ~(off <= tol)
    bad &= ~((np.abs(want) * (1 + rel) >= torch.finfo(t).max) & ~np.isfinite(got.double().cpu().numpy()))
    assert not bad.any(), (np.argwhere(bad)[:3], off[bad][:3], tol[bad][:3])


READ = [
    # lengths, H, D, M, K, page, type, scaled, layout
    ([1], 1, 4, 1, 1, 1, "fp32", True, "tight"), ([5, 0, 7, 1], 3, 128, 8, 256, 16, "bf16", True, "wide"),
    ([100, 33, 0], 2, 80, 5, 200, 24, "fp16", False, "heads"), ([0, 0], 2, 64, 3, 16, 4, "fp32", True, "tight"),
    ([3000, 1, 1500], 4, 128, 8, 256, 64, "bf16", True, "heads"), ([2500], 1, 192, 16, 256, 7, "fp32", False, "wide"),
    ([700] * 6, 2, 256, 4, 256, 16, "fp16", True, "tight"), ([1200, 900], 5, 36, 11, 77, 1, "bf16", True, "wide"),
    ([5000], 2, 64, 33, 256, 64, "bf16", False, "tight"), ([6000], 1, 128, 8, 20, 32, "fp32", True, "heads"),
    ([4100], 3, 132, 2, 256, 8, "bf16", True, "wide"),
]


@pytest.mark.parametrize("lens,H,D,M,K,page,kind,scaled,layout", READ)
def test_read(lens, H, D, M, K, page, kind, scaled, layout):
    from paper_1509_05194_amd import hclae
    rng = np.random.default_rng(sum(lens) + D)
    t = TYPES[kind]
    C = rng.standard_normal((H, M, K, D)).astype(np.float32)
    B, P = len(lens), max(1, max((x + page - 1) // page for x in lens))
    need = sum((x + page - 1) // page for x in lens)
    pages = need + 3
    n_slots = pages * page + page - 1                      # not a whole number of pages
    tables = np.full((B, P), -5, np.int32)
    order = rng.permutation(pages)
    at = 0
    for b, x in enumerate(lens):
        p = (x + page - 1) // page
        tables[b, :p] = order[at:at + p]
        at += p
    bad = []                                               # rows of a page that the cache does not have
    if lens[0] > 3 * page:
        tables[0, 1], tables[0, 2] = pages, -1
        bad = list(range(page, 3 * page))
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    n = int(starts[-1]) + 6
    ids = rng.integers(0, 256, (n_slots, H, M)).astype(np.uint8)   # codes of K or more among them
    g = np.exp(rng.standard_normal((n_slots, H))).astype(np.float32)
    out = placed(torch.full((n, H, D), 5.0, dtype=t, device="cuda"), layout)
    around = out.untyped_storage().nbytes()
    ctx = hclae.Context(n, D, M, K)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    ctx.cache_read(torch.from_numpy(ids).cuda(), torch.from_numpy(g).cuda() if scaled else None, torch.from_numpy(tables).cuda(),
                   torch.from_numpy(starts).cuda(), page, out)
    torch.cuda.synchronize()
    assert bool((out[int(starts[-1]):] == 5.0).all())      # rows behind the last sequence
    if layout != "tight":                                  # and what lies between the rows
        flat = torch.as_strided(out, (around // out.element_size(),), (1,), 0)
        assert int((flat == 7.0).sum()) >= flat.numel() - n * H * D
    slot = np.zeros(n - 6, np.int64)
    for b, x in enumerate(lens):
        pos = np.arange(x)
        slot[starts[b]:starts[b + 1]] = tables[b][pos // page].astype(np.int64) * page + pos % page
    live = np.ones(n - 6, bool)
    live[bad] = False
    for h in range(H):
        assert bool((out[:n - 6, h][torch.from_numpy(~live).cuda()] == 0).all())
        if live.any():
            want, mag = decoded(ids[slot[live], h], C[h], g[slot[live], h] if scaled else 1.0)
            close_to(out[:n - 6, h][torch.from_numpy(live).cuda()], want, mag, M, t)
    ctx.close()


def test_read_sequences_longer_than_their_pages():
    from paper_1509_05194_amd import hclae
    C = torch.ones((1, 1, 1, 8), device="cuda")
    ctx = hclae.Context(64, 8, 1, 1)
    ctx.cache_begin(C)
    codes = torch.zeros((16, 1, 1), dtype=torch.uint8, device="cuda")
    out = torch.full((20, 1, 8), 9.0, device="cuda")
    ctx.cache_read(codes, None, torch.tensor([[1, 3]], dtype=torch.int32, device="cuda"), torch.tensor([0, 17], dtype=torch.int32, device="cuda"),
                   4, out)
    want = torch.tensor([1.0] * 8 + [0.0] * 9 + [9.0] * 3, device="cuda")
    assert torch.equal(out[:, 0], want[:, None].expand(-1, 8))
    ctx.close()


@pytest.mark.parametrize("n,M", [(6, 8), (40000, 8), (40000, 16)])
def test_rows_that_are_not_there_are_zero_whatever_the_codewords_are(n, M):
    from paper_1509_05194_amd import hclae
    K, D = 256, 64
    C = torch.randn((1, M, K, D), generator=torch.Generator().manual_seed(3)).cuda()
    C[0, 0, 0, 5], C[0, M - 1, 0, 7], C[0, 1, 0, 9] = float("inf"), float("nan"), -3e38
    codes = torch.zeros((n, 1, M), dtype=torch.uint8, device="cuda")
    codes[3] = 1
    ctx = hclae.Context(n, D, M, K)
    ctx.cache_begin(C)
    out = torch.full((n, 1, D), 9.0, device="cuda")
    tables = torch.full((1, n), -1, dtype=torch.int32, device="cuda")
    tables[0, 3] = 3
    ctx.cache_read(codes, None, tables, torch.tensor([0, n - 1], dtype=torch.int32, device="cuda"), 1, out)
    want = torch.zeros((n, 1, D), device="cuda")
    want[3], want[n - 1] = C[0, :, 1].double().sum(0).float(), 9.0
    assert torch.allclose(out, want, rtol=0, atol=(M + 3) * U32 * 8 * M)      # |c| < 8
    # pages of 2 rows, two of them in the table: row 3 is the last one that is there
    out.fill_(9.0)
    ctx.cache_read(codes, None, torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"), torch.tensor([0, n - 1], dtype=torch.int32, device="cuda"), 2, out)
    assert torch.allclose(out[3:], want[3:], rtol=0, atol=(M + 3) * U32 * 8 * M)
    looked = torch.full((n, D), 9.0, device="cuda")
    rows = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    rows[4] = n
    ctx.lookup(codes[:, 0], C[0], looked, rows=rows)
    assert bool((looked == 0).all())
    ctx.close()


def test_cache_whose_offsets_pass_32_bits():
    """Slots at both ends of a cache of 5e9 bytes of codes: written, read back, and nothing else touched."""
    from paper_1509_05194_amd import hclae
    n, H, D, M, K, page = 40, 16, 32, 16, 256, 64
    n_slots = 5 * 10 ** 9 // (H * M) // page * page
    x, C = heads(n, H, D, M, K, 3)
    Cg = torch.from_numpy(C).cuda()
    codes = torch.zeros((n_slots, H, M), dtype=torch.uint8, device="cuda")
    scale = torch.zeros((n_slots, H), device="cuda")
    assert codes.numel() > 2 ** 32
    pages = n_slots // page
    tables = torch.tensor([[pages - 1], [pages // 2], [0]], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 20, 30, n], dtype=torch.int32, device="cuda")
    slots = torch.cat([(pages - 1) * page + torch.arange(20), pages // 2 * page + torch.arange(10), torch.arange(10)]).cuda()
    ctx = hclae.Context(n, D, M, K)
    ctx.cache_begin(Cg)
    X = torch.from_numpy(x).cuda()
    ctx.cache_write(X, slots, codes, scale)
    small, small_g = torch.zeros((n, H, M), dtype=torch.uint8, device="cuda"), torch.zeros((n, H), device="cuda")
    ctx.cache_write(X, torch.arange(n, device="cuda"), small, small_g)
    assert torch.equal(codes[slots], small) and torch.equal(scale[slots], small_g)
    assert int((scale != 0).sum()) == n * H
    out = torch.zeros((n, H, D), device="cuda")
    ctx.cache_read(codes, scale, tables, starts, page, out)
    for h in range(H):
        want, mag = decoded(small[:, h].cpu().numpy(), C[h], small_g[:, h].cpu().numpy())
        close_to(out[:, h], want, mag, M, torch.float32)
    ctx.close()


LOOKUP = [
    # T, V, D, M, K, type, rows ("all": rows 0..T-1), factor, gap between output rows
    (1, 1, 4, 1, 1, "fp32", "all", 1.0, 0), (64, 1000, 4096, 8, 256, "bf16", "some", 64.0, 0), (77, 50, 960, 16, 256, "fp32", "some", 1.0, 4),
    (5000, 300, 132, 3, 100, "fp16", "some", -0.5, 12), (9001, 9001, 128, 8, 256, "bf16", "all", 1.0, 0), (3, 9, 36, 40, 256, "fp32", "some", 2.0, 0),
    (20000, 20005, 128, 16, 256, "fp32", "all", 1.0, 0), (2500, 100, 1028, 4, 17, "bf16", "some", 3.0, 8), (4000, 70, 200, 70, 256, "fp16", "some", 0.1, 0),
    (6000, 500, 4096, 8, 256, "bf16", "some", 64.0, 0),
]


def table(T, V, D, M, K, rows, seed):
    rng = np.random.default_rng(seed)
    C = (rng.standard_normal((M, K, D)) * 0.7 ** np.arange(M)[:, None, None]).astype(np.float32)
    ids = rng.integers(0, 256, (V, M)).astype(np.uint8)
    r = None
    if rows == "some":
        r = rng.integers(0, V, T).astype(np.int64)
        if T > 8:
            r[[1, 4, 7]] = [-1, V, -2 ** 62]
            r[8:8 + T // 4] = r[0]                          # one row many times
    return C, ids, r


@pytest.mark.parametrize("T,V,D,M,K,kind,rows,factor,gap", LOOKUP)
def test_lookup(T, V, D, M, K, kind, rows, factor, gap):
    from paper_1509_05194_amd import hclae
    t = TYPES[kind]
    C, ids, r = table(T, V, D, M, K, rows, T + D)
    wide = torch.full((T, D + gap), 7.0, dtype=t, device="cuda")
    out = wide[:, :D]
    ctx = hclae.Context(T, D, M, K)
    ctx.lookup(torch.from_numpy(ids).cuda(), torch.from_numpy(C).cuda(), out, rows=None if r is None else torch.from_numpy(r).cuda(), scale=factor)
    torch.cuda.synchronize()
    assert bool((wide[:, D:] == 7.0).all())
    at = np.arange(T) if r is None else r
    live = (at >= 0) & (at < V)
    assert bool((out[torch.from_numpy(~live).cuda()] == 0).all())
    for i in np.array_split(np.nonzero(live)[0], max(1, live.sum() * D // 2 ** 22)):
        want, mag = decoded(ids[at[i]], C, np.float32(factor))
        close_to(out[torch.from_numpy(i).cuda()], want, mag, M, t)
    ctx.close()


GRAD = [
    # T, V, D, M, K, type, rows, factor, gap
    (1, 1, 4, 1, 1, "fp32", "all", 1.0, 0), (1, 5, 4096, 8, 256, "bf16", "some", 64.0, 0), (64, 1000, 960, 16, 256, "fp32", "some", 1.0, 4),
    (509, 300, 132, 3, 100, "fp16", "some", -0.5, 12), (4096, 4096, 128, 8, 256, "bf16", "all", 1.0, 0), (4097, 5000, 128, 8, 256, "bf16", "all", 1.0, 0),
    (5000, 100, 36, 11, 256, "fp16", "some", 2.0, 0), (9000, 1, 64, 2, 256, "fp32", "some", 1.0, 0), (70001, 900, 20, 3, 7, "bf16", "some", 0.25, 4),
    (6000, 3000, 1028, 2, 200, "bf16", "some", 3.0, 8), (8000, 8000, 516, 9, 256, "fp32", "all", 1.0, 0), (300, 7, 4, 2, 1, "bf16", "some", 1.0, 0),
    (300007, 40000, 12, 2, 256, "bf16", "some", 1.0, 0), (700001, 700001, 4, 3, 90, "fp32", "all", 2.0, 4),
]


@pytest.mark.parametrize("T,V,D,M,K,kind,rows,factor,gap", GRAD)
def test_lookup_grad(T, V, D, M, K, kind, rows, factor, gap):
    from paper_1509_05194_amd import hclae
    t = TYPES[kind]
    C, ids, r = table(T, V, D, M, K, rows, T + D)
    g = torch.randn((T, D + gap), generator=torch.Generator().manual_seed(T), dtype=torch.float32).to(t)
    dC = torch.full((M, K, D), 5.0, device="cuda")
    idsg, rg, gg = torch.from_numpy(ids).cuda(), None if r is None else torch.from_numpy(r).cuda(), g.cuda()[:, :D]
    ctx = hclae.Context(T, D, M, K)
    ctx.lookup_grad(idsg, gg, dC, rows=rg, scale=factor)
    again = torch.full((M, K, D), -1.0, device="cuda")
    ctx.lookup_grad(idsg, gg, again, rows=rg, scale=factor)
    assert torch.equal(dC, again)                          # the same bits
    at = np.arange(T) if r is None else r
    live = np.nonzero((at >= 0) & (at < V))[0]
    gd = g[:, :D].double()[torch.from_numpy(live)]
    f = float(np.float32(factor))
    for m in range(M):
        c = torch.from_numpy(np.minimum(ids[at[live], m], K - 1).astype(np.int64))
        want = torch.zeros((K, D), dtype=torch.float64).index_add_(0, c, gd) * f
        mag = torch.zeros((K, D), dtype=torch.float64).index_add_(0, c, gd.abs()) * abs(f)
        n = torch.bincount(c, minlength=K).double()[:, None]
        tol = (n + 2) * U32 * mag * (1 + 2.0 ** -8)
        off = (dC[m].cpu().double() - want).abs()
        assert bool((off <= tol).all()), (m, float((off - tol).max()))
    ctx.close()


@pytest.mark.parametrize("T,K", [(300, 40), (6000, 256)])
def test_lookup_grad_is_the_slope_of_the_lookup(T, K):
    """f(C) = <w, lookup(C)> is linear in C: its slope along E, from two lookups in fp32, is <dC, E>.  The difference of the two is off by
    their rounding: 2 (M + 3) 2^-24 of the sum of magnitudes."""
    from paper_1509_05194_amd import hclae
    V, D, M = 200, 64, 3
    C, ids, r = table(T, V, D, M, K, "some", 1)
    rng = np.random.default_rng(2)
    E = rng.standard_normal(C.shape).astype(np.float32)
    w = torch.from_numpy(rng.standard_normal((T, D)).astype(np.float32)).cuda()
    idsg, rg = torch.from_numpy(ids).cuda(), torch.from_numpy(r).cuda()
    ctx = hclae.Context(T, D, M, K)
    outs = []
    for s in (1.0, -1.0):
        out = torch.empty((T, D), device="cuda")
        ctx.lookup(idsg, torch.from_numpy((C + np.float32(s) * E)).cuda(), out, rows=rg, scale=1.5)
        outs.append(out.double())
    dC = torch.empty((M, K, D), device="cuda")
    ctx.lookup_grad(idsg, w, dC, rows=rg, scale=1.5)
    slope = float((w.double() * (outs[0] - outs[1])).sum()) / 2
    got = float((dC.cpu().double() * torch.from_numpy(E).double()).sum())
    size = float((w.double().abs() * (M * 1.5 * float(np.abs(C).max() + np.abs(E).max()))).sum())
    assert abs(slope - got) <= size * ((M + 3 + 2) * U32 + T * U32)
    ctx.close()


def test_cache_written_and_read_as_a_program_does():
    """Prompts of three sequences written together, then single tokens step by step, captured in a graph; all of it read back
    equals the lookup of the same codes; another stream than torch's current one."""
    from paper_1509_05194_amd import hclae
    H, D, M, K, page, steps = 4, 128, 8, 256, 16, 5
    lens = [37, 1, 90]
    total = sum(lens)
    x, C = heads(total + 3 * steps, H, D, M, K, 12)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        X = torch.from_numpy(x).cuda().to(torch.bfloat16)
        Cg = torch.from_numpy(C).cuda()
        pages = 24
        tables = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).int().cuda().reshape(3, 8)
        codes = torch.zeros((pages * page, H, M), dtype=torch.uint8, device="cuda")
        scale = torch.zeros((pages * page, H), device="cuda")
        ctx = hclae.Context(total + 3 * steps, D, M, K)    # takes the current stream: s
        ctx.cache_begin(Cg)

        def slot(b, pos):
            return int(tables[b, pos // page]) * page + pos % page

        prompt = torch.tensor([slot(b, p) for b, n in enumerate(lens) for p in range(n)], device="cuda")
        ctx.cache_write(X[:total], prompt, codes, scale)
        step_x = torch.empty((4, H, D), dtype=torch.bfloat16, device="cuda")   # a padded batch: the last row is no token's
        step_slots = torch.full((4,), -1, dtype=torch.int64, device="cuda")
        step_x.zero_()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            ctx.cache_write(step_x, step_slots, codes, scale)
        for i in range(steps):
            step_x[:3] = X[total + 3 * i:total + 3 * i + 3]
            step_slots[:3] = torch.tensor([slot(b, lens[b] + i) for b in range(3)], device="cuda")
            graph.replay()
            torch.cuda.synchronize()
        # all rows again, sequence after sequence
        order, at = [], 0
        for b, n in enumerate(lens):
            order += list(range(at, at + n)) + [total + 3 * i + b for i in range(steps)]
            at += n
        starts = torch.tensor(np.concatenate([[0], np.cumsum([n + steps for n in lens])]), dtype=torch.int32, device="cuda")
        out = torch.zeros((total + 3 * steps, H, D), dtype=torch.bfloat16, device="cuda")
        ctx.cache_read(codes, scale, tables, starts, page, out)
        one = torch.zeros_like(codes[:total + 3 * steps])
        one_g = torch.zeros_like(scale[:total + 3 * steps])
        ctx.cache_write(X[order], torch.arange(total + 3 * steps, device="cuda"), one, one_g)
        torch.cuda.synchronize()
        want_rows = torch.tensor([slot(b, p) for b, n in enumerate(lens) for p in range(n + steps)], device="cuda")
        assert torch.equal(codes[want_rows], one) and torch.equal(scale[want_rows], one_g)
        assert int((scale != 0).sum()) == (total + 3 * steps) * H
        for h in range(H):
            want, mag = decoded(one[:, h].cpu().numpy(), C[h], one_g[:, h].cpu().numpy())
            close_to(out[:, h], want, mag, M, torch.bfloat16)
            look = torch.empty((total + 3 * steps, D), device="cuda")
            ctx.lookup(one[:, h].contiguous(), Cg[h], look)
            scaled_look = look * one_g[:, h:h + 1]
            close_to(scaled_look, want, mag, M, torch.float32)
        ctx.close()


@pytest.mark.parametrize("T", [700, 9000])
def test_table_captured_and_replayed(T):
    """A lookup and its gradient in one graph, replayed with other rows: the eager answers."""
    from paper_1509_05194_amd import hclae
    V, D, M, K = 400, 256, 4, 256
    C, ids, _ = table(T, V, D, M, K, "all", 4)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = hclae.Context(T, D, M, K)
        Cg, idsg = torch.from_numpy(C).cuda(), torch.from_numpy(ids).cuda()
        rows = torch.zeros((T,), dtype=torch.int64, device="cuda")
        g = torch.randn((T, D), device="cuda").to(torch.bfloat16)
        out, dC = torch.zeros((T, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((M, K, D), device="cuda")
        ctx.lookup_grad(idsg, g, dC, rows=rows)            # the first call of this size allocates
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            ctx.lookup(idsg, Cg, out, rows=rows, scale=2.0)
            ctx.lookup_grad(idsg, g, dC, rows=rows, scale=2.0)
        for i in range(3):
            rows.copy_(torch.randint(-1, V, (T,), generator=torch.Generator().manual_seed(i)).cuda())
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone(), dC.clone()
            ctx.lookup(idsg, Cg, out, rows=rows, scale=2.0)
            ctx.lookup_grad(idsg, g, dC, rows=rows, scale=2.0)
            torch.cuda.synchronize()
            assert torch.equal(out, got[0]) and torch.equal(dC, got[1])
        ctx.close()


def test_dictionaries_laid_out_again():
    """Other dictionaries, fewer heads, then more: every call uses those of the last hclae_cache_begin."""
    from paper_1509_05194_amd import hclae
    n, D, M, K = 20, 64, 3, 40
    ctx = hclae.Context(n, D, M, K)
    for H, seed in ((3, 1), (3, 2), (1, 3), (2, 4), (7, 5)):
        x, C = heads(n, H, D, M, K, seed)
        ctx.cache_begin(torch.from_numpy(C).cuda())
        codes, scale = torch.zeros((n, H, M), dtype=torch.uint8, device="cuda"), torch.zeros((n, H), device="cuda")
        ctx.cache_write(torch.from_numpy(x).cuda(), torch.arange(n, device="cuda"), codes, scale)
        out = torch.zeros((n, H, D), device="cuda")
        ctx.cache_read(codes, scale, torch.arange(5, dtype=torch.int32, device="cuda")[None], torch.tensor([0, n], dtype=torch.int32, device="cuda"), 4, out)
        for h in range(H):
            want, g = quantise(x[:, h].copy(), C[h], True)
            assert np.array_equal(codes[:, h].cpu().numpy(), want)
            back, mag = decoded(want, C[h], g)
            close_to(out[:, h], back, mag, M, torch.float32)
    ctx.close()


def test_large_calls_captured_on_two_streams_at_once():
    """Two contexts on two streams, each with a prompt written, read back, and the gradient of a lookup in one graph, replayed side by side
    with eager work in between: the bits of the same calls one after another."""
    from paper_1509_05194_amd import hclae
    H, D, M, K, n, page = 4, 128, 8, 256, 3000, 16
    jobs = []
    for seed in (1, 2):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            x, C = heads(n, H, D, M, K, seed)
            j = {"s": s, "X": torch.from_numpy(x).cuda().to(torch.bfloat16), "C": torch.from_numpy(C).cuda(), "ctx": hclae.Context(2 * n, D, M, K)}
            j["slots"] = torch.randperm(n, generator=torch.Generator().manual_seed(seed)).cuda()
            j["codes"], j["scale"] = torch.zeros((n, H, M), dtype=torch.uint8, device="cuda"), torch.zeros((n, H), device="cuda")
            j["tables"] = torch.arange((n + page - 1) // page, dtype=torch.int32, device="cuda")[None]
            j["starts"] = torch.tensor([0, n], dtype=torch.int32, device="cuda")
            j["out"], j["dC"] = torch.zeros((n, H, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((M, K, D), device="cuda")
            j["rows"] = torch.randint(-1, n * H, (2 * n,), generator=torch.Generator().manual_seed(seed)).cuda()
            j["g"] = torch.randn((2 * n, D), generator=torch.Generator().manual_seed(seed)).cuda()

            def work(j=j):
                j["ctx"].cache_write(j["X"], j["slots"], j["codes"], j["scale"])
                j["ctx"].cache_read(j["codes"], j["scale"], j["tables"], j["starts"], page, j["out"])
                j["ctx"].lookup_grad(j["codes"].view(n * H, M), j["g"], j["dC"], rows=j["rows"])

            j["ctx"].cache_begin(j["C"])
            work()
            torch.cuda.synchronize()
            j["want"] = [j[k].clone() for k in ("codes", "scale", "out", "dC")]
            j["graph"] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(j["graph"], stream=s):
                work()
        jobs.append(j)
    for _ in range(3):
        for j in jobs:
            for k in ("codes", "scale", "out", "dC"):
                j[k].zero_()
        torch.cuda.synchronize()
        for j in jobs:
            with torch.cuda.stream(j["s"]):
                j["graph"].replay()
        torch.cuda.synchronize()
        for j in jobs:
            for k, want in zip(("codes", "scale", "out", "dC"), j["want"]):
                assert torch.equal(j[k], want), k
    for j in jobs:
        j["ctx"].close()


def test_refusals():
    from paper_1509_05194_amd import hclae
    L = hclae.lib()
    ctx = hclae.Context(100, 16, 2, 8)
    x = torch.zeros((10, 3, 16), device="cuda")
    C = torch.zeros((3, 2, 8, 16), device="cuda")
    slots = torch.arange(10, device="cuda")
    codes, scale = torch.zeros((10, 3, 2), dtype=torch.uint8, device="cuda"), torch.zeros((10, 3), device="cuda")
    tables, starts = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros((2,), dtype=torch.int32, device="cuda")

    def refused(code, f, *a, **k):
        with pytest.raises(hclae.HclaeError) as e:
            f(*a, **k)
        assert e.value.code == code

    refused(hclae.ESTATE, ctx.cache_write, x, slots, codes, scale)
    refused(hclae.ESTATE, ctx.cache_read, codes, scale, tables, starts, 4, x)
    for H in (0, 1025):
        assert L.hclae_cache_begin(ctx._h, C.data_ptr(), H, 2, 8, 16) == hclae.EINVAL
    assert L.hclae_cache_begin(ctx._h, None, 3, 2, 8, 16) == hclae.EINVAL
    assert L.hclae_cache_begin(ctx._h, C.data_ptr() + 4, 3, 2, 8, 16) == hclae.EINVAL
    assert L.hclae_cache_begin(ctx._h, C.data_ptr(), 3, 2, 8, 12) == hclae.ESTATE
    ctx.cache_begin(C)

    def write(X=x.data_ptr(), kind=0, n=10, rs=48, hs=16, s=slots.data_ptr(), ns=10, c=codes.data_ptr(), g=scale.data_ptr()):
        return L.hclae_cache_write(ctx._h, X, kind, n, rs, hs, s, ns, c, g)

    assert write() == hclae.OK and write(n=0, X=None) == hclae.OK and write(ns=0, c=None) == hclae.OK
    for bad in (dict(X=None), dict(s=None), dict(c=None), dict(kind=3), dict(kind=-1), dict(X=x.data_ptr() + 4), dict(X=x.data_ptr() + 2, kind=1),
                dict(rs=47), dict(hs=18), dict(rs=-48), dict(ns=-1), dict(ns=2 ** 41), dict(n=-1), dict(s=slots.data_ptr() + 4),
                dict(g=scale.data_ptr() + 2)):
        assert write(**bad) == hclae.EINVAL, bad
    assert write(n=101) == hclae.ESTATE

    def read(c=codes.data_ptr(), ns=10, t=tables.data_ptr(), B=1, P=1, page=4, st=starts.data_ptr(), n=10, out=x.data_ptr(), kind=0, rs=48, hs=16):
        return L.hclae_cache_read(ctx._h, c, scale.data_ptr(), ns, t, B, P, page, st, n, out, kind, rs, hs)

    assert read() == hclae.OK and read(n=0, out=None) == hclae.OK and read(B=0, st=None) == hclae.OK and read(hs=160, rs=16) == hclae.OK
    for bad in (dict(c=None), dict(t=None), dict(st=None), dict(out=None), dict(kind=7), dict(page=0), dict(P=-1), dict(B=-1), dict(out=x.data_ptr() + 8),
                dict(rs=44), dict(rs=0), dict(hs=0), dict(hs=12), dict(hs=156, rs=16), dict(ns=-1)):
        assert read(**bad) == hclae.EINVAL, bad
    assert read(n=101) == hclae.ESTATE

    out, dC = torch.zeros((10, 16), device="cuda"), torch.zeros((2, 8, 16), device="cuda")
    ids = torch.zeros((10, 2), dtype=torch.uint8, device="cuda")

    def look(r=slots.data_ptr(), T=10, c=ids.data_ptr(), V=10, C=C.data_ptr(), out=out.data_ptr(), kind=0, rs=16):
        return L.hclae_lookup(ctx._h, r, T, c, V, 1.0, C, 2, 8, 16, out, kind, rs)

    def grad(r=slots.data_ptr(), T=10, c=ids.data_ptr(), V=10, C=dC.data_ptr(), out=out.data_ptr(), kind=0, rs=16):
        return L.hclae_lookup_grad(ctx._h, r, T, c, V, 1.0, out, kind, rs, 2, 8, 16, C)

    for f in (look, grad):
        assert f() == hclae.OK and f(r=None) == hclae.OK and f(V=0, c=None) == hclae.OK
        for bad in (dict(c=None), dict(C=None), dict(out=None), dict(r=None, V=9), dict(kind=3), dict(rs=18), dict(rs=-16), dict(out=out.data_ptr() + 4),
                    dict(C=C.data_ptr() + 4), dict(T=-1), dict(V=-1)):
            assert f(**bad) == hclae.EINVAL, (f, bad)
        assert f(T=101) == hclae.ESTATE
    assert look(rs=12) == hclae.EINVAL and look(T=0, out=None) == hclae.OK
    dC.fill_(3.0)
    assert grad(T=0, out=None) == hclae.OK and bool((dC == 0).all())
    for bad, err in ((x.double(), TypeError), (x[:, :, ::2], ValueError), (x[:, :2], ValueError), (x.cpu(), TypeError)):
        with pytest.raises(err):
            ctx.cache_write(bad, slots, codes, scale)
    ctx.close()
