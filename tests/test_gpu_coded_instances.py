"""Every form of the reads (how many dictionaries share a half line of LDS, one or several rounds a row, rows of words or of bytes), and writes of the most
heads and of many dictionaries, against 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U32 = 2.0 ** -24
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}

# M, K, D: one, two, four and eight dictionaries a half line, a row in one round and in several; M a multiple of four and not
SHAPES = [(4, 256, 64), (3, 200, 36), (8, 64, 64), (7, 100, 20), (8, 256, 64), (6, 256, 16), (16, 64, 64), (14, 100, 44), (16, 256, 64), (13, 256, 8), (24, 100, 64),
          (22, 120, 28), (32, 200, 64), (30, 190, 12), (8, 256, 4), (5, 256, 4)]


def decoded(ids, C, factor):
    """factor * sum_m C[m][ids[:, m]] and the sum of magnitudes."""
    c = [C[m].double()[ids[:, m].long().clamp(max=C.shape[1] - 1)] for m in range(C.shape[0])]
    return sum(c) * factor, sum(v.abs() for v in c) * factor.abs()


def check(got, want, mag, M, t):
    """Off by (M + 3) 2^-24 of the sum of magnitudes and half a step of the type."""
    f = torch.finfo(t)
    tol = (1 + 2.0 ** -8) * (want.abs() * f.eps / 2 + (M + 3) * U32 * mag) + f.tiny * f.eps / 2
    assert bool(((got.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("M,K,D", SHAPES)
def test_reads_and_lookups_of_many_rows(M, K, D, kind):
    from paper_1509_05194_amd import hclae
    H, page, t = 3, 16, TYPES[kind]
    gen = torch.Generator().manual_seed(M * K + D)
    lens = [20011, 0, 1, 63, 64, 8005]
    n = sum(lens)
    C = torch.randn((H, M, K, D), generator=gen) / M
    pages = sum((x + page - 1) // page for x in lens) + 2
    ids = torch.randint(0, 256, (pages * page, H, M), dtype=torch.uint8, generator=gen)
    scale = torch.exp(torch.randn((pages * page, H), generator=gen))
    order, P = torch.randperm(pages, generator=gen).int(), (max(lens) + page - 1) // page
    tables, at, slots = torch.full((len(lens), P), -1, dtype=torch.int32), 0, []
    for b, x in enumerate(lens):
        p = (x + page - 1) // page
        tables[b, :p] = order[at:at + p]
        at += p
        pos = torch.arange(x)
        slots.append(tables[b][pos // page].long() * page + pos % page)
    slots = torch.cat(slots)
    starts = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32)
    out = torch.full((n + 7, H, D), 5.0, dtype=t, device="cuda")
    ctx = hclae.Context(n + 7, D, M, K)
    ctx.cache_begin(C.cuda())
    ctx.cache_read(ids.cuda(), scale.cuda(), tables.cuda(), starts.cuda(), page, out)
    got = out.cpu()
    assert bool((got[n:] == 5.0).all())
    for h in range(H):
        want, mag = decoded(ids[slots, h], C[h], scale[slots, h].double()[:, None])
        check(got[:n, h], want, mag, M, t)
    # rows of a table: one head's codes, some rows of none
    rows = torch.randint(-50, pages * page + 50, (n,), generator=gen)
    flat = ids[:, 1].contiguous()
    look = torch.full((n, D), 5.0, dtype=t, device="cuda")
    ctx.lookup(flat.cuda(), C[1].cuda(), look, rows=rows.cuda(), scale=-2.5)
    live = (rows >= 0) & (rows < pages * page)
    want, mag = decoded(flat[rows[live]], C[1], torch.tensor(-2.5, dtype=torch.float64))
    check(look.cpu()[live], want, mag, M, t)
    assert bool((look.cpu()[~live] == 0).all())
    ctx.close()


def quantise(x, C):
    """Codes and scales of the rows x of one head."""
    g = np.abs(x).max(1)
    r = (x / g[:, None]).astype(np.float32)
    codes = np.zeros((len(x), C.shape[0]), np.uint8)
    for m in range(C.shape[0]):
        c = C[m].astype(np.float64)
        for i in range(len(r)):
            codes[i, m] = ((r[i].astype(np.float64) - c) ** 2).sum(1).argmin()
        r = r - C[m][codes[:, m]]
    return codes, g


# n, H, D, M, K: the most heads; the most dictionaries and nearly; in each kernel of the writes
@pytest.mark.parametrize("n,H,D,M,K", [(1, 1024, 8, 2, 16), (9, 1024, 8, 2, 16), (200, 1024, 8, 2, 16), (700, 1024, 8, 1, 3), (3, 1, 32, 256, 8), (1100, 2, 32, 70, 16),
                                       (4200, 2, 32, 70, 16), (9100, 1, 64, 256, 8)])
def test_writes_of_the_most_heads_and_of_many_dictionaries(n, H, D, M, K):
    from paper_1509_05194_amd import hclae
    rng = np.random.default_rng(n + H)
    x = rng.standard_normal((n, H, D)).astype(np.float32)
    C = (rng.standard_normal((H, M, K, D)) * (0.5 * 0.98 ** np.arange(M))[None, :, None, None]).astype(np.float32)
    codes, scale = torch.full((n, H, M), 251, dtype=torch.uint8, device="cuda"), torch.full((n, H), -3.0, device="cuda")
    slots = torch.randperm(n, generator=torch.Generator().manual_seed(n))
    ctx = hclae.Context(n, D, M, K)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    ctx.cache_write(torch.from_numpy(x).cuda(), slots.cuda(), codes, scale)
    got, got_g, to = codes.cpu().numpy(), scale.cpu().numpy(), slots.numpy()
    assert np.array_equal(got_g[to], np.abs(x).max(2))
    at = np.unique(np.concatenate([[0, n - 1], rng.integers(0, n, 12)]))
    for h in np.unique(np.concatenate([[0, H - 1], rng.integers(0, H, 6)])):
        assert np.array_equal(got[to[at], h], quantise(x[at, h], C[h])[0]), h
    # and read back: all of it
    out = torch.empty((n, H, D), device="cuda")
    ctx.cache_read(codes, scale, torch.arange(n, dtype=torch.int32, device="cuda")[None], torch.tensor([0, n], dtype=torch.int32, device="cuda"), 1, out)
    for h in (0, H - 1):
        want, mag = decoded(codes[:, h].cpu(), torch.from_numpy(C[h]), scale[:, h].cpu().double()[:, None])
        check(out[:, h].cpu(), want, mag, M, torch.float32)
    ctx.close()


def test_rows_whose_offsets_pass_32_bits():
    """A lookup of 600,011 rows of 4096, 4.9e9 bytes, and the gradient from as many: the last rows, the first, and some between, exactly."""
    from paper_1509_05194_amd import hclae
    T, V, D, M, K = 600011, 500, 4096, 2, 16
    gen = torch.Generator().manual_seed(3)
    C = torch.randint(-8, 9, (M, K, D), generator=gen).float().cuda()
    ids = torch.randint(0, K, (V, M), dtype=torch.uint8, generator=gen).cuda()
    rows = torch.randint(0, V, (T,), generator=gen).cuda()
    at = torch.cat([torch.arange(20), torch.arange(T - 300, T), torch.randint(0, T, (500,), generator=gen)]).unique().cuda()
    ctx = hclae.Context(T, D, M, K)
    x = torch.full((T, D), 3.0, dtype=torch.bfloat16, device="cuda")
    assert x.numel() * 2 > 2 ** 32
    ctx.lookup(ids, C, x, rows=rows)
    picked = ids[rows[at]].long()
    assert torch.equal(x[at].float(), C[0][picked[:, 0]] + C[1][picked[:, 1]])      # whole numbers to 16
    x.zero_()
    g = torch.randint(-8, 9, (len(at), D), generator=gen).float().cuda()
    x[at] = g.to(torch.bfloat16)
    dC, want = torch.full((M, K, D), 7.0, device="cuda"), torch.zeros((M, K, D), device="cuda")
    ctx.lookup_grad(ids, x, dC, rows=rows)
    for m in range(M):
        for k in range(K):
            want[m, k] = g[picked[:, m] == k].sum(0)
    assert torch.equal(dC, want)
    ctx.close()
