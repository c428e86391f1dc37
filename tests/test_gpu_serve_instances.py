"""Every form of the kernels that serve a paged cache of codes: query heads a block takes, widths of the fixed point, code rows by words, wide words and
bytes, pages a wave is in one of, calls taken in rounds.  The plain forms and tolerances are those of test_gpu_serve."""
import numpy as np
import pytest

from test_gpu_serve import Case, compact, extend, extend_on_device, select

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("M,K", [(8, 256), (16, 256), (7, 256), (8, 100), (20, 64), (32, 256)])
@pytest.mark.parametrize("R,kind", [(1, "bf16"), (2, "bf16"), (4, "fp16"), (1, "fp32"), (2, "fp32"), (3, "fp32")])
def test_attend_through_tables(R, kind, M, K, page):
    c = Case([2100, 1100, 0, 3], 1, R, 16, M, K, page, kind, True, seed=R * M + K + page)
    ctx = c.device()
    c.check(*c.run(ctx))
    ctx.close()


@pytest.mark.parametrize("D", [4, 36, 64, 68, 100, 128, 132, 196, 256])
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_attend_row_lengths(D, kind):
    c = Case([700, 40], 2, 4, D, 4, 32, 16, kind, True, seed=D)
    ctx = c.device()
    c.check(*c.run(ctx))
    c.check(*c.run(ctx, layout="wide"))
    ctx.close()


@pytest.mark.parametrize("page", [64, 192])
@pytest.mark.parametrize("kind,M", [("bf16", 8), ("fp32", 16)])
def test_attend_pages_of_waves(kind, M, page):
    """Pages that hold whole waves of rows: picked ones, pages that are not there, a first row on, lengths that end within a wave."""
    c = Case([5000, 330, 64, 129], 2, 4, 32, M, 256, page, kind, True, seed=M + page)
    ctx = c.device()
    c.check(*c.run(ctx))
    picked = c.rng.integers(-2, c.max_pages + 2, (c.B, 2, 40)).astype(np.int32)
    c.check(*c.run(ctx, picked=picked), picked=picked)
    begins = np.array([70, 64, 63, 0], np.int32)
    c.check(*c.run(ctx, begins=begins, picked=picked), begins=begins, picked=picked)
    c.tables[:, 1::3] = -1
    c.tables[:, 2::5] = c.n_pages
    c.check(*c.run(ctx))
    c.check(*c.run(ctx, picked=picked), picked=picked)
    ctx.close()


@pytest.mark.parametrize("n,M", [(100, 8), (2500, 8), (2500, 5), (900, 16)])
def test_attend_codes_at_any_address(n, M):
    c = Case([n], 1, 4, 32, M, 256, 16, "bf16", True, seed=n)
    ctx = c.device()
    want, want_lse, tol = c.attend()
    for off in (1, 2, 4):
        flat = torch.zeros((c.codes.size + off,), dtype=torch.uint8, device="cuda")
        codes = flat[off:].view(c.codes.shape)
        codes.copy_(torch.from_numpy(c.codes))
        scale = torch.zeros((c.scale.size + 1,), device="cuda")[1:].view(c.scale.shape)
        scale.copy_(torch.from_numpy(c.scale))
        out = torch.zeros((1, 4, 32), dtype=c.kind, device="cuda")
        ctx.cache_attend(c.Q.cuda(), codes, scale, torch.from_numpy(c.tables).cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"), 16, out)
        assert not (np.abs(out.double().cpu().numpy() - want) > tol).any()
    ctx.close()


@pytest.mark.parametrize("lens,R", [([3] * 700, 32), ([400, 330] * 300, 32), ([50] * 5, 4000)])
def test_attend_in_rounds(lens, R):
    """More query heads than a round takes, and more than a sequence's share of one."""
    c = Case(lens, 1, R, 8, 2, 8, 16, "bf16", True, seed=len(lens))
    ctx = c.device()
    out, lse = c.run(ctx)
    keep = sorted(set([0, 1, c.B // 2, c.B - 2, c.B - 1]) | set(range(508, min(516, c.B))))     # around the rounds' border
    part = Case(lens, 1, R, 8, 2, 8, 16, "bf16", True, seed=len(lens))
    part.lens = [part.lens[b] for b in keep]
    part.tables, part.Q, part.B = part.tables[keep], part.Q[keep], len(keep)
    part.check(out[keep], lse[keep])
    same, _ = c.run(ctx)
    assert torch.equal(same, out)
    ctx.close()


def test_attend_steep_scores():
    """Scores of tens of thousands beside values of very different size: one row decides, and nothing overflows."""
    for kind in ("bf16", "fp32"):
        c = Case([3000], 1, 4, 32, 4, 256, 16, kind, True, seed=8)
        slots = c.rows(0, 0)
        c.scale[slots, 0] = c.rng.uniform(1e4, 1e5, len(slots))
        c.scale[slots, 1] = np.where(np.arange(len(slots)) % 3, 1e-4, 1e4)
        ctx = c.device()
        out, lse = c.run(ctx)
        assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
        x = c.x(0, slots)
        for r in range(4):
            s = c.factor * (x @ c.Q[0, r].double().numpy())
            first, second = np.sort(s)[::-1][:2]
            if first - second > 1e3:                                 # far beyond what the scores may be off by: the row itself
                v = c.x(1, slots[[s.argmax()]])[0]
                assert np.abs(out[0, r].double().cpu().numpy() - v).max() <= 2.0 ** -7 * np.abs(v).max()
        ctx.close()


def test_attend_begins_of_zero_change_nothing():
    """Rows from 0 on given as an array: the same bits as without."""
    for page in (16, 64):
        c = Case([2600, 100], 2, 4, 64, 8, 256, page, "bf16", True, seed=page)
        ctx = c.device()
        a, la = c.run(ctx)
        b, lb = c.run(ctx, begins=np.zeros(2, np.int32))
        assert torch.equal(a, b) and torch.equal(la, lb)
        every = np.tile(np.arange(c.max_pages, dtype=np.int32), (2, 2, 1))
        b, lb = c.run(ctx, picked=np.ascontiguousarray(every))        # all pages picked
        c.check(b, lb)
        ctx.close()


def test_select_in_rounds():
    from paper_1509_05194_amd import hclae
    B, H, M, K, D, page, n_pages = 1100, 8, 16, 256, 8, 4, 40
    rng = np.random.default_rng(1)
    C = rng.standard_normal((H, M, K, D)).astype(np.float32)
    codes, scale = rng.integers(0, 256, (n_pages, H, M)).astype(np.uint8), rng.standard_normal((n_pages, H)).astype(np.float32)
    tables, lens = rng.integers(0, n_pages, (B, 9)).astype(np.int32), rng.integers(0, 37, B).astype(np.int32)
    Q = rng.standard_normal((B, 2 * H, D)).astype(np.float32)
    ctx = hclae.Context(B, D, M, K)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    picked = torch.zeros((B, H, 3), dtype=torch.int32, device="cuda")
    ctx.cache_select(torch.from_numpy(Q).cuda(), torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda(), torch.from_numpy(tables).cuda(), torch.from_numpy(lens).cuda(), page, picked)
    keep = [0, 1, 500, 980, 985, 990, 995, 1000, 1098, 1099]
    want = select(Q[keep].astype(np.float64), C, codes, scale, tables[keep], lens[keep], page, n_pages, 3, 1, 1)
    assert np.array_equal(picked.cpu().numpy()[keep], want)
    ctx.close()


@pytest.mark.parametrize("P,k,values", [(3000, 700, 5), (5000, 64, 3000), (2500, 2499, 2), (1500, 33, 1500), (70, 69, 3), (20000, 40, 50)])
def test_select_equal_scores(P, k, values):
    """Few different scores among many pages: the lowest pages of those that share the last one taken."""
    from paper_1509_05194_amd import hclae
    rng = np.random.default_rng(P)
    C = np.ones((1, 1, 2, 4), np.float32)
    scale = rng.permutation(np.arange(P) % values).astype(np.float32)[:, None] - values // 2
    codes = np.zeros((P, 1, 1), np.uint8)
    order = rng.permutation(P).astype(np.int32)
    ctx = hclae.Context(1, 4, 1, 2)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    picked = torch.zeros((1, 1, k), dtype=torch.int32, device="cuda")
    Q = torch.full((1, 1, 4), 0.37, device="cuda")
    ctx.cache_select(Q, torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda(), torch.from_numpy(order[None]).cuda(), torch.tensor([P], dtype=torch.int32, device="cuda"), 1, picked,
                     first=0, recent=0)
    want = select(Q.double().cpu().numpy(), C, codes, scale, order[None], [P], 1, P, k, 0, 0)
    assert np.array_equal(picked.cpu().numpy(), want)
    ctx.close()


@pytest.mark.parametrize("off", [0, 1, 4, 8])
@pytest.mark.parametrize("H,M", [(2, 8), (3, 5), (1, 16)])
def test_copy_at_any_address(H, M, off):
    from paper_1509_05194_amd import hclae
    page, pages = 7, 50
    rng = np.random.default_rng(off)
    codes = rng.integers(0, 256, (pages * page, H, M)).astype(np.uint8)
    scale = rng.standard_normal((pages * page, H)).astype(np.float32)
    dc = torch.zeros((codes.size + off,), dtype=torch.uint8, device="cuda")[off:].view(codes.shape)
    ds = torch.zeros((scale.size + 1,), device="cuda")[1:].view(scale.shape)
    dc.copy_(torch.from_numpy(codes))
    ds.copy_(torch.from_numpy(scale))
    order = rng.permutation(pages).astype(np.int32)
    src, dst, rows = order[:20], order[20:40], rng.integers(0, page + 1, 20).astype(np.int32)
    ctx = hclae.Context(1, 4, M, 1)
    ctx.cache_begin(torch.zeros((H, M, 1, 4), device="cuda"))
    ctx.cache_copy(dc, ds, page, torch.from_numpy(src).cuda(), torch.from_numpy(dst).cuda(), torch.from_numpy(rows).cuda())
    for f, d, r in zip(src, dst, rows):
        codes[d * page:d * page + r] = codes[f * page:f * page + r]
        scale[d * page:d * page + r] = scale[f * page:f * page + r]
    assert np.array_equal(dc.cpu().numpy(), codes) and np.array_equal(ds.cpu().numpy(), scale)
    ctx.close()


@pytest.mark.parametrize("B,most,page,n,seed", [(3, 20000, 2, 30000, 0), (40000, 2, 3, 50000, 1), (7, 300, 16, 20000, 2), (1, 32768, 1, 9000, 3), (1100, 20, 4, 3000, 4)])
def test_extend_large(B, most, page, n, seed):
    """Beyond what one block does, and at its edges: many entries, many sequences, many rows, more sequences than a block has threads."""
    from paper_1509_05194_amd import hclae
    rng = np.random.default_rng(seed)
    adds = rng.multinomial(n, np.ones(B) / B)
    lens = np.minimum(rng.integers(0, most * page // 2 + 1, B), most * page - 1)
    pages = [-(-int(x) // page) for x in lens]
    n_pages = sum(pages) + int(n // page * 0.8) + 5
    order = rng.permutation(n_pages)
    tables = np.zeros((B, most), np.int32)
    at = 0
    for b, p in enumerate(pages):
        tables[b, :p] = order[at:at + p]
        at += p
    starts = np.concatenate([[0], np.cumsum(adds)])
    ctx = hclae.Context(n, 8, 1, 2)
    t, l, slots, moves = extend_on_device(ctx, tables, lens, starts, n, page, n_pages)
    want = extend(tables, lens, starts, n, page, n_pages)
    assert np.array_equal(slots.cpu().numpy(), want[2]) and np.array_equal(l.cpu().numpy(), np.array(want[1])) and np.array_equal(t.cpu().numpy(), want[0])
    for got, w in zip(moves, want[3]):
        assert np.array_equal(got.cpu().numpy(), w)
    ctx.close()


@pytest.mark.parametrize("B,most,page,pool,seed", [(50, 1000, 2, 40000, 0), (9000, 3, 4, 30000, 1), (8000, 4, 4, 65536, 2), (3, 5, 4, 65537, 3), (1, 32768, 1, 32800, 4)])
def test_compact_large(B, most, page, pool, seed):
    from paper_1509_05194_amd import hclae
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, most * page + 1, B)
    tables = rng.integers(-2, pool + 2, (B, most)).astype(np.int32)
    t = torch.from_numpy(tables).cuda()
    src, dst = (torch.full((pool // 2,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    used = torch.zeros((1,), dtype=torch.int32, device="cuda")
    ctx = hclae.Context(1, 4, 1, 1)
    ctx.cache_compact(t, torch.from_numpy(lens.astype(np.int32)).cuda(), page, pool, src, dst, used)
    want_t, want_src, want_dst, u = compact(tables, lens, page, pool)
    assert int(used) == u and np.array_equal(src.cpu().numpy(), want_src) and np.array_equal(dst.cpu().numpy(), want_dst) and np.array_equal(t.cpu().numpy(), want_t)
    ctx.close()


def test_two_contexts_on_two_streams():
    """Two caches served at the same time, steps enqueued in turn, give what each gives alone."""
    from paper_1509_05194_amd import hclae
    cases = [Case([2500, 300], 2, 4, 64, 8, 256, 16, "bf16", True, seed=i) for i in range(2)]
    dev = lambda a: torch.from_numpy(a).cuda()
    alone = [c.run(c.device())[0] for c in cases]
    state = []
    for c in cases:
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            ctx = hclae.Context(c.B, 64, 8, 256, stream=st.cuda_stream)
            ctx.cache_begin(dev(c.C))
            state.append((st, ctx, c.Q.cuda(), dev(c.codes), dev(c.scale), dev(c.tables), torch.tensor(c.lens, dtype=torch.int32, device="cuda"),
                          [torch.zeros((c.B, 8, 64), dtype=c.kind, device="cuda") for _ in range(6)]))
    torch.cuda.synchronize()
    for i in range(6):
        for st, ctx, Q, codes, scale, tables, lengths, outs in state:
            ctx.cache_attend(Q, codes, scale, tables, lengths, 16, outs[i])
    torch.cuda.synchronize()
    for want, (st, ctx, *_, outs) in zip(alone, state):
        assert all(torch.equal(o, want) for o in outs)
        ctx.close()
