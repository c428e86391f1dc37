"""What a context keeps for coded caches and tables, beside its other calls and from one size of call to another."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U32 = 2.0 ** -24


def test_cache_and_gradient_beside_multi_path_encoding():
    """Dictionaries learned by a sweep, a table encoded with several paths, its gradient, and a cache with the same dictionaries, all in one
    context, eager and recorded: the multi-path scratch grows twice in between, and every later call gives the bits of the first."""
    from paper_1509_05194_amd import hclae, synth
    n, D, M, K, page = 6000, 32, 4, 64, 16
    x = torch.from_numpy(synth.tiny_gmm(N=n, D=D)).cuda()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = hclae.Context(n, D, M, K)
        C, codes, r = torch.zeros((M, K, D), device="cuda"), torch.zeros((n, M), dtype=torch.uint8, device="cuda"), x.clone()
        ctx.sweep(C, codes, r, 3, init_idx=synth.init_indices(n, M, K))
        g = torch.randn((n, D), generator=torch.Generator().manual_seed(1)).cuda()
        rows = torch.randint(-1, n, (n,), generator=torch.Generator().manual_seed(2)).cuda()
        slots = torch.randperm(n, generator=torch.Generator().manual_seed(3)).cuda()
        tables = torch.arange(n // page, dtype=torch.int32, device="cuda")[None]
        starts = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        kept, scale = torch.zeros((n, 1, M), dtype=torch.uint8, device="cuda"), torch.zeros((n, 1), device="cuda")
        out, dC = torch.zeros((n, 1, D), device="cuda"), torch.zeros((M, K, D), device="cuda")
        results = (kept, scale, out, dC)
        table = codes.clone()

        def work():
            ctx.cache_write(x[:, None], slots, kept, scale)
            ctx.cache_read(kept, scale, tables, starts, page, out)
            ctx.lookup_grad(table, g, dC, rows=rows)

        ctx.cache_begin(C[None])
        work()
        torch.cuda.synchronize()
        want = [t.clone() for t in results]
        assert all(bool((t != 0).any()) for t in want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            work()
        coded = []
        for L in (2, 8, 8):                                # sized, grown, as it was
            res = torch.empty_like(x)
            ctx.encode_beam(x, C, L, codes, res)
            torch.cuda.synchronize()
            coded.append(codes.clone())
            filler = [torch.full((1 << 18,), float("nan"), device="cuda") for _ in range(8)]   # whatever is free now, is used
            for again in (work, graph.replay):
                for t in results:
                    t.zero_()
                again()
                torch.cuda.synchronize()
                for t, w in zip(results, want):
                    assert torch.equal(t, w), (L, again)
            assert all(bool(f.isnan().all()) for f in filler)
        assert torch.equal(coded[1], coded[2])
        # other dictionaries, and more heads of them, in the room there is and beyond it
        for H in (1, 3):
            heads = torch.stack([C + h for h in range(H)])
            ctx.cache_begin(heads)
            k2, s2 = torch.zeros((n, H, M), dtype=torch.uint8, device="cuda"), torch.zeros((n, H), device="cuda")
            ctx.cache_write(x[:, None].expand(n, H, D), slots, k2, s2)
            assert torch.equal(k2[:, :1], want[0]) and torch.equal(s2[:, :1], want[1])
        ctx.encode_beam(x, C, 10, codes, res)
        torch.cuda.synchronize()
        ctx.close()


def codes_and_rows(T, V, M, K, seed):
    """A table of V rows of codes, and T row numbers: a tenth of them of one row, some of none."""
    rng = np.random.default_rng(seed)
    ids = torch.from_numpy(rng.integers(0, K, (V, M)).astype(np.uint8)).cuda()
    rows = torch.from_numpy(rng.integers(0, V, T)).cuda()
    rows[5:5 + T // 10] = 3
    rows[[0, T // 2]] = torch.tensor([-1, V], device="cuda")
    return ids, rows


def check_grad(dC, ids, rows, g, V, factor):
    """A gradient is a sum of n values in fp32, in some order, times the factor: (n + 2) 2^-24 of the sum of their magnitudes."""
    rows, ids, dC = rows.cpu(), ids.cpu(), dC.cpu().double()
    live = (rows >= 0) & (rows < V)
    gd, at = g.cpu().double()[live], ids[rows[live]].long()
    M, K, D = dC.shape
    for m in range(M):
        c = at[:, m]
        want = torch.zeros((K, D), dtype=torch.float64).index_add_(0, c, gd) * factor
        mag = torch.zeros((K, D), dtype=torch.float64).index_add_(0, c, gd.abs()) * abs(factor)
        n = torch.bincount(c, minlength=K).double()[:, None]
        assert bool(((dC[m] - want).abs() <= (n + 2) * U32 * mag * (1 + 2.0 ** -8)).all()), m


# Where the rows of an item grow (its last number of rows before, and the first), where the ranges of the sort do, both in contexts of
# just that size; dictionaries from few to the most there can be.
@pytest.mark.parametrize("T,M,K", [(65663, 8, 256), (65664, 8, 256), (66047, 8, 256), (66048, 8, 256), (66047, 64, 256), (66047, 256, 64), (98304, 8, 256),
                                   (98305, 8, 256), (98815, 8, 256), (98815, 64, 256), (131583, 9, 256), (164351, 3, 256), (197119, 3, 255), (229887, 3, 256),
                                   (32768, 8, 256), (32769, 8, 256), (131072, 3, 256), (131073, 3, 256), (524288, 2, 256), (524289, 2, 256),
                                   (262143, 2, 1), (262145, 2, 1)])
def test_gradient_where_items_and_ranges_grow(T, M, K):
    from paper_1509_05194_amd import hclae
    V, D = 1000, 12
    ids, rows = codes_and_rows(T, V, M, K, T)
    g = torch.randn((T, D), generator=torch.Generator().manual_seed(T)).cuda()
    ctx = hclae.Context(T, D, M, K)
    dC = torch.full((M, K, D), float("nan"), device="cuda")
    ctx.lookup_grad(ids, g, dC, rows=rows, scale=0.5)
    torch.cuda.synchronize()
    check_grad(dC, ids, rows, g, V, 0.5)
    ctx.close()


def test_gradients_of_fewer_rows_than_a_context_has_room_for():
    """One context for more than a million rows: the bits of contexts of just the size, whatever was summed before."""
    from paper_1509_05194_amd import hclae
    V, D, M, K, most = 3000, 8, 8, 256, (1 << 20) + 70001
    ids, rows = codes_and_rows(most, V, M, K, 1)
    g = torch.randn((most, D), generator=torch.Generator().manual_seed(2)).cuda()
    big = hclae.Context(most, D, M, K)
    for T in (5000, most, 66047, 4097, 32769, 524288, 98815, 131072, 700001, 4096, 229887, most - 1):
        dC, alone = (torch.full((M, K, D), float("nan"), device="cuda") for _ in range(2))
        big.lookup_grad(ids, g[:T], dC, rows=rows[:T])
        ctx = hclae.Context(T, D, M, K)
        ctx.lookup_grad(ids, g[:T], alone, rows=rows[:T])
        torch.cuda.synchronize()
        assert torch.equal(dC, alone), T
        check_grad(dC, ids, rows[:T], g[:T], V, 1.0)
        print("gradient of %d rows" % T, flush=True)
        ctx.close()
    big.close()


def test_calls_after_one_that_found_no_memory():
    """Scratch for a sorted gradient of 256 dictionaries and 330 million rows is more than a device has: the call says so, and the next
    ones, which need none of it, are not blamed for it."""
    from paper_1509_05194_amd import hclae
    T, V, D, M, K = 5000, 300, 4, 256, 256
    ids, rows = codes_and_rows(T, V, M, K, 4)
    g, C = torch.randn((T, D), device="cuda"), torch.randn((M, K, D), device="cuda")
    assert 330_000_000 * M * 4 > torch.cuda.get_device_properties(0).total_memory
    ctx = hclae.Context(330_000_000, D, M, K)
    dC, out = torch.full((M, K, D), 5.0, device="cuda"), torch.empty((T, D), device="cuda")
    for _ in range(2):
        with pytest.raises(hclae.HclaeError, match="HCLAE_ENOMEM"):
            ctx.lookup_grad(ids, g, dC, rows=rows)
        ctx.lookup(ids, C, out, rows=rows)
    assert bool((dC == 5.0).all())
    ctx.lookup_grad(ids, g[:4096], dC, rows=rows[:4096])
    torch.cuda.synchronize()
    check_grad(dC, ids, rows[:4096], g[:4096], V, 1.0)
    ctx.close()
