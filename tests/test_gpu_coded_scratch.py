"""What a context keeps for coded caches and tables, beside its other calls and from one size of call to another."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


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
