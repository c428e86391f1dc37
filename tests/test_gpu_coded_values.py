"""Values at which the kernels of a coded cache could disagree with the definition of a write: rows in fp32, distances in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def quantise(x, C, scaled):
    """codes [n][M] of the fp32 rows x of one head, and their scales."""
    g = np.abs(x).max(1)
    r = np.where((g > 0)[:, None], x / np.where(g > 0, g, 1)[:, None], x).astype(np.float32) if scaled else x.copy()
    codes = np.zeros((len(x), C.shape[0]), np.uint8)
    for m in range(C.shape[0]):
        c = C[m].astype(np.float64)
        for i in range(len(r)):
            codes[i, m] = ((r[i].astype(np.float64) - c) ** 2).sum(1).argmin()
        r = r - C[m][codes[:, m]]
    return codes, g


def written(x, C, scaled):
    """The codes and scales of rows [n][H][D] with the dictionaries [H][M][K][D]."""
    from paper_1509_05194_amd import hclae
    n, H, D = x.shape
    M, K = C.shape[1:3]
    ctx = hclae.Context(n, D, M, K)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    codes = torch.full((n, H, M), 251, dtype=torch.uint8, device="cuda")
    scale = torch.full((n, H), -3.0, device="cuda") if scaled else None
    ctx.cache_write(torch.from_numpy(x).cuda(), torch.arange(n, device="cuda"), codes, scale)
    torch.cuda.synchronize()
    ctx.close()
    return codes.cpu().numpy(), scale.cpu().numpy() if scaled else None


@pytest.mark.parametrize("top", [1.8e19, 2.5e19])
@pytest.mark.parametrize("n", [6, 1100, 4200])              # a row a block, sixteen, tiles
@pytest.mark.parametrize("K,D", [(255, 64), (200, 128), (129, 36), (127, 64), (100, 132), (63, 64), (20, 128), (256, 64)])
def test_write_of_codewords_whose_squares_are_near_the_largest_number(n, K, D, top):
    """Codewords of norms from 1.45e19 on, -||c||^2 / 2 from -1.05e38 to -1.7e38 or -3.1e38 (where the square itself is infinite); rows of
    zeros, near zero, and among the codewords."""
    rng = np.random.default_rng(K + D)
    way = rng.standard_normal((2, 2, K, D))
    C = (way / np.linalg.norm(way, axis=3, keepdims=True) * rng.uniform(1.45e19, top, (2, 2, K, 1))).astype(np.float32)
    x = (rng.standard_normal((n, 2, D)) * 10.0 ** rng.integers(14, 19, (n, 1, 1))).astype(np.float32)
    x[1] = 0
    x[2] = C[:, 0, K // 2]
    x[3] = 0.5 * C[:, 0, K - 1]
    codes, _ = written(x, C, False)
    for h in range(2):
        assert np.array_equal(codes[:, h], quantise(x[:, h], C[h], False)[0])


@pytest.mark.parametrize("n", [40, 1100, 4200, 9001])       # a row a block, sixteen, tiles of half and of all waves
@pytest.mark.parametrize("D", [64, 128, 200])
def test_write_of_rows_whose_quotients_are_halfway_between_subnormal_numbers(n, D):
    """g = 2 G and x = (2 j + 1) G 2^-149 with odd G: x / g is halfway between two numbers, and the even one is x / g in fp32.  The last
    dictionary holds what rows leave with that rounding and with that of the product with a rounded 1 / g, side by side."""
    rng = np.random.default_rng(D)
    base, x, twin = 32, np.zeros((32, D), np.float32), np.zeros((32, D), np.float32)
    for i in range(base):
        while True:
            G = 2 * int(rng.integers(3, 200)) + 1
            x[i] = ((2 * rng.integers(0, 2000, D) + 1) * G * (1 - 2 * rng.integers(0, 2, D))).astype(np.float32) * np.float32(2.0 ** -149)
            x[i, 0] = 2 * G
            twin[i] = (x[i].astype(np.float64) * (1.0 / np.float64(2 * G))).astype(np.float32)
            if (twin[i] != x[i] / np.float32(2 * G)).any():
                break
    u = x / x[:, :1]
    assert (np.abs(u[:, 1:]) < 2.0 ** -126).all()           # zero among them, where j is 0
    C = np.zeros((1, 2, 2 * base, D), np.float32)
    C[0, 0, :, 0] = 1 + np.arange(2 * base)                 # the first codeword leaves zero in front
    C[0, 1, 0::2], C[0, 1, 1::2] = twin, u
    C[0, 1, :, 0] = 0
    rows = x[np.arange(n) % base][:, None]
    codes, scale = written(rows, C, True)
    want, g = quantise(rows[:base, 0], C[0], True)
    assert np.array_equal(want[:, 1], 2 * np.arange(base) + 1)
    assert np.array_equal(codes[:, 0], want[np.arange(n) % base]) and np.array_equal(scale[:, 0], g[np.arange(n) % base])


@pytest.mark.parametrize("n", [40, 1100, 4200])
def test_write_of_rows_whose_products_are_subnormal(n):
    """Codeword 2 has 255 products of 1.1e-38 with the row, which are 2.8e-36 together and nearer than codeword 1 by 0.8e-36 in the score; without
    them codeword 1 would lead by more than 2e-36."""
    D, K = 256, 40
    x = np.full((n, 1, D), 1e-19, np.float32)
    x[:, :, 0] = 1e-18
    C = np.full((1, 1, K, D), 1e-17, np.float32)
    C[0, 0, 1] = 0
    C[0, 0, 1, 0] = 1e-18
    C[0, 0, 2] = 1.1e-19
    C[0, 0, 2, 0] = 0
    want = quantise(x[:1, 0], C[0], False)[0]
    assert want[0, 0] == 2
    assert np.array_equal(written(x, C, False)[0][:, 0], np.repeat(want, n, 0))


@pytest.mark.parametrize("T", [900, 9000])
def test_gradient_of_rows_that_take_no_part_may_be_anything(T):
    from paper_1509_05194_amd import hclae
    V, D, M, K = 100, 20, 3, 256
    gen = torch.Generator().manual_seed(T)
    ids = torch.randint(0, K, (V, M), dtype=torch.uint8, generator=gen).cuda()
    rows = torch.randint(-V, 2 * V, (T,), generator=gen).cuda()
    g = torch.randint(-8, 9, (T, D), generator=gen).float().cuda()
    out = (rows < 0) | (rows >= V)
    clean = torch.where(out[:, None], 0.0, g)
    g[out] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], device="cuda").repeat(D // 4)
    ctx = hclae.Context(T, D, M, K)
    dC, want = (torch.full((M, K, D), float("nan"), device="cuda") for _ in range(2))
    ctx.lookup_grad(ids, g, dC, rows=rows)
    ctx.lookup_grad(ids, clean, want, rows=rows)
    assert torch.equal(dC, want) and bool((dC != 0).any()) and bool(dC.isfinite().all())
    ctx.close()


def test_dictionaries_laid_out_again_inside_a_graph():
    """cache_begin, a write and the read of it recorded together: every replay takes what C holds by then."""
    from paper_1509_05194_amd import hclae
    n, H, D, M, K = 1500, 2, 64, 3, 100
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = hclae.Context(n, D, M, K)
        C, X = torch.randn((H, M, K, D), device="cuda"), torch.randn((n, H, D), device="cuda")
        slots, starts = torch.randperm(n, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
        tables = torch.arange(n // 4, dtype=torch.int32, device="cuda")[None]
        codes, scale, out = torch.zeros((n, H, M), dtype=torch.uint8, device="cuda"), torch.zeros((n, H), device="cuda"), torch.zeros((n, H, D), device="cuda")

        def work():
            ctx.cache_begin(C)
            ctx.cache_write(X, slots, codes, scale)
            ctx.cache_read(codes, scale, tables, starts, 4, out)

        work()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            work()
        for i in range(3):
            C.copy_(torch.randn((H, M, K, D), generator=torch.Generator().manual_seed(i)).cuda())
            graph.replay()
            torch.cuda.synchronize()
            got = codes.clone(), scale.clone(), out.clone()
            out.zero_()
            work()
            torch.cuda.synchronize()
            assert torch.equal(codes, got[0]) and torch.equal(scale, got[1]) and torch.equal(out, got[2])
        ctx.close()


@pytest.mark.parametrize("n", [40, 1100, 4200])
@pytest.mark.parametrize("spread", [1e-44, 1e-40, 2e-38, 1e37])
def test_write_of_rows_whose_scales_are_at_the_ends_of_the_range(n, spread):
    """Rows of subnormal numbers, and rows up to the largest ones: divided by their scale they are ordinary."""
    rng = np.random.default_rng(n)
    D, M, K = 100, 3, 70
    x = np.clip(rng.standard_normal((n, 1, D)) * spread, -3.4e38, 3.4e38).astype(np.float32)
    C = (rng.standard_normal((1, M, K, D)) * 0.5 ** np.arange(M)[None, :, None, None]).astype(np.float32)
    codes, scale = written(x, C, True)
    want, g = quantise(x[:, 0], C[0], True)
    assert np.array_equal(codes[:, 0], want) and np.array_equal(scale[:, 0], g)
