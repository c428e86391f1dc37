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
