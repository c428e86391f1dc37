"""Attention over a cache of codes with codewords that are not finite: they count in the rows that have them, and nowhere else.  And with the largest ones."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
PAGE = 16


def attend(C, codes, Q, kind, B):
    from paper_1509_05194_amd import hclae
    n, (H, M, K, D) = codes.shape[0], C.shape
    ctx = hclae.Context(B, D, M, K)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    tables = torch.arange(n // PAGE, dtype=torch.int32, device="cuda").repeat(B, 1)
    out = torch.full((B,) + Q.shape, 7.0, dtype=TYPES[kind], device="cuda")
    lse = torch.full((B, Q.shape[0]), 7.0, device="cuda")
    ctx.cache_attend(torch.from_numpy(Q).to(TYPES[kind]).cuda().repeat(B, 1, 1), torch.from_numpy(codes).cuda(), None, tables,
                     torch.full((B,), n, dtype=torch.int32, device="cuda"), PAGE, out, factor=1.0, lse=lse)
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    ctx.close()
    for b in range(1, B):
        assert np.array_equal(got[b], got[0], equal_nan=True) and np.array_equal(got_lse[b], got_lse[0], equal_nan=True)
    return got[0], got_lse[0]


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("n,R,B", [(32, 1, 1), (160, 4, 1), (512, 2, 1), (4096, 4, 1), (48, 1, 300), (512, 4, 128), (512, 5, 128)])
def test_codewords_that_are_not_finite(n, R, B, kind):
    """Outputs are those with zeros in place of the codewords that no row has; a value that some row has makes its coordinates infinite or NaN."""
    rng = np.random.default_rng(n)
    G, M, K, D = 2, 3, 32, 36
    C = rng.standard_normal((2 * G, M, K, D)).astype(np.float32)
    codes = rng.integers(0, K - 4, (n, 2 * G, M)).astype(np.uint8)
    Q = rng.standard_normal((G * R, D)).astype(np.float32)
    C[:, :, K - 4:] = 0
    want, want_lse = attend(C, codes, Q, kind, B)
    C[:, 0, K - 1] = np.nan
    C[:, 1, K - 2, ::3] = np.inf
    C[:, 2, K - 3, 1::2] = -np.inf
    got, got_lse = attend(C, codes, Q, kind, B)
    # finite as before, in another order of sums: both are within (M K + 8) U of the values' sizes of what is meant
    tol = 2 * (M * K + 8) * U * np.abs(C[np.isfinite(C)]).max() * M + 2 * torch.finfo(TYPES[kind]).eps * np.abs(want)
    assert (np.abs(got - want) <= tol).all() and np.array_equal(got_lse, want_lse)
    codes[n // 2, G, 1] = K - 2                    # a value of head 0
    codes[n // 3, G + 1, 0] = K - 1                # and one of head 1
    got, _ = attend(C, codes, Q, kind, B)
    assert np.isfinite(np.delete(got[:R], np.s_[::3], 1)).all()
    for r in range(G * R):
        h = r // R
        s = C[h].astype(np.float64)[np.arange(M)[None], codes[:, h]].sum(1) @ torch.from_numpy(Q[r]).to(TYPES[kind]).double().numpy()
        p = np.exp(s - s.max())[n // 2 if h == 0 else n // 3] / np.exp(s - s.max()).sum()
        # a weight is held to 2^-24 of the weights' sum: a smaller one may be no step, and its row's value then counts as finite ones of that weight do
        lost = np.array_equal(got[r], want[r]) or np.isfinite(got[r]).all()
        made = (got[r, ::3] == np.inf).all() if h == 0 else np.isnan(got[r]).all()
        assert made or (p < 2.0 ** -24 and lost), (r, p)


@pytest.mark.parametrize("n,B", [(64, 1), (512, 1), (512, 128)])
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_the_largest_codewords(n, B, kind):
    """Values of 3.4e38, which 16 bits round to infinity, that cancel."""
    G, R, M, K, D = 1, 4, 1, 4, 32
    C = np.zeros((2 * G, M, K, D), np.float32)
    C[1, 0, 1], C[1, 0, 2] = 3.4e38, -3.4e38
    codes = np.zeros((n, 2 * G, M), np.uint8)
    codes[:, 1, 0] = np.arange(n) % 4              # zero, plus, minus, zero
    codes[3::4, 1, 0] = 1
    got, _ = attend(C, codes, np.zeros((G * R, D), np.float32), kind, B)
    if n <= 320:                                   # rows decoded: 32 times 3.4e38 of one sign, weights of 1 before their division, are beyond a float
        assert not np.isfinite(got).any()
        return
    y = float(C[1, 0, 1, 0]) / 4                   # weights of 1 / n: powers of two
    assert (np.abs(got - y) <= (torch.finfo(TYPES[kind]).eps / 2 + 2 * n * U) * y).all(), got[0, :4] / y


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [64, 512, 4096])
def test_queries_that_are_not_finite(n, kind):
    """They are NaN or zero, and their neighbours as they are without them."""
    rng = np.random.default_rng(n)
    G, R, M, K, D = 2, 4, 8, 256, 64
    C = rng.standard_normal((2 * G, M, K, D)).astype(np.float32)
    codes = rng.integers(0, K, (n, 2 * G, M)).astype(np.uint8)
    Q = rng.standard_normal((G * R, D)).astype(np.float32)
    want, want_lse = attend(C, codes, Q, kind, 1)
    Q[1, 3], Q[2, 5], Q[6, 7] = np.inf, np.nan, -np.inf
    got, got_lse = attend(C, codes, Q, kind, 1)
    others = [0, 3, 4, 5, 7]
    assert np.array_equal(got[others], want[others]) and np.array_equal(got_lse[others], want_lse[others])
    for r in (1, 2, 6):
        assert np.isnan(got[r]).all() or (got[r] == 0).all()
