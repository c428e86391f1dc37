"""Attention over a cache of codes where scores are infinite: a row whose score is -infinity weighs nothing, whatever rows it shares a tile, a window or a part of
its sequence with; +infinity makes its query head's outputs NaN, and nobody else's.

Tolerance of an output, U = 2^-24: a finite score is off by d = (D + M + 8) U sum |q c|, an exponential by that and 2^-21, sums of n terms by (n + 4) U, and weights are held to U of
their sum."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
D, M, K, PAGE = 64, 2, 256, 16
# query heads: a positive and a negative product with every key, and two products of zero
HEADS = (1.0, -0.5, 0.0, 0.25)


def check(n, key_scale, kind, R, B=1, value_nan=None):
    """Every row's keys sum to 1 in the first coordinate; key_scale[n] says the rest."""
    from paper_1509_05194_amd import hclae
    rng = np.random.default_rng(n + R)
    C = np.zeros((2, M, K, D), np.float32)
    C[0, 0, :, 0] = 1.0
    C[1] = rng.standard_normal((M, K, D))
    codes = rng.integers(0, K, (-(-n // PAGE) * PAGE, 2, M)).astype(np.uint8)
    scale = np.ones((codes.shape[0], 2), np.float32)
    scale[:n, 0] = key_scale
    scale[:, 1] = rng.uniform(0.5, 2.0, codes.shape[0])
    if value_nan is not None:
        scale[value_nan, 1] = np.nan
    Q = np.zeros((R, D), np.float32)
    Q[:, 0] = HEADS[:R]
    ctx = hclae.Context(B, D, M, K)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    tables = torch.arange(codes.shape[0] // PAGE, dtype=torch.int32, device="cuda").repeat(B, 1)
    out = torch.full((B, R, D), 7.0, dtype=TYPES[kind], device="cuda")
    lse = torch.full((B, R), 7.0, device="cuda")
    ctx.cache_attend(torch.from_numpy(Q).to(TYPES[kind]).cuda().repeat(B, 1, 1), torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda(), tables,
                     torch.full((B,), n, dtype=torch.int32, device="cuda"), PAGE, out, factor=1.0, lse=lse)
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    ctx.close()
    v = C[1].astype(np.float64)[np.arange(M)[None], codes[:n, 1]].sum(1) * scale[:n, 1].astype(np.float64)[:, None]
    for r in range(R):
        # the products and what fits a float, as in 32 bits
        with np.errstate(all="ignore"):
            s = (np.float32(Q[r, 0]) * scale[:n, 0]).astype(np.float64)
            s = np.where(np.abs(s) * np.log2(np.e) > np.finfo(np.float32).max, np.sign(s) * np.inf, s)
            if not (s < np.inf).all():
                y, l = np.full(D, np.nan), np.nan
            elif (s == -np.inf).all():
                y, l = np.zeros(D), -np.inf
            else:
                p = np.exp(s - s.max())
                l = s.max() + np.log(p.sum())
                p /= p.sum()
                y = p @ v
        if value_nan is not None:
            y = np.full(D, np.nan)
        rel = 0.0
        if np.isfinite(l):
            rel = (D + M + 8) * U * np.abs(s[np.isfinite(s)]).max() + 2.0 ** -21 + (n + 4) * U
        t = torch.finfo(TYPES[kind])
        for b in range(B):
            assert np.array_equal(np.isnan(got[b, r]), np.isnan(y)), (r, got[b, r, :4], y[:4])
            if not np.isnan(y).any():
                tol = (2 * rel * (p @ np.abs(v)) + n * U * np.abs(v).max() if np.isfinite(l) else 0) + t.tiny * t.eps / 2
                off = np.abs(got[b, r] - y)
                assert (off <= tol + t.eps / 2 * (np.abs(y) + tol)).all(), (r, off.max())
            if np.isfinite(l):
                assert abs(got_lse[b, r] - l) <= rel + 2 * U * abs(l), (r, got_lse[b, r], l)
            else:
                assert got_lse[b, r] == l or (np.isnan(l) and np.isnan(got_lse[b, r])), (r, got_lse[b, r], l)


def lost_rows(n, which):
    at = np.arange(n)
    return {"first": at < 1, "last": at == n - 1, "half": at < (n + 1) // 2, "but_last": at < n - 1, "tail": at >= 32, "all": at >= 0, "every_other": at % 2 == 0,
            "parts": at // 256 % 2 == 0}[which]


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("R", [1, 2, 4])
@pytest.mark.parametrize("which", ["first", "last", "half", "but_last", "tail", "all", "every_other", "parts"])
@pytest.mark.parametrize("n", [33, 200, 513, 2500])
def test_scores_of_minus_infinity(n, which, R, kind):
    """Infinite scales, and finite ones that leave a score beyond a float."""
    g = np.linspace(-1, 2, n).astype(np.float32)
    g[lost_rows(n, which)] = -np.inf
    check(n, g, kind, R)
    g[lost_rows(n, which)] = -3.3e38             # times log2(e), as scores are kept: beyond a float for the first head alone
    check(n, g, kind, R)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("which", ["half", "but_last", "parts"])
def test_windows_of_minus_infinity(which, kind):
    """Parts of several windows, 2048 rows each: more sequences than there are blocks at once."""
    n = 2 * 2048 + 1
    g = np.linspace(-1, 2, n).astype(np.float32)
    g[lost_rows(n, which)] = -np.inf
    check(n, g, kind, 4, B=1024)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [33, 200, 2500])
def test_rows_that_weigh_nothing_take_part(n, kind):
    """A value whose scale is NaN makes its heads' outputs NaN, also where all rows weigh nothing."""
    g = np.linspace(-1, 2, n).astype(np.float32)
    g[n - 1] = -np.inf
    check(n, g, kind, 4, value_nan=n - 1)
    g[:] = -np.inf
    check(n, g, kind, 4, value_nan=n - 1)
