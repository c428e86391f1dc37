"""The gradient of a lookup against differences of lookups, in numbers that leave nothing to round."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("kind", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,M,K", [(300, 3, 40), (4096, 4, 256), (6000, 3, 256), (6000, 9, 7), (66047, 8, 256)])
def test_lookup_grad_is_the_difference_of_lookups(T, M, K, kind):
    """f(C) = <w, lookup(C)> with whole numbers: C and E to 8, w to 8, the factor 1.5.  An element of a lookup is 1.5 times a whole number to
    16 M, one of the gradient 1.5 times one to 8 T < 2^20: both are fp32 numbers, and so is every sum on the way.  So f(C + E) - f(C - E) = 2 <dC, E>
    without any error, for E over all codewords and for single elements of them."""
    from paper_1509_05194_amd import hclae
    V, D = 200, 16
    rng = np.random.default_rng(T + K)
    C, E = (torch.from_numpy(rng.integers(-8, 9, (M, K, D)).astype(np.float32)).cuda() for _ in range(2))
    w = torch.from_numpy(rng.integers(-8, 9, (T, D))).cuda().to(kind)
    ids = torch.from_numpy(rng.integers(0, 256, (V, M)).astype(np.uint8)).cuda()    # codes of K or more are K - 1
    rows = torch.from_numpy(rng.integers(-2, V + 2, T)).cuda()                      # some of no row
    ctx = hclae.Context(T, D, M, K)
    dC, out = torch.full((M, K, D), float("nan"), device="cuda"), torch.empty((T, D), device="cuda")
    ctx.lookup_grad(ids, w, dC, rows=rows, scale=1.5)

    def f(c):
        ctx.lookup(ids, c, out, rows=rows, scale=1.5)
        return float((w.double() * out.double()).sum())

    slope = f(C + E) - f(C - E)
    assert slope != 0                                       # and nothing is allowed for: a gradient of zeros would not do
    assert slope == 2 * float((dC.double() * E.double()).sum())
    for m, k, d in zip(rng.integers(0, M, 20), rng.integers(0, K, 20), rng.integers(0, D, 20)):
        one = torch.zeros_like(C)
        one[m, k, d] = 1
        assert f(C + one) - f(C - one) == 2 * float(dC[m, k, d]), (m, k, d)
    ctx.close()
