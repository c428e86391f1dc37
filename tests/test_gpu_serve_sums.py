"""What attention over a cache of codes adds up is held in 32 bits or more, for outputs of 16 bits too: small weights beside large ones, small differences of
large sums.  Tolerances are counted, with U = 2^-24 half a step of a float."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def attend(C, codes, Q, kind, page, B, factor=1.0):
    """The same sequence B times over: out [G R][D] in 64 bits, after a look at all B being equal."""
    from paper_1509_05194_amd import hclae
    n = codes.shape[0]
    pages = -(-n // page)
    M, K, D = C.shape[1:]
    ctx = hclae.Context(B, D, M, K)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    room = torch.zeros((pages * page,) + codes.shape[1:], dtype=torch.uint8)
    room[:n] = torch.from_numpy(codes)
    tables = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(B, 1)
    out = torch.full((B,) + Q.shape, 7.0, dtype=TYPES[kind], device="cuda")
    ctx.cache_attend(torch.from_numpy(Q).to(TYPES[kind]).cuda().repeat(B, 1, 1), room.cuda(), None, tables, torch.full((B,), n, dtype=torch.int32, device="cuda"), page, out,
                     factor=factor)
    got = out.double().cpu().numpy()
    ctx.close()
    assert (got == got[:1]).all()
    return got[0]


def half_step(y, kind):
    t = torch.finfo(TYPES[kind])
    return t.eps / 2 * np.abs(y) + t.tiny * t.eps / 2


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("R,B", [(1, 1), (2, 1), (4, 1), (4, 64)])
@pytest.mark.parametrize("M", [1, 9])
def test_weights_far_below_the_largest(M, R, B, kind):
    """One row weighs 2^19 times as much as each other and has a value of zeros: the others' weights are what the output is made of.

    A weight is held to 2^-24 of the sum of all weights; a score is off by d = (D + M + 8) U sum |q c|, an exponential by 2^-21 more, and a sum of n terms by (n + 4) U."""
    n, D, G, K = 512, 64, 8, 256
    rng = np.random.default_rng(R + M)
    C = np.zeros((2 * G, M, K, D), np.float32)
    C[:G, 0, 1, 0] = 19 * np.log(2.0)
    for k in range(1, K):
        C[G:, 0, k, k % D] = 1024.0
    codes = np.zeros((n, 2 * G, M), np.uint8)
    codes[:, G:, 0] = rng.integers(1, K, (n, G))
    top = 100
    codes[top, :G, 0], codes[top, G:, 0] = 1, 0
    Q = np.zeros((G * R, D), np.float32)
    Q[:, 0] = 1.0
    got = attend(C, codes, Q, kind, 16, B)
    score = np.where(np.arange(n) == top, np.float64(C[0, 0, 1, 0]), 0.0)
    p = np.exp(score)
    p /= p.sum()
    d = (D + M + 8) * U * score.max()
    for h in range(G):
        x = C[G + h, 0].astype(np.float64)[codes[:, G + h, 0]]
        y = p @ x
        tol = 2 * (d + 2.0 ** -21 + (n + 4) * U) * (p @ np.abs(x)) + U * np.abs(x).sum(0)
        for r in range(R):
            off = np.abs(got[h * R + r] - y)
            assert (off <= tol + half_step(np.abs(y) + tol, kind)).all(), (h, r, np.nanmax(off / tol))


@pytest.mark.parametrize("R,B", [(1, 1), (2, 1), (4, 1), (4, 64)])
@pytest.mark.parametrize("M", [1, 9])
def test_difference_of_large_sums(M, R, B):
    """Half of the rows have 1 + f as their value and half -1, all the same weight: f / 2 is left.

    With equal scores weights, their sums and what they are divided by are powers of two.  A float as its three parts adds up without a rounding, and the two
    products differ by a number that a float holds; eight roundings of numbers below 2 are granted."""
    n, D, G, K, kind = 512, 64, 8, 256, "fp16"
    rng = np.random.default_rng(R + M)
    C = np.zeros((2 * G, M, K, D), np.float32)
    C[G:, 0, 1] = 1 + rng.uniform(2.0 ** -9, 2.0 ** -8, (G, D))
    C[G:, 0, 2] = -1
    codes = np.zeros((n, 2 * G, M), np.uint8)
    codes[:, G:, 0] = 1 + rng.permuted(np.arange(n * G).reshape(n, G) // G % 2, axis=0)
    got = attend(C, codes, np.zeros((G * R, D), np.float32), kind, 16, B)
    for h in range(G):
        y = (C[G + h, 0, 1].astype(np.float64) - 1) / 2
        for r in range(R):
            off = np.abs(got[h * R + r] - y)
            assert (off <= half_step(y, kind) + 8 * 2 * U).all(), (h, r, off.max())
