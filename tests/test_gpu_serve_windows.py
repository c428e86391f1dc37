"""Attention over a cache of codes in blocks that take several windows of 2048 rows one after the other: more sequences than the card holds blocks, so that each is one part.
The sequences are copies of a few; equal ones give equal bits, one of each is held to the 64-bit form of test_gpu_serve."""
import numpy as np
import pytest

from test_gpu_serve import U, Case, half_step

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

WINDOW = 2048
COPIES = 512                                       # of each: with two, and two key heads, 2048 blocks


def run(c, copies=COPIES, begins=None):
    """A case's sequences `copies` times over: out and lse of one of each, after a look at all."""
    from paper_1509_05194_amd import hclae
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    ctx = hclae.Context(c.B * copies, c.D, c.M, c.K)
    ctx.cache_begin(dev(c.C))
    out = torch.full((c.B * copies, c.G * c.R, c.D), 7.0, dtype=c.kind, device="cuda")
    lse = torch.full((c.B * copies, c.G * c.R), 7.0, device="cuda")
    lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda").repeat(copies)
    ctx.cache_attend(c.Q.cuda().repeat(copies, 1, 1), dev(c.codes), dev(c.scale), dev(c.tables).repeat(copies, 1), lens, c.page, out,
                     begins=None if begins is None else dev(begins).repeat(copies), lse=lse)
    torch.cuda.synchronize()
    ctx.close()
    for t in (out, lse):
        same = t.reshape((copies, c.B) + t.shape[1:])
        assert ((same == same[:1]) | (same.isnan() & same[:1].isnan())).all()
    return out[:c.B], lse[:c.B]


def hold(c, out, lse, begins=None):
    """The case's own look, and closer ones: weights held to 2^-24 of their sum, lse to a score's error and a sum's."""
    c.check(out, None, begins=begins)
    rel, tiny = half_step(c.kind)
    for b in range(c.B):
        for h in range(c.G):
            slots = c.rows(b, h, begins)
            k, ka, v = c.x(h, slots), c.x(h, slots, True), c.x(c.G + h, slots)
            for r in range(h * c.R, (h + 1) * c.R):
                q = c.Q[b, r].double().numpy()
                s = c.factor * (k @ q)
                d = (c.D + c.M + 8) * U * c.factor * (ka @ np.abs(q))
                with np.errstate(all="ignore"):
                    p = np.exp(s - s.max())
                    l, p = s.max() + np.log(p.sum()), p / p.sum()
                    g = np.abs(c.scale[slots, c.G + h]) if c.scale is not None else np.ones(len(slots))
                    # a row's own weight is off by 2 (d_t + ...) of itself, the sum they are divided by as well; decoded values by M U; steps of weights
                    off = 2 * (d + 2.0 ** -21) + (len(slots) + c.M + 8) * U
                    va = c.x(c.G + h, slots, True)
                    tol = (p * off) @ va + (p @ off) * (p @ va) + U * (p @ g) * len(slots) * np.abs(c.C[c.G + h]).max(1).sum(0)
                    tol = tol + rel * (np.abs(p @ v) + tol) + tiny
                    got = out[b, r].double().cpu().numpy()
                    assert not (np.abs(got - p @ v) > tol).any(), (b, r, np.nanmax(np.abs(got - p @ v) / tol))
                    assert np.array_equal(np.isnan(got), np.isnan(p @ v))
                    assert not abs(float(lse[b, r]) - l) > p @ d + 2.0 ** -21 + (len(slots) + 4) * U + 2 * U * abs(l), (b, r, float(lse[b, r]), l)
                    assert np.isnan(float(lse[b, r])) == np.isnan(l)


# RB 1, 2 and 4 query heads a block, 32 and 64 bits a sum, code rows by wide words, words and bytes, pages found by the wave
FORMS = [(1, "bf16", 8, 64, 256), (2, "fp16", 8, 64, 256), (4, "bf16", 8, 64, 256), (4, "fp16", 16, 16, 256), (4, "bf16", 16, 128, 256), (3, "fp32", 8, 64, 256), (2, "fp32", 16, 16, 256),
         (4, "fp16", 5, 24, 200), (4, "fp32", 4, 16, 100), (2, "bf16", 20, 16, 64)]


def case(form, lens, seed):
    R, kind, M, page, K = form
    return Case(lens, 2, R, 32, M, K, page, kind, True, seed=seed)


@pytest.mark.parametrize("form", FORMS)
def test_windows(form):
    """Lengths that end in a window's first row, its last, and between."""
    c = case(form, [3 * WINDOW + 1, 4 * WINDOW], 1)
    hold(c, *run(c))
    c = case(form, [3 * WINDOW - 1, 5000], 2)
    begins = np.array([130, 700], np.int32)
    hold(c, *run(c, begins=begins), begins=begins)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("shape", ["rise", "steps", "fall", "level", "last", "first"])
def test_scores_over_windows(shape, form):
    """The reference is raised in every window, in some, never again, and in the last row; running sums fade by as much."""
    n = 4 * WINDOW + 77
    c = case(form, [n], 3)
    slots = c.rows(0, 0)
    at = np.arange(n)
    ramp = {"rise": 1e-3 + 30.0 * at / n, "steps": np.array([1.0, 1.0, 9.0, 9.0, 30.0])[at // WINDOW], "fall": 30.0 * (1 - at / n) + 1e-3, "level": np.ones(n),
            "last": np.where(at == n - 1, 40.0, 0.5), "first": np.where(at == 0, 40.0, 0.5)}[shape]
    for h in range(2):
        c.scale[slots, h] = ramp
    hold(c, *run(c, 1024))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("shape", ["grow", "shrink", "one", "signs", "zeros"])
def test_value_scales_over_windows(shape, form):
    """The largest weight grows from window to window by more than the steps allow for, shrinks, stands out once, changes its sign, and is zero at first."""
    n = 4 * WINDOW + 77
    c = case(form, [n], 4)
    slots = c.rows(0, 0)
    at = np.arange(n)
    g = {"grow": 10.0 ** (at // WINDOW * 2.0 - 3), "shrink": 10.0 ** (3 - at // WINDOW * 2.0), "one": np.where(at == 3 * WINDOW + 5, 3e4, 1.0),
         "signs": np.where(at // 700 % 2 == 0, 1.0, -1.5), "zeros": np.where(at < 2 * WINDOW + 9, 0.0, 1.0)}[shape]
    if form[1] == "fp16":
        g = g / 100
    for h in range(2):
        c.scale[slots, h] = 0.5
        c.scale[slots, 2 + h] = g
    hold(c, *run(c, 1024))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("row", [5, WINDOW, 3 * WINDOW + 9, 4 * WINDOW + 76])
def test_nan_in_one_window(row, form):
    """A scale of NaN in any window: a key's makes its head's outputs NaN, a value's all but lse; the other head's are as they are."""
    n = 4 * WINDOW + 77
    c = case(form, [n], 5)
    want, want_lse = run(c, 1024)
    slot = c.rows(0, 0)[row]
    c.scale[slot, 0] = np.nan                      # a key of head 0
    c.scale[slot, 2 + 1] = np.nan                  # a value of head 1
    out, lse = run(c, 1024)
    assert torch.isnan(out).all() and torch.isnan(lse[0, :c.R]).all()
    # a weight that is no number has the reference looked for anew: the same exponentials (to 2^-21 and a rounding of their exponents, below 64) in another order of sums
    assert ((lse - want_lse)[0, c.R:].abs() <= 2 * (2.0 ** -21 + 64 * U + (n + 4) * U) + 2 * U * want_lse[0, c.R:].abs()).all()
    c.scale[slot, 0] = 1.0
    out, lse = run(c, 1024)
    assert torch.isnan(out[0, c.R:]).all() and not torch.isnan(out[0, :c.R]).any()
    c.scale[slot, 2 + 1] = 1.0
    hold(c, *run(c, 1024))


@pytest.mark.parametrize("form", FORMS)
def test_pages_that_are_not_there_over_windows(form):
    """Whole windows without a row, and rows without a scale array."""
    n = 5 * WINDOW
    c = case(form, [n], 6)
    page = c.page
    c.tables[0, WINDOW // page + 1:3 * WINDOW // page] = -1
    hold(c, *run(c, 1024))
    c.tables[0, :2 * WINDOW // page] = -1
    hold(c, *run(c, 1024))
    c.scale = None
    hold(c, *run(c, 1024))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("copies,n", [(1, 150), (1, 4 * WINDOW + 77), (1024, 4 * WINDOW + 77)])
def test_lse_joins_parts(copies, n, form):
    """Rows up to a place and those from it on, joined by lse, are the whole; few rows, parts of one window and of several."""
    c = case(form, [n], 7)
    whole, whole_lse = run(c, copies)
    hold(c, whole, whole_lse)
    for cut in (64, min(2 * WINDOW, n // 2), n - 1):
        begins = np.array([cut], np.int32)
        back, back_lse = run(c, copies, begins=begins)
        hold(c, back, back_lse, begins=begins)
        c.lens = [cut]
        front, front_lse = run(c, copies)
        hold(c, front, front_lse)
        c.lens = [n]
        top = torch.maximum(front_lse, back_lse).double()
        f, b = torch.exp(front_lse.double() - top), torch.exp(back_lse.double() - top)
        joined = (f[..., None] * front.double() + b[..., None] * back.double()) / (f + b)[..., None]
        # each side to its own error: scores as in hold, at most (D + M + 8) U factor sum |q| |x|, and three roundings to the type
        d = 0.0
        for h in range(2):
            slots = c.rows(0, h)
            ka = c.x(h, slots, True)
            for r in range(h * c.R, (h + 1) * c.R):
                d = max(d, (c.D + c.M + 8) * U * c.factor * (ka @ np.abs(c.Q[0, r].double().numpy())).max())
        big = max(np.abs(c.x(2 + h, c.rows(0, h), True)).max() for h in range(2))
        e = 2 * (d + 2.0 ** -21 + (n + 4) * U) + n * U
        assert (torch.log(f + b) + top - whole_lse.double()).abs().max() <= 2 * (d + 2.0 ** -21 + (n + 4) * U) + 4 * U * whole_lse.abs().max()
        assert ((joined - whole.double()).abs() <= 3 * e * big + torch.finfo(c.kind).eps * (whole.double().abs() + 3 * e * big) + 1e-7).all()
