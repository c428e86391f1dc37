"""Serving from a paged cache of codes (hclae_cache_attend / select / extend / compact / copy) against plain 64-bit forms.

Tolerances of attention.  A score is a sum of M D products in fp32, in some order, times a scale and a factor: off by at most
d = (D + M + 8) 2^-24 factor g sum_m |q| . |c_m|, and an exponential by that and 2^-21 of itself (exponent and function).  An output is a quotient of two sums
of n such terms, so it is off by at most 2 (d + 2^-21 + (n + 4) 2^-24) of the largest |g' sum_m |c_m||, and half a step of its type.  With outputs of 16 bits a weight
may be held in steps of 2^-19 of the largest weight |p g'| of its 2048 rows, rounded up or down so that the mean error is zero: the sum of n such
errors is beyond 6 sqrt(n) half steps with a chance under 1e-7 (Hoeffding), whatever the order.
Choices of pages, pages, slots and copies are whole numbers: equal."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24


def half_step(t):
    return torch.finfo(t).eps / 2, torch.finfo(t).tiny * torch.finfo(t).eps / 2


class Case:
    """A cache of 2 G heads with sequences of the given lengths, on the host."""

    def __init__(self, lens, G, R, D, M, K, page, kind, scaled, seed, spread=1.0, spare=3):
        rng = np.random.default_rng(seed)
        self.rng, self.lens, self.G, self.R, self.D, self.M, self.K, self.page, self.kind = rng, list(lens), G, R, D, M, K, page, TYPES[kind]
        self.B = len(lens)
        pages = [-(-n // page) for n in lens]
        self.max_pages = max(pages + [1]) + 1
        self.n_pages = sum(pages) + spare
        order = rng.permutation(self.n_pages)
        self.tables = rng.integers(-5, 2 ** 31 - 1, (self.B, self.max_pages)).astype(np.int32)     # behind a sequence: anything
        at = 0
        for b, p in enumerate(pages):
            self.tables[b, :p] = order[at:at + p]
            at += p
        self.C = (rng.standard_normal((2 * G, M, K, D)) * spread * 0.8 ** np.arange(M)[None, :, None, None]).astype(np.float32)
        self.codes = rng.integers(0, 256, (self.n_pages * page, 2 * G, M)).astype(np.uint8)         # those of K or more are K - 1
        self.scale = np.exp(0.5 * rng.standard_normal((self.n_pages * page, 2 * G))).astype(np.float32) if scaled else None
        self.Q = torch.from_numpy(rng.standard_normal((self.B, G * R, D)).astype(np.float32)).to(self.kind)
        self.factor = 1 / math.sqrt(D)

    def rows(self, b, h, begins=None, picked=None):
        """Slots of the rows that take part, one by one."""
        n = min(max(self.lens[b], 0), self.max_pages * self.page)
        first = 0 if begins is None else max(int(begins[b]), 0)
        if picked is None:
            ts = range(first, n)
        else:
            ts = [t for j in picked[b, h] if 0 <= j < self.max_pages for t in range(j * self.page, (j + 1) * self.page) if first <= t < n]
        out = []
        for t in ts:
            p = int(self.tables[b, t // self.page])
            if 0 <= p < self.n_pages:
                out.append(p * self.page + t % self.page)
        return np.array(out, np.int64)

    def x(self, head, slots, absolute=False):
        C = np.abs(self.C[head]).astype(np.float64) if absolute else self.C[head].astype(np.float64)
        ids = np.minimum(self.codes[slots, head], self.K - 1)
        v = sum(C[m][ids[:, m]] for m in range(self.M))
        g = self.scale[slots, head].astype(np.float64)[:, None] if self.scale is not None else 1.0
        return v * (np.abs(g) if absolute else g)

    def attend(self, begins=None, picked=None):
        """out, lse, and how far out may be off."""
        out, lse = np.zeros((self.B, self.G * self.R, self.D)), np.full((self.B, self.G * self.R), -np.inf)
        tol = np.zeros_like(out)
        rel, tiny = half_step(self.kind)
        for b in range(self.B):
            for h in range(self.G):
                slots = self.rows(b, h, begins, picked)
                if len(slots) == 0:
                    continue
                k, v, va, ka = self.x(h, slots), self.x(self.G + h, slots), self.x(self.G + h, slots, True), self.x(h, slots, True)
                g = np.abs(self.scale[slots, self.G + h]) if self.scale is not None else np.ones(len(slots))
                for r in range(self.R):
                    q = self.Q[b, h * self.R + r].double().numpy()
                    s = self.factor * (k @ q)
                    with np.errstate(all="ignore"):
                        p = np.exp(s - s.max())
                        y = (p @ v) / p.sum()
                        out[b, h * self.R + r] = y
                        lse[b, h * self.R + r] = s.max() + np.log(p.sum())
                        d = (self.D + self.M + 8) * U * np.abs(self.factor) * (ka @ np.abs(q)).max()
                        e = 2 * (d + 2.0 ** -21 + (len(slots) + 4) * U) * va.max(0)
                        if self.kind is not torch.float32:
                            e = e + 2.0 ** -20 * 6 * np.sqrt(len(slots)) * (p * g).max() / p.sum() * np.abs(self.C[self.G + h]).max(1).sum(0)
                        tol[b, h * self.R + r] = e + rel * (np.abs(y) + e) + tiny
        return out, lse, tol

    def device(self):
        from paper_1509_05194_amd import hclae
        ctx = hclae.Context(max(self.B, 1), self.D, self.M, self.K)
        ctx.cache_begin(torch.from_numpy(self.C).cuda())
        return ctx

    def run(self, ctx, begins=None, picked=None, lse=True, layout="tight"):
        Q = self.Q.cuda()
        out = torch.full((self.B, self.G * self.R, self.D), 7.0, dtype=self.kind, device="cuda")
        if layout == "wide":
            w = torch.full((self.B, self.G * self.R + 3, self.D), 7.0, dtype=self.kind, device="cuda")
            w[:, 1:1 + self.G * self.R] = Q
            Q = w[:, 1:1 + self.G * self.R]
            out = torch.full((self.G * self.R, self.B, self.D + 4), 7.0, dtype=self.kind, device="cuda").transpose(0, 1)[:, :, :self.D]
        l = torch.full((self.B, self.G * self.R), 7.0, device="cuda") if lse else None
        dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
        ctx.cache_attend(Q, dev(self.codes), dev(self.scale), dev(self.tables), torch.tensor(self.lens, dtype=torch.int32, device="cuda"), self.page, out,
                         begins=dev(begins), picked=dev(picked), lse=l)
        torch.cuda.synchronize()
        return out, l

    def check(self, out, lse, begins=None, picked=None):
        want, want_lse, tol = self.attend(begins, picked)
        off = np.abs(out.double().cpu().numpy() - want)
        assert np.array_equal(np.isnan(off), np.isnan(want)), "NaN elsewhere than it should be"
        assert not (off > tol).any(), (np.nanmax(off / tol), np.argwhere(off > tol)[:4])
        if lse is not None:
            got = lse.double().cpu().numpy()
            assert np.array_equal(np.isinf(got), np.isinf(want_lse))
            ok = np.isfinite(want_lse)
            # a score's error, and a logarithm of a sum
            bound = (self.D + self.M + 8) * U * self.factor * self.Q.double().abs().numpy().max() * self.D * self.M * np.abs(self.C).max() * (1 if self.scale is None else np.nanmax(np.abs(self.scale)))
            assert (np.abs(got[ok] - want_lse[ok]) <= bound + 2.0 ** -20 + 2.0 ** -22 * np.abs(want_lse[ok])).all()


ATTEND = [
    ([1], 1, 1, 4, 1, 1, 1, "fp32", False), ([5, 0, 17], 2, 1, 64, 8, 256, 16, "bf16", True), ([150], 8, 4, 128, 8, 256, 16, "bf16", True),
    ([300, 1, 33], 3, 5, 80, 5, 200, 24, "fp32", False), ([64, 65, 63], 1, 2, 128, 16, 256, 64, "fp16", True), ([40], 2, 3, 36, 3, 20, 1, "fp32", True),
    ([200, 100], 1, 16, 256, 4, 64, 24, "bf16", True), ([77], 16, 1, 12, 2, 33, 5, "fp16", False), ([33, 0, 0, 9], 2, 8, 132, 40, 17, 16, "fp32", True),
    ([2500, 700], 1, 4, 64, 8, 256, 64, "bf16", True), ([2300], 2, 7, 128, 8, 256, 16, "fp32", True), ([5000], 1, 1, 32, 16, 256, 128, "fp16", True),
    ([4100, 2048, 2049, 1], 1, 2, 64, 7, 255, 16, "bf16", False), ([3000], 1, 5, 68, 16, 250, 24, "fp32", False), ([2200], 1, 4, 128, 32, 60, 64, "bf16", True),
]


@pytest.mark.parametrize("lens,G,R,D,M,K,page,kind,scaled", ATTEND)
def test_attend(lens, G, R, D, M, K, page, kind, scaled):
    c = Case(lens, G, R, D, M, K, page, kind, scaled, seed=sum(lens) + D)
    ctx = c.device()
    c.check(*c.run(ctx))
    c.check(*c.run(ctx, layout="wide"))
    again = [c.run(ctx)[0] for _ in range(3)]
    assert all(torch.equal(again[0], x) for x in again[1:])          # equal calls, equal bits
    ctx.close()


@pytest.mark.parametrize("lens,R,kind,M", [([50, 0, 200], 4, "bf16", 8), ([2600, 2100, 5], 4, "bf16", 8), ([3000, 40], 3, "fp32", 4), ([2500], 1, "fp16", 16)])
def test_attend_rows_that_take_part(lens, R, kind, M):
    """From a first row on, of picked pages, with pages that are not there, and all of it together."""
    c = Case(lens, 2, R, 64, M, 256, 16, kind, True, seed=sum(lens))
    ctx = c.device()
    begins = np.array([min(n, 7 + 3 * i) for i, n in enumerate(lens)], np.int32)
    begins[0] = -4
    c.check(*c.run(ctx, begins=begins), begins=begins)
    beyond = np.array([n + 5 for n in lens], np.int32)               # nothing left
    out, lse = c.run(ctx, begins=beyond)
    assert (out == 0).all() and (lse == -math.inf).all()
    picked = c.rng.integers(-2, c.max_pages + 2, (c.B, 2, 9)).astype(np.int32)
    picked[:, :, 1] = picked[:, :, 0]                                # a page named twice counts twice
    picked[-1, 1] = -1                                               # a head with none
    c.check(*c.run(ctx, picked=picked), picked=picked)
    c.check(*c.run(ctx, begins=begins, picked=picked), begins=begins, picked=picked)
    for b, n in enumerate(lens):                                     # pages outside the cache
        for j in range(0, -(-n // 16), 3):
            c.tables[b, j] = [-1, c.n_pages, 2 ** 31 - 1, -2 ** 31][j % 4]
    c.check(*c.run(ctx))
    c.check(*c.run(ctx, picked=picked), picked=picked)
    c.lens[0] = -3                                                   # lengths outside the table
    c.lens[-1] = 2 ** 31 - 1
    c.check(*c.run(ctx))
    ctx.close()


@pytest.mark.parametrize("n,kind", [(90, "bf16"), (3000, "bf16"), (3000, "fp32")])
def test_attend_nan_scales(n, kind):
    """A row that was written with a NaN or an infinity has the scale NaN: it counts where it takes part, and only there."""
    c = Case([n, n], 2, 4, 64, 8, 256, 16, kind, True, seed=n)
    ctx = c.device()
    key, value = c.rows(0, 0)[n // 2], c.rows(1, 1)[n // 3]
    c.scale[key, 0] = np.nan                                          # a key of sequence 0, head 0
    c.scale[value, 2 + 1] = np.nan                                    # a value of sequence 1, head 1
    free = np.setdiff1d(np.arange(c.n_pages * 16), np.concatenate([c.rows(0, 0), c.rows(1, 0)]))
    c.scale[free] = np.nan                                            # and rows of no sequence
    out, lse = c.run(ctx)
    bad = torch.isnan(out).all(2).cpu().numpy()
    assert np.array_equal(bad, torch.isnan(out).any(2).cpu().numpy())
    want = np.zeros((2, 8), bool)
    want[0, :4] = want[1, 4:] = True
    assert np.array_equal(bad, want)
    assert np.array_equal(torch.isnan(lse).cpu().numpy(), np.repeat([[True, False], [False, False]], 4, 1))
    c.check(out, None)
    # where the row does not take part nothing is NaN
    begins = np.array([n // 2 + 1, n // 3 + 1], np.int32)
    c.check(*c.run(ctx, begins=begins), begins=begins)
    ctx.close()


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [100, 6000])
def test_attend_scores_far_apart(n, kind):
    """Scores that rise along the sequence by far more than an exponential holds, fall, or stand out in one row; scales at both ends."""
    for shape in ("rise", "fall", "one", "zero", "large"):
        c = Case([n], 1, 4, 32, 4, 256, 16, kind, True, seed=n)
        slots = c.rows(0, 0)
        ramp = np.linspace(1e-3, 60, n)
        if shape == "rise":
            c.scale[slots, 0] = ramp
        elif shape == "fall":
            c.scale[slots, 0] = ramp[::-1]
        elif shape == "one":
            c.scale[slots, 0] = 1e-3
            c.scale[slots[n // 2], 0] = 200
        elif shape == "zero":
            c.scale[slots, 1] = 0
        else:
            c.scale[slots, 1] = np.where(np.arange(n) % 2, 1e30, -1e25)
            if kind == "bf16":
                c.scale[slots[5], 1] = 0
        ctx = c.device()
        c.check(*c.run(ctx))
        ctx.close()


def test_attend_small_weights_add_up():
    """One row far above all others, whose weights are below every step of a fixed point: their sum is not lost."""
    n = 40000
    for kind in ("bf16", "fp32"):
        c = Case([n], 1, 4, 32, 2, 256, 16, kind, True, seed=3)
        slots = c.rows(0, 0)
        c.scale[slots, 0] = 0
        c.Q[:] = 1.0
        c.C[0] = np.abs(c.C[0]) + 0.05
        top = slots[1234]
        s = c.factor * c.x(0, np.array([top]))                        # zero now; the scale that lifts the row to ln 2^23
        c.scale[top, 0] = 1.0
        c.scale[top, 0] = math.log(2.0 ** 23) / float(c.factor * c.x(0, np.array([top])).sum())
        c.scale[slots, 1] = 1.0
        c.C[1] = np.abs(c.C[1])                                       # values of one sign
        ctx = c.device()
        out, lse = c.run(ctx)
        c.check(out, lse)
        ctx.close()


def test_attend_very_long():
    """Slots beyond 2^31 bytes, and a sequence in many parts."""
    n, page, G, M = 70000, 64, 1, 8
    c = Case([n], G, 4, 64, M, 256, page, "bf16", True, seed=1)
    want, want_lse, tol = c.attend()
    far = (2 ** 31 // (2 * G * M * page) + 77)                       # pages in front: codes begin beyond 2^31 bytes
    ctx = c.device()
    codes = torch.zeros(((far + c.n_pages) * page, 2 * G, M), dtype=torch.uint8, device="cuda")
    scale = torch.zeros(((far + c.n_pages) * page, 2 * G), device="cuda")
    codes[far * page:] = torch.from_numpy(c.codes).cuda()
    scale[far * page:] = torch.from_numpy(c.scale).cuda()
    tables = torch.from_numpy(np.where(np.arange(c.max_pages) < -(-n // page), c.tables + far, -1).astype(np.int32)).cuda()
    out = torch.zeros((1, 4, 64), dtype=c.kind, device="cuda")
    ctx.cache_attend(c.Q.cuda(), codes, scale, tables, torch.tensor([n], dtype=torch.int32, device="cuda"), page, out)
    off = np.abs(out.double().cpu().numpy() - want)
    assert not (off > tol).any(), np.nanmax(off / tol)
    ctx.close()


# ---- the choice of pages -------------------------------------------------------------------------

def select(Q, C, codes, scale, tables, lens, page, n_pages, k, first, recent):
    """picked int32 [B][H][k] in plain Python, scores in 64 bits."""
    B, Hq, _ = Q.shape
    H, M, K, D = C.shape
    R = Hq // H
    out = np.full((B, H, k), -1, np.int32)
    for b in range(B):
        P = min(-(-max(int(lens[b]), 0) // page), tables.shape[1])
        for h in range(H):
            q = Q[b, h * R:(h + 1) * R].astype(np.float64).sum(0)
            T = C[h].astype(np.float64) @ q                          # [M][K]
            items = []
            for j in range(P):
                p = int(tables[b, j])
                if not 0 <= p < n_pages:
                    continue
                forced = j < first or j >= P - recent
                x = 0.0
                if not forced:
                    for m in range(M):
                        x += T[m][min(int(codes[p, h, m]), K - 1)]
                    if scale is not None:
                        x *= float(scale[p, h])
                    if x != x:
                        x = -math.inf
                items.append((not forced, -x, j))
            best = sorted(j for _, _, j in sorted(items)[:k])
            out[b, h, :len(best)] = best
    return out


SELECT = [
    ([1], 1, 1, 4, 1, 1, 1, 1, 0, 0, "fp32", False), ([800], 2, 4, 64, 8, 256, 16, 6, 1, 1, "bf16", True), ([5000, 100, 0], 3, 5, 128, 16, 256, 16, 16, 2, 1, "fp16", True),
    ([4000, 3999], 1, 1, 256, 2, 7, 1, 64, 0, 1, "fp32", False), ([30000], 2, 8, 80, 5, 200, 4, 200, 4, 4, "bf16", True), ([900], 1, 2, 36, 40, 20, 24, 50, 1, 0, "fp32", True),
    ([26000], 1, 1, 64, 8, 256, 1, 1024, 0, 0, "bf16", True), ([2 ** 31 - 1, 64], 2, 3, 128, 130, 256, 64, 5, 1, 1, "bf16", True),
]


@pytest.mark.parametrize("lens,H,R,D,M,K,page,k,first,recent,kind,scaled", SELECT)
def test_select(lens, H, R, D, M, K, page, k, first, recent, kind, scaled):
    from paper_1509_05194_amd import hclae
    rng = np.random.default_rng(len(lens) + D + k)
    lens = np.array(lens, np.int64)
    max_pages = int(max(-(-min(n, 9000 * page) // page) for n in lens)) + 2
    n_pages = max_pages * len(lens) + 3
    tables = rng.integers(0, n_pages, (len(lens), max_pages)).astype(np.int32)
    if max_pages > 40:
        tables[:, 5::11] = rng.choice([-1, n_pages, -2 ** 31, 2 ** 31 - 1], tables[:, 5::11].shape)
        tables[:, 0] = -1
    C = rng.standard_normal((H, M, K, D)).astype(np.float32)
    codes = rng.integers(0, 256, (n_pages, H, M)).astype(np.uint8)
    scale = rng.standard_normal((n_pages, H)).astype(np.float32) if scaled else None
    if scaled:
        scale[::7] = 0                                               # equal scores: the lower page
        scale[3::29] = np.nan
    codes[1::5] = codes[0]
    Q = torch.from_numpy(rng.standard_normal((len(lens), H * R, D)).astype(np.float32)).to(TYPES[kind])
    ctx = hclae.Context(len(lens), D, M, K)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    picked = torch.full((len(lens), H, k), 99, dtype=torch.int32, device="cuda")
    ctx.cache_select(Q.cuda(), torch.from_numpy(codes).cuda(), None if scale is None else torch.from_numpy(scale).cuda(), torch.from_numpy(tables).cuda(),
                     torch.from_numpy(lens.astype(np.int32)).cuda(), page, picked, first=first, recent=recent)
    want = select(Q.double().numpy(), C, codes, scale, tables, lens, page, n_pages, k, first, recent)
    assert np.array_equal(picked.cpu().numpy(), want)
    ctx.close()


def test_select_all_equal():
    """A query of zeros: every score is zero, whatever the signs, and the first pages are taken."""
    from paper_1509_05194_amd import hclae
    ctx = hclae.Context(1, 16, 4, 8)
    ctx.cache_begin(torch.randn((1, 4, 8, 16), device="cuda"))
    P = 5000
    codes = torch.randint(0, 8, (P, 1, 4), dtype=torch.uint8, device="cuda")
    scale = torch.randn((P, 1), device="cuda")
    tables = torch.randperm(P, device="cuda").int()[None]
    picked = torch.zeros((1, 1, 33), dtype=torch.int32, device="cuda")
    ctx.cache_select(torch.zeros((1, 2, 16), device="cuda"), codes, scale, tables, torch.tensor([P], dtype=torch.int32, device="cuda"), 1, picked, first=0, recent=2)
    assert picked.flatten().tolist() == list(range(31)) + [P - 2, P - 1]
    ctx.close()


@pytest.mark.parametrize("P,k,first,recent", [(5, 3, 1, 1), (40, 10, 1, 1), (40, 2, 1, 1), (40, 10, 0, 0), (120, 30, 3, 2), (3000, 33, 1, 1)])
@pytest.mark.parametrize("which", ["scales", "queries"])
def test_select_infinite_scores(which, P, k, first, recent):
    """Scores of both infinities, more of the greater than are asked for, beside pages that are taken whatever their scores."""
    from paper_1509_05194_amd import hclae
    rng = np.random.default_rng(P + k)
    C = rng.standard_normal((2, 2, 16, 16)).astype(np.float32)
    codes = rng.integers(0, 16, (P, 2, 2)).astype(np.uint8)
    scale = rng.standard_normal((P, 2)).astype(np.float32)
    Q = rng.standard_normal((2, 4, 16)).astype(np.float32)
    if which == "scales":
        scale[:] = np.inf
    else:
        Q[:, ::2, 5] = np.inf
    tables = np.stack([rng.permutation(P) for _ in range(2)]).astype(np.int32)
    ctx = hclae.Context(2, 16, 2, 16)
    ctx.cache_begin(torch.from_numpy(C).cuda())
    picked = torch.full((2, 2, k), 99, dtype=torch.int32, device="cuda")
    ctx.cache_select(torch.from_numpy(Q).cuda(), torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda(), torch.from_numpy(tables).cuda(),
                     torch.tensor([P, P], dtype=torch.int32, device="cuda"), 1, picked, first=first, recent=recent)
    want = select(Q.astype(np.float64), C, codes, scale, tables, [P, P], 1, P, k, first, recent)
    assert np.array_equal(picked.cpu().numpy(), want)
    ctx.close()


# ---- pages ---------------------------------------------------------------------------------------

def extend(tables, lens, starts, n, page, n_pages):
    """The definition, a sequence after another: tables, lens, slots, src, dst, rows."""
    tables, lens = tables.copy(), [int(x) for x in lens]
    most = tables.shape[1]
    held = [min(max(x, 0), most * page) for x in lens]
    users = {}
    for b, x in enumerate(held):
        for p in tables[b, :-(-x // page)].tolist():
            if 0 <= p < n_pages:
                users[p] = users.get(p, 0) + 1
    free = [p for p in range(n_pages) if p not in users]
    slots, moves, asked = np.full(n, -1, np.int64), [], 0
    for b, x in enumerate(held):
        lo, hi = min(max(int(starts[b]), 0), n), min(max(int(starts[b + 1]), 0), n)
        add, move = max(hi - lo, 0), (-1, -1, 0)
        e = x // page
        split = add > 0 and x % page > 0 and users.get(int(tables[b, e]), 0) > 1
        need = -(-(x + add) // page) - -(-x // page) + split
        if add and -(-(x + add) // page) <= most:
            asked += need
            if need == 0 or asked <= len(free):
                mine = free[asked - need:asked]
                if split:
                    move = (int(tables[b, e]), mine[0], x % page)
                    tables[b, e] = mine.pop(0)
                for j in range(-(-x // page), -(-(x + add) // page)):
                    tables[b, j] = mine.pop(0)
                for i in range(add):
                    p = int(tables[b, (x + i) // page])
                    slots[lo + i] = p * page + (x + i) % page if 0 <= p < n_pages else -1
                lens[b] = x + add
        moves.append(move)
    return tables, lens, slots, [np.array([m[i] for m in moves], np.int32) for i in range(3)]


def extend_on_device(ctx, tables, lens, starts, n, page, n_pages):
    B = len(lens)
    t, l = torch.from_numpy(tables).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    slots = torch.full((n,), 77, dtype=torch.int64, device="cuda")
    moves = [torch.full((B,), 77, dtype=torch.int32, device="cuda") for _ in range(3)]
    ctx.cache_extend(t, l, torch.tensor(starts, dtype=torch.int32, device="cuda"), page, n_pages, slots, *moves)
    return t, l, slots, moves


@pytest.mark.parametrize("B,most,page,spare,seed", [(1, 1, 1, 0, 0), (3, 8, 16, 100, 1), (9, 30, 5, 40, 2), (70, 6, 24, 20, 3), (300, 12, 4, 900, 4), (40, 9, 7, 3, 5), (2500, 3, 2, 2000, 6),
                                                    (5, 400, 3, 9000, 7), (64, 2000, 1, 60000, 8)])
def test_extend(B, most, page, spare, seed):
    from paper_1509_05194_amd import hclae
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, most * page + 1, B)
    lens[rng.random(B) < 0.2] = 0
    need = int(sum(-(-x // page) for x in lens))
    n_pages = need + spare
    order = rng.permutation(n_pages)[:need]
    tables = rng.integers(-9, n_pages + 9, (B, most)).astype(np.int32)
    at = 0
    for b, x in enumerate(lens):
        p = -(-int(x) // page)
        tables[b, :p] = order[at:at + p]
        at += p
    for b in range(1, B, 3):                                         # forks: of the whole, and shorter ones
        tables[b] = tables[b - 1]
        lens[b] = lens[b - 1] if b % 2 else rng.integers(0, lens[b - 1] + 1)
    if B > 20:
        lens[5], lens[6] = -7, 2 ** 31 - 1                           # outside the table
        tables[7, max(0, -(-int(lens[7]) // page) - 1)] = -1         # a last page that is not there
    adds = rng.integers(0, 3 * page + 2, B) * (rng.random(B) < 0.7)
    if seed == 8:
        adds[3] = 900
    starts = np.concatenate([[2], 2 + np.cumsum(adds)])
    n = int(starts[-1]) + 3                                          # rows of no sequence in front and behind
    ctx = hclae.Context(n, 16, 2, 4)
    t, l, slots, moves = extend_on_device(ctx, tables, lens, starts, n, page, n_pages)
    want = extend(tables, lens, starts, n, page, n_pages)
    assert np.array_equal(slots.cpu().numpy(), want[2])
    assert np.array_equal(l.cpu().numpy(), np.array(want[1]))
    assert np.array_equal(t.cpu().numpy(), want[0])
    for got, w in zip(moves, want[3]):
        assert np.array_equal(got.cpu().numpy(), w)
    live = [s for s in want[2].tolist() if s >= 0]
    assert len(set(live)) == len(live)                               # a slot for each row
    ctx.close()


@pytest.mark.parametrize("B", [4, 9000])        # one block, and several kernels
def test_extend_up_to_the_longest(B):
    """Lengths are 32-bit: the last row that one can count is number 2^31 - 2, and a sequence that asks for more is left as it is."""
    from paper_1509_05194_amd import hclae
    page, max_pages, n_pages, top = 2 ** 30, 4, 5, 2 ** 31 - 1
    tables = np.full((B, max_pages), -1, np.int32)
    lens, adds = np.zeros(B, np.int32), np.zeros(B, np.int64)
    tables[0, :2], lens[0], adds[0] = (3, 1), top - 3, 3
    tables[1, :2], lens[1], adds[1] = (0, 4), top - 3, 4
    tables[2, :2], lens[2], adds[2] = (1, 3), top, 1
    adds[3] = 2
    starts = np.concatenate([[0], np.cumsum(adds)]).astype(np.int32)
    n = int(starts[-1])
    slots = torch.full((n,), -7, dtype=torch.int64, device="cuda")
    moves = [torch.full((B,), -7, dtype=torch.int32, device="cuda") for _ in range(3)]
    t, l = torch.from_numpy(tables).cuda(), torch.from_numpy(lens).cuda()
    ctx = hclae.Context(16, 8, 2, 4)
    ctx.cache_extend(t, l, torch.from_numpy(starts).cuda(), page, n_pages, slots, *moves)
    torch.cuda.synchronize()
    ctx.close()
    # page 1 is of sequences 0 and 2: sequence 0's last page is copied to page 2, the only free one, and sequence 3 finds none
    tables[0, 1], lens[0] = 2, top
    first = 2 * page + (top - 3) % page
    assert t.cpu().numpy().tolist() == tables.tolist()
    assert l.cpu().numpy().tolist() == lens.tolist()
    assert slots.cpu().tolist() == [first, first + 1, first + 2] + [-1] * 7
    src, dst, rows = [m.cpu().numpy() for m in moves]
    assert (src[0], dst[0], rows[0]) == (1, 2, (top - 3) % page)
    assert (src[1:] == -1).all() and (dst[1:] == -1).all() and (rows[1:] == 0).all()


def compact(tables, lens, page, n_pages):
    tables = tables.copy()
    held = [min(max(int(x), 0), tables.shape[1] * page) for x in lens]
    used = sorted({p for b, x in enumerate(held) for p in tables[b, :-(-x // page)].tolist() if 0 <= p < n_pages})
    u = len(used)
    holes = [p for p in range(u) if p not in set(used)]
    movers = [p for p in used if p >= u]
    to = dict(zip(movers, holes))
    for b, x in enumerate(held):
        for j in range(-(-x // page)):
            tables[b, j] = to.get(int(tables[b, j]), tables[b, j])
    pad = [-1] * (n_pages // 2 - len(movers))
    return tables, np.array(movers + pad, np.int32), np.array(holes + pad, np.int32), u


@pytest.mark.parametrize("B,most,page,pool,H,M,scaled,seed", [(1, 1, 1, 1, 1, 1, False, 0), (4, 9, 16, 90, 2, 8, True, 1), (7, 20, 5, 150, 3, 5, True, 2), (60, 70, 3, 9000, 2, 3, False, 3),
                                                              (3, 5, 4, 15, 1, 16, True, 4), (2, 3, 2, 1000, 2, 7, True, 5), (9, 600, 1, 70000, 1, 4, True, 6), (5, 6, 16, 33, 16, 8, True, 7), (2, 4, 3, 64, 1, 1, True, 8)])
def test_compact_and_copy(B, most, page, pool, H, M, scaled, seed):
    from paper_1509_05194_amd import hclae
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, most * page + 1, B)
    lens[rng.random(B) < 0.3] = 0
    tables = rng.integers(-3, pool + 3, (B, most)).astype(np.int32)  # shared pages, pages outside
    if seed == 4:
        lens[:] = most * page                                        # every page in use: nothing moves
        tables = rng.permutation(pool).reshape(B, most).astype(np.int32)
    codes = rng.integers(0, 256, (pool * page + 1, H, M)).astype(np.uint8)
    scale = rng.standard_normal((pool * page + 1, H)).astype(np.float32) if scaled else None
    want_t, want_src, want_dst, u = compact(tables, lens, page, pool)
    ctx = hclae.Context(1, 4, M, 1)
    ctx.cache_begin(torch.zeros((H, M, 1, 4), device="cuda"))
    t = torch.from_numpy(tables).cuda()
    src, dst = (torch.full((pool // 2,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    used = torch.zeros((1,), dtype=torch.int32, device="cuda")
    ctx.cache_compact(t, torch.from_numpy(lens.astype(np.int32)).cuda(), page, pool, src, dst, used)
    assert int(used) == u
    assert np.array_equal(src.cpu().numpy(), want_src) and np.array_equal(dst.cpu().numpy(), want_dst)
    assert np.array_equal(t.cpu().numpy(), want_t)
    # the copies, and copies of parts of pages
    dc, ds = torch.from_numpy(codes).cuda(), None if scale is None else torch.from_numpy(scale).cuda()
    rows = rng.integers(-2, page + 3, pool // 2).astype(np.int32)
    for keep in (None, rows):
        ctx.cache_copy(dc, ds, page, src, dst, None if keep is None else torch.from_numpy(keep).cuda())
        for i, (f, d) in enumerate(zip(want_src, want_dst)):
            if f >= 0:
                k = page if keep is None else min(max(int(keep[i]), 0), page)
                codes[d * page:d * page + k] = codes[f * page:f * page + k]
                if scale is not None:
                    scale[d * page:d * page + k] = scale[f * page:f * page + k]
        assert np.array_equal(dc.cpu().numpy(), codes)
        assert scale is None or np.array_equal(ds.cpu().numpy(), scale)
    # pages outside the cache, and a page to itself
    out = len(codes) // page
    src, dst = torch.tensor([-1, out, 0, 0, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), torch.tensor([0, 0, out, 0, -2 ** 31], dtype=torch.int32, device="cuda")
    ctx.cache_copy(dc, ds, page, src, dst)
    assert np.array_equal(dc.cpu().numpy(), codes)
    ctx.close()


# ---- together ------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind,R,M", [("bf16", 4, 8), ("fp32", 2, 4)])
def test_a_run_of_steps(kind, R, M):
    """Prompts written and attended to, forks, single tokens, a sequence given up, the cache compacted, and pages chosen by the means of their keys:
    every step against attention over the rows as cache_read gives them back."""
    from paper_1509_05194_amd import hclae
    G, D, K, page, n_pages, most, dt = 2, 64, 64, 16, 60, 12, TYPES[kind]
    H, B = 2 * G, 4
    g = torch.Generator(device="cuda").manual_seed(5)
    C = torch.randn((H, M, K, D), generator=g, device="cuda") * 0.5 ** torch.arange(M, device="cuda")[None, :, None, None]
    ctx = hclae.Context(600, D, M, K)
    ctx.cache_begin(C)
    keys = hclae.Context(n_pages, D, M, K)                           # the key heads' dictionaries, for stand-ins
    keys.cache_begin(C[:G].contiguous())
    codes, scale = torch.zeros((n_pages * page, H, M), dtype=torch.uint8, device="cuda"), torch.zeros((n_pages * page, H), device="cuda")
    tables, lengths = torch.zeros((B, most), dtype=torch.int32, device="cuda"), torch.zeros((B,), dtype=torch.int32, device="cuda")
    src, dst, rows = (torch.zeros((B,), dtype=torch.int32, device="cuda") for _ in range(3))

    def step(adds):
        starts = torch.tensor([0] + list(np.cumsum(adds)), dtype=torch.int32, device="cuda")
        n = sum(adds)
        slots = torch.zeros((n,), dtype=torch.int64, device="cuda")
        before = lengths.tolist()
        ctx.cache_extend(tables, lengths, starts, page, n_pages, slots, src, dst, rows)
        ctx.cache_copy(codes, scale, page, src, dst, rows)
        ctx.cache_write(torch.randn((n, H, D), generator=g, device="cuda").to(dt), slots, codes, scale)
        assert lengths.tolist() == [a + b for a, b in zip(before, adds)] and (slots >= 0).all()
        attend()

    def decoded(b):
        n = int(lengths[b])
        out = torch.zeros((n, H, D), device="cuda")
        ctx.cache_read(codes, scale, tables[b:b + 1].contiguous(), torch.tensor([0, n], dtype=torch.int32, device="cuda"), page, out)
        return out.double()

    def attend(picked=None):
        Q = torch.randn((B, G * R, D), generator=g, device="cuda").to(dt)
        out = torch.zeros_like(Q)
        ctx.cache_attend(Q, codes, scale, tables, lengths, page, out, picked=picked)
        for b in range(B):
            x = decoded(b)
            for h in range(G):
                keep = torch.arange(len(x), device="cuda")
                if picked is not None:
                    keep = keep[torch.isin(keep // page, picked[b, h].long())]
                if len(keep) == 0:
                    assert (out[b, h * R:(h + 1) * R] == 0).all()
                    continue
                q = Q[b, h * R:(h + 1) * R].double()
                p = torch.softmax(q @ x[keep, h].T / math.sqrt(D), 1)
                want = p @ x[keep, G + h]
                # roundings as at the top, with |x| up to M codewords of the size of the largest
                top = float(C.abs().amax(3).amax(2).sum(1).max() * scale.max())
                d = (D + M + 8) * U * float(q.abs().sum(1).max()) * top / math.sqrt(D)
                e = 2 * (d + 2.0 ** -21 + (len(keep) + 8) * U) * top
                if dt is not torch.float32:
                    e += 2.0 ** -20 * 6 * math.sqrt(len(keep)) * top
                off = (out[b, h * R:(h + 1) * R].double() - want).abs()
                assert (off <= e + half_step(dt)[0] * (want.abs() + e)).all(), (float(off.max()), e)

    step([37, 64, 0, 5])
    tables[2], lengths[2] = tables[1].clone(), lengths[1].clone()     # a fork at a page's end, and one within a page
    step([1, 1, 1, 1])
    tables[3], lengths[3] = tables[0].clone(), lengths[0].clone()
    for _ in range(3):
        step([1, 1, 1, 1])
    lengths[1] = 0
    n = n_pages // 2
    msrc, mdst, used = torch.zeros((n,), dtype=torch.int32, device="cuda"), torch.zeros((n,), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda")
    before = [decoded(b) for b in range(B)]
    ctx.cache_compact(tables, lengths, page, n_pages, msrc, mdst, used)
    ctx.cache_copy(codes, scale, page, msrc, mdst)
    for b in range(B):
        assert torch.equal(decoded(b), before[b])
        assert (tables[b, :-(-int(lengths[b]) // page)] < used).all()
    step([60, 70, 1, 90])
    # stand-ins: the means of the keys of every page, written as codes to the page's number
    means = torch.zeros((n_pages, G, D), device="cuda")
    for b in range(B):
        x = decoded(b)
        for j in range(-(-int(lengths[b]) // page)):
            means[tables[b, j]] = x[j * page:(j + 1) * page, :G].mean(0).float()
    sc, ss = torch.zeros((n_pages, G, M), dtype=torch.uint8, device="cuda"), torch.zeros((n_pages, G), device="cuda")
    keys.cache_write(means, torch.arange(n_pages, device="cuda"), sc, ss)
    picked = torch.zeros((B, G, 3), dtype=torch.int32, device="cuda")
    Q = torch.randn((B, G * R, D), generator=g, device="cuda").to(dt)
    keys.cache_select(Q, sc, ss, tables, lengths, page, picked)
    want = select(Q.double().cpu().numpy(), C[:G].cpu().numpy(), sc.cpu().numpy(), ss.cpu().numpy(), tables.cpu().numpy(), lengths.tolist(), page, n_pages, 3, 1, 1)
    assert np.array_equal(picked.cpu().numpy(), want)
    attend(picked)
    ctx.close()
    keys.close()


def test_graph_and_streams():
    """A step recorded into a graph and replayed between eager calls, on a stream that is not the current one; what needs more scratch is refused
    while recording, and scratch that grows leaves recorded graphs valid."""
    from paper_1509_05194_amd import hclae
    c = Case([300, 2300, 5], 2, 4, 64, 8, 256, 16, "bf16", True, seed=11)
    dev = lambda a: torch.from_numpy(a).cuda()
    codes, scale, tables = dev(c.codes), dev(c.scale), dev(np.clip(c.tables, -1, c.n_pages))
    Q = c.Q.cuda()
    add = 2
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ctx = hclae.Context(64, 64, 8, 256, stream=stream.cuda_stream)
        ctx.cache_begin(dev(c.C))
        lengths0 = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
        lengths = lengths0.clone()
        starts = torch.arange(4, dtype=torch.int32, device="cuda") * add
        slots = torch.zeros((3 * add,), dtype=torch.int64, device="cuda")
        moves = [torch.zeros((3,), dtype=torch.int32, device="cuda") for _ in range(3)]
        X = torch.randn((3 * add, 4, 64), device="cuda", dtype=torch.bfloat16)
        out = torch.zeros_like(Q)
        picked = torch.zeros((3, 2, 6), dtype=torch.int32, device="cuda")
        tables0 = tables.clone()

        def step():
            tables.copy_(tables0)
            lengths.copy_(lengths0)
            ctx.cache_extend(tables, lengths, starts, 16, c.n_pages, slots, *moves)
            ctx.cache_copy(codes, scale, 16, *moves)
            ctx.cache_write(X, slots, codes, scale)
            ctx.cache_attend(Q, codes, scale, tables, lengths, 16, out)

        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with pytest.raises(hclae.HclaeError) as e:                     # nothing has allocated the scratch yet
            with torch.cuda.graph(graph, stream=stream):
                ctx.cache_attend(Q, codes, scale, tables, lengths, 16, out)
        assert e.value.code == hclae.ESTATE
        step()
        stream.synchronize()
        want = [x.clone() for x in (out, tables, lengths, slots, codes)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for i in range(4):
            out.zero_()
            slots.zero_()
            graph.replay()
            if i == 1:                                                # more scratch for an eager call: the graph keeps its own
                big = Case([4000] * 40, 2, 4, 64, 8, 256, 16, "bf16", True, seed=12)
                ctx.cache_attend(big.Q.cuda(), dev(big.codes), dev(big.scale), dev(big.tables), torch.tensor(big.lens, dtype=torch.int32, device="cuda"), 16,
                                 torch.zeros((40, 8, 64), dtype=torch.bfloat16, device="cuda"))
                graph.replay()
            stream.synchronize()
            for got, w in zip((out, tables, lengths, slots, codes), want):
                assert torch.equal(got, w)
            Q.mul_(1.0)                                               # eager work between replays
        Q.neg_()
        graph.replay()
        stream.synchronize()
        replayed = out.clone()
        step()
        stream.synchronize()
        assert torch.equal(out, replayed) and not torch.equal(out, want[0])
    ctx.close()


def test_select_sizes_beyond_what_it_counts():
    """Of an empty batch, which is looked at for its sizes alone: no pointer is used."""
    from paper_1509_05194_amd import hclae
    ctx = hclae.Context(1, 16, 2, 4)
    ctx.cache_begin(torch.zeros((1, 2, 4, 16), device="cuda"))
    call = lambda max_pages, k: hclae.lib().hclae_cache_select(ctx._h, None, 0, 0, 1, 16, 16, None, None, 0, None, max_pages, 1, None, 0, 0, k, None)
    most = 2 ** 30
    assert call(most, most) == hclae.OK
    assert call(most + 1, 1) == hclae.EINVAL
    assert call(1, most + 1) == hclae.EINVAL
    assert call(2 ** 31 - 1, 2 ** 31 - 1) == hclae.EINVAL
    ctx.close()


def test_refusals():
    from paper_1509_05194_amd import hclae
    c = Case([20], 2, 2, 16, 2, 4, 4, "fp32", True, seed=0)
    dev = lambda a: torch.from_numpy(a).cuda()
    codes, scale, tables, lengths = dev(c.codes), dev(c.scale), dev(c.tables), torch.tensor([20], dtype=torch.int32, device="cuda")
    Q, out = c.Q.cuda(), torch.zeros((1, 4, 16), device="cuda")
    ctx = hclae.Context(4, 16, 2, 4)

    def refused(code, call):
        with pytest.raises(hclae.HclaeError) as e:
            call()
        assert e.value.code == code
        torch.cuda.synchronize()

    picked = torch.zeros((1, 4, 3), dtype=torch.int32, device="cuda")
    move = torch.zeros((1,), dtype=torch.int32, device="cuda")
    refused(hclae.ESTATE, lambda: ctx.cache_attend(Q, codes, scale, tables, lengths, 4, out))      # before cache_begin
    refused(hclae.ESTATE, lambda: ctx.cache_select(Q, codes, scale, tables, lengths, 4, picked))
    refused(hclae.ESTATE, lambda: ctx.cache_copy(codes, scale, 4, move, move))
    ctx.cache_begin(dev(c.C))
    attend = lambda **k: ctx.cache_attend(*[k.get(n, v) for n, v in (("Q", Q), ("codes", codes), ("scale", scale), ("tables", tables), ("lengths", lengths), ("page", 4), ("out", out))])
    refused(hclae.EINVAL, lambda: attend(page=0))
    refused(hclae.EINVAL, lambda: attend(Q=torch.zeros((1, 3, 16), device="cuda"), out=torch.zeros((1, 3, 16), device="cuda")))
    refused(hclae.EINVAL, lambda: attend(out=torch.zeros((1, 1, 16), device="cuda").expand(1, 4, 16)))
    refused(hclae.EINVAL, lambda: attend(Q=torch.zeros((1, 4, 17), device="cuda")[:, :, 1:]))
    refused(hclae.ESTATE, lambda: ctx.cache_attend(Q.expand(9, 4, 16), codes, scale, tables.expand(9, -1).contiguous(), lengths.expand(9).contiguous(), 4, torch.zeros((9, 4, 16), device="cuda")))
    for bad in (dict(codes=codes[:, :2].contiguous()), dict(scale=scale[:-1]), dict(lengths=lengths.repeat(2)), dict(out=out[:, :2])):
        with pytest.raises(ValueError):
            attend(**bad)
    for bad in (dict(codes=codes.int()), dict(tables=tables.long()), dict(out=out.half()), dict(Q=Q.double()), dict(scale=scale.cpu())):
        with pytest.raises(TypeError):
            attend(**bad)
    with pytest.raises(ValueError):
        ctx.cache_attend(Q, codes, scale, tables, lengths, 4, out, picked=torch.zeros((1, 2, 0), dtype=torch.int32, device="cuda"))
    select_ = lambda k, first, recent: ctx.cache_select(torch.zeros((1, 4, 16), device="cuda"), codes[:6], scale[:6], tables, lengths, 4, torch.zeros((1, 4, k), dtype=torch.int32, device="cuda"),
                                                        first=first, recent=recent)
    refused(hclae.EINVAL, lambda: select_(2, 2, 1))
    refused(hclae.EINVAL, lambda: select_(2, -1, 1))
    refused(hclae.EINVAL, lambda: select_(0, 0, 0))
    slots = torch.zeros((2,), dtype=torch.int64, device="cuda")
    starts = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    refused(hclae.EINVAL, lambda: ctx.cache_extend(tables, lengths, starts, 0, 6, slots, move, move.clone(), move.clone()))
    refused(hclae.EINVAL, lambda: ctx.cache_extend(tables, lengths, starts, 4, 2 ** 31, slots, move, move.clone(), move.clone()))
    refused(hclae.ESTATE, lambda: ctx.cache_extend(tables, lengths, starts, 4, 6, torch.zeros((5,), dtype=torch.int64, device="cuda"), move, move.clone(), move.clone()))
    refused(hclae.EINVAL, lambda: ctx.cache_compact(tables, lengths, 0, 6, torch.zeros((3,), dtype=torch.int32, device="cuda"), torch.zeros((3,), dtype=torch.int32, device="cuda")))
    refused(hclae.EINVAL, lambda: ctx.cache_copy(codes, scale, 0, move, move))
    odd = hclae.Context(4, 16, 2, 4)
    odd.cache_begin(dev(c.C)[:3].contiguous())
    refused(hclae.ESTATE, lambda: odd.cache_attend(torch.zeros((1, 3, 16), device="cuda"), codes[:, :3].contiguous(), scale[:, :3].contiguous(), tables, lengths, 4,
                                                   torch.zeros((1, 3, 16), device="cuda")))
    # nothing to do
    none = torch.zeros((0, 4, 16), device="cuda")
    ctx.cache_attend(none, codes, scale, tables[:0], lengths[:0], 4, none.clone())
    ctx.cache_copy(codes, scale, 4, move[:0], move[:0])
    ctx.cache_attend(Q, codes[:0], scale[:0], tables, lengths, 4, out)                              # a cache without pages
    assert (out == 0).all()
    ctx.close()
    odd.close()
