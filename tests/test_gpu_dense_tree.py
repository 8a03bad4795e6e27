"""Attention of drafted tokens on block tables (hata_dense_tree_paged) against attention in 64 bits of every token by itself."""
import ctypes
import math

import numpy as np
import pytest

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]

D = 128
JUNK = 0x7FC0  # bf16 NaN: a read of a row that belongs to nobody shows
KEPT = 0x1234  # what an output holds that nobody writes


@pytest.fixture(scope="module")
def hata():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2506_02572_amd import hata
    return hata


def i32(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


class Drafts:
    """Sequences of base[b] committed rows and draft[b] drafted ones; `gap` packed rows of nobody in front of the first, and 3 behind."""

    def __init__(self, hata, base, draft, Hq=8, Hkv=2, P=16, mask="tree", seed=0, max_draft=None, words=None, outliers=True, scale=None,
                 gap=0, L_cap=None, n_pages=None, spread=1.0):
        import torch
        rng = np.random.default_rng(seed)
        self.hata, self.B, self.Hq, self.Hkv, self.P, self.G = hata, len(base), Hq, Hkv, P, Hq // Hkv
        self.base, self.draft = list(base), list(draft)
        self.len = [a + n for a, n in zip(base, draft)]
        self.scale = scale if scale is not None else 1 / math.sqrt(D)
        self.most = max_draft or max(max(draft), 1)
        blocks = [-(-n // P) for n in self.len]
        self.width = max(max(blocks), 1) + 1
        self.n_pages = n_pages or sum(blocks) + 3
        pages = list(rng.permutation(self.n_pages)) if n_pages is None else list(range(self.n_pages - 1, self.n_pages - 1 - sum(blocks), -1))
        table = np.where(rng.random((self.B, self.width)) < 0.5, -1, 2 ** 31 - 1)
        for b, n in enumerate(blocks):
            table[b, :n] = [pages.pop(0) for _ in range(n)]
        self.table = table.astype(np.int32)
        self.start = gap + np.concatenate([[0], np.cumsum(draft)]).astype(np.int64)
        self.T = int(self.start[-1]) + 3
        self.words = words or -(-self.most // 32)
        self.seen = [self.visible(mask, n, rng) for n in draft]
        self.mask = None
        if mask != "chain":
            bits = rng.random((self.T, 32 * self.words)) < 0.5  # (bits of tokens that are not there mean nothing)
            for b, n in enumerate(draft):
                bits[self.start[b]:self.start[b + 1], :n] = self.seen[b]
            self.mask = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).cuda()
        g = torch.Generator(device="cuda").manual_seed(seed)
        size = torch.ones((Hkv, 1, D), device="cuda")
        if outliers:
            size[:, 0, rng.permutation(D)[:4]] = 8.0
        rand = lambda *s: torch.randn(s, device="cuda", generator=g)
        self.K, self.V = (torch.full((self.n_pages, Hkv, P, D), JUNK, dtype=torch.int16, device="cuda").view(torch.bfloat16) for _ in range(2))
        for b, n in enumerate(self.len):
            page, row = self.where(b, np.arange(n))
            for pool in (self.K, self.V):
                pool[page, :, row] = (rand(n, Hkv, D) * size[:, 0] * spread).to(torch.bfloat16)
        self.q = (rand(self.T, Hkv, self.G, D) * size * spread).to(torch.bfloat16).view(self.T, Hq, D)
        self.cap = L_cap or max(max(self.len), 64)
        self.ctx = hata.Context(self.B, Hq, Hkv, D, 32, self.cap, min(self.cap, 64))
        self.args = (i32(self.table), i32(self.base), i32(self.len), i32(self.start))
        self.scratch = self.ctx.hata_tree_scratch(self.B, self.T, self.most)
        self.out = torch.empty((self.T, Hq, D), dtype=torch.int16, device="cuda")
        self.out32 = torch.empty((self.T, Hq, D), dtype=torch.float32, device="cuda")

    @staticmethod
    def visible(kind, n, rng):
        if kind == "chain":
            return np.tril(np.ones((n, n), bool))
        if kind == "none":
            return np.zeros((n, n), bool)
        if kind == "any":  # not a tree: anything, rows without a token among them
            s = rng.random((n, n)) < rng.random((n, 1))
            s[::5] = False
            return s
        s = np.zeros((n, n), bool)
        for i in range(n):
            parent = int(rng.integers(max(-1, i - 6), i)) if i else -1
            if parent >= 0:
                s[i] = s[parent]
            s[i, i] = True
        return s

    def where(self, b, n):
        import torch
        return torch.from_numpy(self.table[b, n // self.P].astype(np.int64)).cuda(), torch.from_numpy(n % self.P).cuda()

    def exact(self, committed=True):
        """Outputs; sums of weight times absolute value; the largest sum of absolute products of a row (of scores in units of 1).
        committed False: without the committed rows."""
        import torch
        out = torch.zeros((self.T, self.Hq, D), dtype=torch.float64, device="cuda")
        size, products = torch.zeros_like(out), torch.zeros((self.T, self.Hq, 1), dtype=torch.float64, device="cuda")
        for b, n in enumerate(self.draft):
            t0, L = int(self.start[b]), self.len[b]
            if n == 0 or L == 0:
                continue
            see = torch.ones((n, L), dtype=torch.bool, device="cuda")
            see[:, :self.base[b]] = committed
            see[:, self.base[b]:] = torch.from_numpy(self.seen[b]).cuda()
            page, row = self.where(b, np.arange(L))
            K, V = self.K[page, :, row].double(), self.V[page, :, row].double()
            q = self.q[t0:t0 + n].double()
            for h in range(self.Hkv):
                for g in range(self.G):
                    x = q[:, h * self.G + g]
                    # a row that a token does not see has no part in it, whatever it holds
                    logit = torch.where(see, x @ K[:, h].T * self.scale, -math.inf)
                    p = torch.nan_to_num(torch.softmax(logit, 1), 0.0) if not bool(see.any(1).all()) else torch.softmax(logit, 1)
                    finite = torch.isfinite(V[:, h]).all(1)
                    v = torch.where(finite[:, None], V[:, h], 0.0)
                    o = p @ v
                    bad = (see & ~finite).any(1)
                    o[bad] = math.nan  # (looked at by nobody)
                    out[t0:t0 + n, h * self.G + g] = o
                    size[t0:t0 + n, h * self.G + g] = p @ v.abs()
                    products[t0:t0 + n, h * self.G + g, 0] = torch.where(see, torch.nan_to_num(x.abs() @ K[:, h].abs().T), 0.0).max(1).values * abs(self.scale)
        return out, size, products

    def run(self, stream=None, f32=True, fill=True):
        import torch
        if fill:
            self.out.fill_(KEPT)
            self.out32.fill_(7.0)
            torch.cuda.synchronize()
        t, base, lens, start = self.args
        self.ctx.hata_dense_tree_paged(self.q, self.K, self.V, t, self.width, self.P, self.n_pages, base, lens, self.B, start, self.T, self.most,
                                       self.mask, self.words if self.mask is not None else 0, self.scale, self.out, self.out32 if f32 else None,
                                       self.scratch, stream=stream)

    def check(self, ref=None, **kw):
        """The weights are two bf16 terms (2^-16 relative) at the most coarse, in numerator and denominator: 2^-15 (size + |o|). Scores are fp32
        sums of 128 products (some 16 roundings of 2^-24 of the sum of the absolute products), scaled and taken from the maximum: 2^-19 of it,
        which moves the weights by e^(2 d) - 1, twice as many in the quotient. fp32 sums over L rows: (L / 16 + 64) 2^-24 for either."""
        import torch
        self.run(**kw)
        torch.cuda.synchronize()
        want, size, products = ref if ref is not None else self.exact()
        owned = torch.zeros(self.T, dtype=torch.bool, device="cuda")
        for b, n in enumerate(self.draft):
            owned[int(self.start[b]):int(self.start[b]) + min(n, self.most)] = True
        fine = owned[:, None, None] & torch.isfinite(want)
        room = 2.0 ** -15 + 4 * 2.0 ** -19 * products + (max(self.len) / 16 + 64) * 2.0 ** -23
        err = (self.out32.double() - want).abs()
        bad = fine & ~(err <= room * (size + want.abs()))
        assert not bool(bad.any()), f"{int(bad.sum())} values off, first at {bad.nonzero()[0].tolist()}, by {float(err[bad].max()):.3e}"
        assert torch.equal(self.out.view(torch.bfloat16)[fine], self.out32.to(torch.bfloat16)[fine])
        assert bool((self.out[~owned] == KEPT).all()) and bool((self.out32[~owned] == 7.0).all())
        return err


@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (8, 4), (6, 2), (8, 2), (10, 2), (6, 1), (14, 2), (16, 2), (16, 1), (20, 2)])
@pytest.mark.parametrize("mask", ["tree", "chain", "any"])
def test_heads_and_lengths(hata, Hq, Hkv, mask):
    base = [0, 1, 15, 16, 17, 63, 64, 65, 127, 200, 0, 333]
    draft = [1, 3, 16, 1, 33, 2, 64, 5, 7, 40, 11, 0]
    s = Drafts(hata, base, draft, Hq, Hkv, mask=mask, seed=Hq * 7 + Hkv, gap=2)
    s.check()
    s.ctx.close()


@pytest.mark.parametrize("P", [16, 64, 256, 2048])
@pytest.mark.parametrize("draft", [1, 2, 31, 32, 33, 63, 64, 65, 100, 128, 255, 256])
def test_draft_sizes_and_pages(hata, P, draft):
    for mask in ("tree", "chain"):
        s = Drafts(hata, [500, 0, 77], [draft, draft, max(draft // 2, 1)], P=P, mask=mask, seed=draft + P)
        s.check()
        s.ctx.close()


@pytest.mark.parametrize("L", [1000, 4095, 20000, 70001])
@pytest.mark.parametrize("Hq,Hkv,draft", [(32, 8, 1), (32, 8, 7), (64, 8, 40), (40, 8, 13), (8, 8, 64)])
def test_long_contexts(hata, L, Hq, Hkv, draft):
    s = Drafts(hata, [L, L // 3], [draft, draft], Hq, Hkv, P=64, seed=L + draft)
    s.check()
    s.ctx.close()


@pytest.mark.parametrize("B,Hq,Hkv", [(70, 8, 2), (300, 8, 1), (33, 32, 32)])
def test_many_sequences(hata, B, Hq, Hkv):
    """Ragged batches, most of them without much, one of them long; sequences without tokens and without rows."""
    rng = np.random.default_rng(B)
    base, draft = rng.integers(0, 300, B), rng.integers(0, 20, B)
    base[B // 2], base[3] = 9000, 0
    s = Drafts(hata, base.tolist(), draft.tolist(), Hq, Hkv, seed=B, gap=1)
    s.check()
    s.ctx.close()


@pytest.mark.parametrize("B,Hq,Hkv,draft", [(257, 8, 1, 3), (700, 4, 4, 2), (1500, 2, 1, 5), (513, 8, 2, 40)])
def test_more_sequences_than_workgroups(hata, B, Hq, Hkv, draft):
    """Several sequences a workgroup and a thread; every seventh without tokens, the last one long."""
    rng = np.random.default_rng(B)
    base = rng.integers(0, 100, B)
    base[-1] = 5000
    s = Drafts(hata, base.tolist(), [0 if b % 7 == 3 else draft for b in range(B)], Hq, Hkv, seed=B)
    s.check()
    s.ctx.close()


@pytest.mark.parametrize("Hq,Hkv,draft,L", [(8, 2, 64, 30000), (4, 1, 256, 40000), (2, 1, 9, 100000), (8, 8, 256, 9000)])
def test_units_of_many_parts(hata, Hq, Hkv, draft, L):
    """One sequence, few units: a unit's rows in up to 256 parts, joined in batches."""
    s = Drafts(hata, [L], [draft], Hq, Hkv, P=64, seed=L)
    s.check()
    s.ctx.close()


@pytest.mark.parametrize("mask", ["none", "any"])
def test_tokens_that_see_nothing(hata, mask):
    """No committed rows and an empty mask: zeros."""
    import torch
    s = Drafts(hata, [0, 0, 40], [5, 70, 6], mask=mask, seed=9)
    s.check()
    t = int(s.start[0])
    assert not bool(s.out32[t:t + 1].any()) and not bool(s.out[t:t + 1].any())
    s.ctx.close()


@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("base,draft", [(0, 40), (50, 17), (300, 64), (64, 200)])
def test_rows_that_a_token_does_not_see(hata, what, base, draft):
    """Infinities and NaN in drafted rows, in K and in V: tokens that do not see them are as ever, the others are not finite."""
    import torch
    s = Drafts(hata, [base, 20], [draft, 9], mask="tree", seed=draft)
    bad = [draft // 3, draft - 1]
    for j in bad:
        page, row = s.where(0, np.array([base + j]))
        s.K[page, 0, row], s.V[page, 1, row, 5:9] = what, what
        s.V[page, 0, row], s.K[page, 1, row, 3] = what, -what
    hidden = ~torch.from_numpy(s.seen[0][:, bad].any(1)).cuda()
    assert bool(hidden.any()) and not bool(hidden.all())
    ref = s.exact()
    ref[0][int(s.start[0]):int(s.start[1])][~hidden] = math.nan
    s.check(ref)
    # the others: not finite where the formula over the rows that they see is not
    L = s.len[0]
    page, row = s.where(0, np.arange(L))
    K, V = s.K[page, :, row].double(), s.V[page, :, row].double()
    for i in np.flatnonzero(~hidden.cpu().numpy()):
        rows = torch.from_numpy(np.r_[np.arange(base), base + np.flatnonzero(s.seen[0][i])]).cuda()
        t = int(s.start[0]) + int(i)
        for h in range(s.Hq):
            p = torch.softmax((K[rows, h // s.G] * s.q[t, h].double()).sum(1) * s.scale, 0)
            want = (p[:, None] * V[rows, h // s.G]).sum(0)
            assert torch.equal(torch.isfinite(want), torch.isfinite(s.out32[t, h])), (t, h)
    s.ctx.close()


@pytest.mark.parametrize("draft", [1, 40])
def test_scores_of_minus_infinity(hata, draft):
    """Committed rows whose scores are -inf count for nothing; a token that sees no other row gives zeros, and no NaN."""
    s = Drafts(hata, [5000], [draft], mask="any", seed=draft, outliers=False)
    s.q.copy_(s.q.abs() + 1)  # (above zero: every product with -inf is -inf)
    page, row = s.where(0, np.arange(5000))
    s.K[page, :, row] = -math.inf
    s.check(s.exact(committed=False))
    blind = [int(s.start[0]) + i for i in range(draft) if not s.seen[0][i].any()]
    assert blind and not bool(s.out32[blind].any())
    s.ctx.close()


def test_scales_and_large_scores(hata):
    """Scales of zero and below, scores of hundreds, and scores that differ in the committed and the drafted rows."""
    for scale, spread in ((0.0, 1.0), (-0.1, 1.0), (1.0, 1.0), (0.5, 3.0), (1e-3, 1.0)):
        s = Drafts(hata, [400, 3], [20, 33], scale=scale, spread=spread, seed=5)
        s.check()
        s.ctx.close()
    import torch
    for factor in (30.0, 0.01):
        s = Drafts(hata, [300, 100], [20, 33], seed=6)
        for b in range(2):
            page, row = s.where(b, np.arange(s.base[b], s.len[b]))
            s.K[page, :, row] = (s.K[page, :, row].float() * factor).to(torch.bfloat16)
        s.check()
        s.ctx.close()


def test_lengths_that_do_not_fit(hata):
    """Requests that were not granted (no rows behind base_len), lengths and starts out of range, tokens behind max_draft, words to spare."""
    import torch
    s = Drafts(hata, [100, 60, 30, 200], [8, 8, 8, 8], max_draft=5, words=3, seed=2)
    # the tokens behind the first five are seen by nobody, and not written
    for b in range(4):
        s.seen[b][:, 5:] = False
    s.check()
    t, base, lens, start = s.args
    s.base[1], s.len[1] = 60, 60
    lens[1] = 60  # not granted
    s.seen[1] = np.zeros((8, 0), bool)
    lens[2] = -5  # no rows at all: zeros
    base[2] = 7
    s.len[2] = s.base[2] = 0
    s.check()
    assert not bool(s.out32[int(s.start[2]):int(s.start[2]) + 5].any())
    s.ctx.close()
    # a cache longer than the context or the table says is cut there; starts are clamped to the packed rows
    s = Drafts(hata, [100, 60], [8, 8], seed=3)
    s.args[2].fill_(2 ** 31 - 1)
    s.args[1].fill_(2 ** 31 - 1)
    s.args[3].copy_(i32([-7, 5, 10 ** 6]))
    s.run()
    torch.cuda.synchronize()
    s.args[3].copy_(i32([10 ** 6, 10 ** 6, 10 ** 6]))
    s.run()
    torch.cuda.synchronize()
    assert bool((s.out == KEPT).all())
    s.args[3].copy_(i32([0, 0, s.T]))
    s.run(f32=False)
    torch.cuda.synchronize()
    s.ctx.close()


def test_same_bits_every_time(hata):
    s = Drafts(hata, [5000, 300, 12], [64, 20, 33], 32, 8, seed=8)
    import torch
    s.check()
    first, first32 = s.out.clone(), s.out32.clone()
    for _ in range(3):
        s.scratch.random_()  # (carries nothing)
        s.run()
        torch.cuda.synchronize()
        assert torch.equal(s.out, first) and torch.equal(s.out32, first32)
    s.run(f32=False)
    torch.cuda.synchronize()
    assert torch.equal(s.out, first) and bool((s.out32 == 7.0).all())
    s.ctx.close()


def test_pools_beyond_4_gb(hata):
    s = Drafts(hata, [700, 3000], [20, 70], 32, 8, P=256, seed=4, n_pages=9000)
    s.check()
    s.ctx.close()


def test_two_calls_at_once_and_captured(hata):
    """Two batches on two streams with a scratch each; one call recorded and replayed with other inputs, with eager calls between."""
    import torch
    a, b = Drafts(hata, [3000, 100], [40, 9], 32, 8, seed=11), Drafts(hata, [900] * 5, [7] * 5, 32, 8, mask="chain", seed=12)
    refs = a.exact(), b.exact()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        for s, st in zip((a, b), streams):
            s.run(stream=st, fill=False)
    torch.cuda.synchronize()
    for s, ref in zip((a, b), refs):
        keep = s.out32.clone()
        s.check(ref)
        own = slice(0, int(s.start[-1]))
        assert torch.equal(keep[own], s.out32[own])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(streams[0]):
        with torch.cuda.graph(graph, stream=streams[0]):
            a.run(stream=streams[0], fill=False)
    for turn in range(5):
        a.q.normal_()
        if turn % 2:
            a.mask.random_(-2 ** 31, 2 ** 31 - 1)
            bits = np.unpackbits(a.mask.cpu().numpy().view(np.uint8), axis=1, bitorder="little").astype(bool)
            a.seen = [bits[a.start[i]:a.start[i + 1], :n] for i, n in enumerate(a.draft)]
        a.out.fill_(KEPT), a.out32.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = a.out32.clone()
        a.check()  # (eager)
        assert torch.equal(a.out32, replayed)
        b.run(fill=False)
    a.ctx.close(), b.ctx.close()


def test_refusals(hata):
    import torch
    s = Drafts(hata, [30, 10], [4, 4])
    t, base, lens, start = s.args
    lib = hata.load_library()
    s.out.fill_(KEPT)
    p = {"q": s.q.data_ptr(), "K": s.K.data_ptr(), "V": s.V.data_ptr(), "table": t.data_ptr(), "width": s.width, "P": 16, "pages": s.n_pages,
         "base": base.data_ptr(), "seq": lens.data_ptr(), "B": 2, "start": start.data_ptr(), "n": s.T, "most": 4, "mask": s.mask.data_ptr(),
         "words": 1, "scale": 1.0, "out": s.out.data_ptr(), "out32": s.out32.data_ptr(), "scratch": s.scratch.data_ptr(),
         "bytes": s.scratch.numel()}
    call = lambda **kw: lib.hata_dense_tree_paged(s.ctx._h, *dict(p, **kw).values(), None)
    for bad in [dict(B=0), dict(B=3), dict(width=0), dict(P=15), dict(P=24), dict(pages=0), dict(most=0), dict(n=-1), dict(words=0), dict(words=-1),
                dict(most=33, words=1)] + \
               [{k: None} for k in ("q", "K", "V", "table", "base", "seq", "start", "out")] + \
               [{k: p[k] + 8} for k in ("q", "K", "V", "out", "out32")] + [{k: p[k] + 2} for k in ("table", "base", "seq", "start", "mask")]:
        assert call(**bad) == -1, bad
    assert call(most=257, words=9) == -2 and call(n=2 ** 21) == -2
    for bad in (dict(scratch=None), dict(scratch=p["scratch"] + 16), dict(bytes=0)):
        assert call(**bad) == -3, bad
    n = ctypes.c_size_t(0)
    assert lib.hata_tree_scratch_bytes(s.ctx._h, 2, 8, 4, None) == -1 and lib.hata_tree_scratch_bytes(s.ctx._h, 3, 8, 4, ctypes.byref(n)) == -1
    assert lib.hata_tree_scratch_bytes(s.ctx._h, 2, -1, 4, ctypes.byref(n)) == -1 and lib.hata_tree_scratch_bytes(s.ctx._h, 2, 8, 0, ctypes.byref(n)) == -1
    assert lib.hata_tree_scratch_bytes(s.ctx._h, 2, 8, 257, ctypes.byref(n)) == -2
    assert call(n=0) == 0
    torch.cuda.synchronize()
    assert bool((s.out == KEPT).all())
    assert call(out32=None, mask=None, words=-5) == 0
    s.ctx.close()


def masked_by(s, seen):
    """Sequence by sequence, `seen` in the place of the masks."""
    import torch
    s.seen = seen
    bits = np.zeros((s.T, 32 * s.words), bool)
    for b, n in enumerate(s.draft):
        bits[s.start[b]:s.start[b + 1], :n] = seen[b]
    s.mask = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).cuda()


@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("base,draft,Hq,Hkv", [(0, 6, 8, 2), (40, 30, 8, 2), (5000, 12, 8, 2), (5000, 100, 8, 1), (700, 256, 8, 8)])
def test_scores_of_minus_infinity_of_rows_that_are_not_finite(hata, what, base, draft, Hq, Hkv):
    """A token that sees only rows whose scores are -inf gives zeros also where those rows' values are not finite: committed rows, and the first
    drafted one.  In one workgroup, and in parts that are joined."""
    s = Drafts(hata, [base], [draft], Hq, Hkv, mask="any", seed=draft, outliers=False)
    s.q.copy_(s.q.abs() + 1)  # (above zero: every product with -inf is -inf)
    page, row = s.where(0, np.arange(base + 1))
    s.K[page, :, row] = -math.inf
    page, row = s.where(0, np.r_[np.arange(0, base, 7), base])
    s.V[page, :, row] = what
    seen = s.seen[0].copy()
    seen[1::5] = False
    seen[1::5, 0] = True  # the first drafted row alone
    masked_by(s, [seen])
    s.run()
    import torch
    torch.cuda.synchronize()
    blind = [int(s.start[0]) + i for i in range(draft) if not seen[i, 1:].any()]
    assert len(blind) >= 2 + (draft - 1) // 5
    assert not bool(s.out32[blind].any()) and not bool(s.out.view(torch.bfloat16)[blind].float().any())
    assert bool((s.out[int(s.start[-1]):] == KEPT).all())
    s.ctx.close()


@pytest.mark.parametrize("Hq,Hkv,base,draft,mask", [
    (64, 8, "to 3000", [1, 100, 33, 64, 40, 97, 2, 65, 32, 80, 31, 100, 50, 1, 96, 34], "tree"),  # tiles of 32 tokens, last ones of 1 to 32
    (64, 8, "to 3000", [1, 100, 33, 64, 40, 97, 2, 65, 32, 80, 31, 100, 50, 1, 96, 34], "chain"),
    (40, 8, "to 300", [60, 256, 51, 52, 53, 103, 153, 204], "any"),                                # of 51
    (40, 8, "to 20000", [256, 255, 102, 60], "chain"),
    (32, 8, "to 900", [65, 128, 129, 64, 200, 256, 1, 63, 100], "tree"),                           # of 64
    (16, 1, "to 200", [33 if b % 3 else 17 for b in range(90)], "tree"),                           # of 16, more sequences than a wave looks at
    (16, 1, "to 60", [(7 * b) % 50 for b in range(300)], "any"),
    (28, 2, "to 3000", [(11 * b) % 200 for b in range(40)], "chain"),                              # of 18
    (32, 32, "to 700", [256, 256, 255, 200], "any"),                                               # of 256: one
])
def test_tiles_of_tokens_in_equal_pieces(hata, Hq, Hkv, base, draft, mask):
    """Sequences with several tiles of tokens, in batches of more than 64 units (a KV head of such a tile) or sequences: all units one behind
    the other in equal pieces, full tiles and last ones of other weights, a tile's mask, pieces that end inside a unit."""
    rng = np.random.default_rng(len(draft) + Hq)
    rows = rng.integers(0, int(base[3:]), len(draft))
    rows[len(draft) // 2], rows[0] = int(base[3:]), 0
    per = 256 // (Hq // Hkv)
    tiles = [-(-n // per) for n in draft]
    assert Hkv * sum(tiles) > 64 or len(draft) > 64
    assert max(tiles) > 1 or per == 256
    s = Drafts(hata, rows.tolist(), draft, Hq, Hkv, mask=mask, seed=Hq, gap=1)
    s.check()
    first = s.out32.clone()
    s.scratch.fill_(0xff)
    s.run()
    import torch
    torch.cuda.synchronize()
    assert torch.equal(s.out32, first)
    s.ctx.close()


@pytest.mark.parametrize("L_cap,width,cap", [(100, 8, 100), (4096, 8, 128), (4096, 7, 112), (97, 8, 97)])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (16, 1)])
def test_lengths_cut_and_starts_clamped(hata, L_cap, width, cap, Hq, Hkv):
    """A cache longer than the context or the table says is cut there, starts are clamped to the packed rows, a sequence's tokens to
    max_draft, base_len to the length: each against attention over what is left, and packed rows of no sequence as they were."""
    s = Drafts(hata, [120, 120], [8, 8], Hq, Hkv, seed=width, L_cap=L_cap, max_draft=8)
    s.width, s.table = width, np.ascontiguousarray(s.table[:, :width])
    most = 2 ** 31 - 1

    def case(lens, bases, starts, want_len, want_base, want_start):
        s.args = tuple(i32(a) for a in (s.table, bases, lens, starts))
        s.len, s.base, s.start = want_len, want_base, np.asarray(want_start)
        s.draft = [min(int(n), 8) for n in np.diff(want_start)]
        seen = []
        for b in range(2):  # no token sees more than the drafted rows that are there: those of the tokens that are there
            n = s.len[b] - s.base[b]
            assert 0 <= n <= s.draft[b]
            seen.append(np.random.default_rng(b).random((s.draft[b], n)) < 0.5)
        bits = np.ones((s.T, 32), bool)
        for b in range(2):
            t0 = int(s.start[b])
            bits[t0:t0 + s.draft[b], :seen[b].shape[1]] = seen[b]
        s.seen = seen
        import torch
        s.mask = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).cuda()
        s.check()
    T = s.T
    assert T == 19
    case([most, most], [most, most], [-7, 5, 10 ** 6], [cap, cap], [cap, cap], [0, 5, T])      # (14 rows, eight of which are tokens)
    case([most, cap + 1], [cap - 3, cap - 8], [0, 8, 16], [cap, cap], [cap - 3, cap - 8], [0, 8, 16])
    case([50, -5], [60, 7], [3, 9, 12], [50, 0], [50, 0], [3, 9, 12])                          # a base behind the length, no rows at all
    case([most, 90], [-9, 88], [0, 0, T], [0 + 0, 90], [0, 88], [0, 0, T])                     # no tokens in front: nothing of the first
    case([cap, cap], [cap, -1], [10 ** 6, 10 ** 6, 10 ** 6], [cap, 0], [cap, 0], [T, T, T])
    s.ctx.close()
