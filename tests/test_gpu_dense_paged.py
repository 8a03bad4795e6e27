"""Dense decode attention on block tables, alone and with rows that groups of sequences share (hata_dense_decode_paged),
against attention in 64 bits of every sequence by itself."""
import math

import numpy as np
import pytest

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]

D = 128
SCALE = 1.0 / math.sqrt(D)
JUNK = 0x7FC0  # bf16 NaN: a read of a row that belongs to nobody shows


@pytest.fixture(scope="module")
def hata():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2506_02572_amd import hata
    return hata


class World:
    """Sequences of the given lengths, members of group g with the same pages over the first shared[g] rows (whole pages)."""

    def __init__(self, lens, groups=(), Hq=8, Hkv=2, P=16, seed=0, outliers=True, L_cap=None):
        import torch
        rng = np.random.default_rng(seed)
        self.lens, self.Hq, self.Hkv, self.P, self.B = list(lens), Hq, Hkv, P, len(lens)
        self.starts, self.shared, at = [], [], 0
        blocks = [-(-n // P) for n in lens]
        owner = {}  # (sequence, block) -> first member of its group
        for members, rows in groups:
            self.starts.append(at)
            self.shared.append(rows)
            for b in range(at, at + members):
                for i in range(min(rows // P, blocks[b])):
                    owner[b, i] = min(m for m in range(at, at + members) if blocks[m] > i)
            at += members
        if groups:
            self.starts.append(at)
        self.width = max(max(blocks), 1) + 1
        need = sum(blocks) - sum(1 for (b, i), o in owner.items() if o != b)
        self.n_pages = need + 3
        pages = list(rng.permutation(self.n_pages))
        table = np.where(rng.random((self.B, self.width)) < 0.5, -1, 2 ** 31 - 1).astype(np.int64)
        for b in range(self.B):
            for i in range(blocks[b]):
                o = owner.get((b, i), b)
                table[b, i] = table[o, i] if o != b else pages.pop()
        self.table = table.astype(np.int32)
        g = torch.Generator(device="cuda").manual_seed(seed)
        scale = torch.ones((Hkv, 1, D), device="cuda")
        if outliers:
            scale[:, 0, rng.permutation(D)[:4]] = 8.0
        rand = lambda *s: torch.randn(s, device="cuda", generator=g)
        self.K, self.V = ((rand(self.n_pages, Hkv, P, D) * scale).to(torch.bfloat16) for _ in range(2))
        self.q = (rand(self.B, Hkv, Hq // Hkv, D) * scale).to(torch.bfloat16).view(self.B, Hq, D)
        # rows that no sequence has
        live = torch.zeros((self.n_pages, P), dtype=torch.bool, device="cuda")
        for b, n in enumerate(lens):
            r = np.arange(n)
            live[torch.from_numpy(table[b, r // P]).cuda(), torch.from_numpy(r % P).cuda()] = True
        for pool in (self.K, self.V):
            pool.view(torch.int16).masked_fill_(~live[:, None, :, None], JUNK)
        self.L_cap = L_cap or max(max(lens), 64)
        self.ctx = hata_module().Context(self.B, Hq, Hkv, D, 32, self.L_cap, min(self.L_cap, 64))

    def rows(self, pool, b):
        import torch
        n = np.arange(self.lens[b])
        page, row = torch.from_numpy(self.table[b, n // self.P].astype(np.int64)).cuda(), torch.from_numpy(n % self.P).cuda()
        return pool[page, :, row].double()  # [n, Hkv, D]

    scale = SCALE

    def exact(self):
        """The outputs, and per output the sum of weight times absolute value: what a relative error of the weights costs."""
        import torch
        out = torch.zeros((self.B, self.Hq, D), dtype=torch.float64, device="cuda")
        size = torch.zeros_like(out)
        G = self.Hq // self.Hkv
        for b, n in enumerate(self.lens):
            if n == 0:
                continue
            K, V = self.rows(self.K, b), self.rows(self.V, b)
            for h in range(self.Hkv):
                p = torch.softmax(self.q[b, h * G:(h + 1) * G].double() @ K[:, h].T * self.scale, dim=1)
                out[b, h * G:(h + 1) * G] = p @ V[:, h]
                size[b, h * G:(h + 1) * G] = p @ V[:, h].abs()
        return out, size

    def run(self, groups=True, stream=None, fill=True):
        import torch
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
        if not hasattr(self, "dev"):
            self.dev = (torch.from_numpy(self.table).cuda(), i32(self.lens), i32(self.starts), i32(self.shared))
            self.out = torch.full((self.B, self.Hq, D), JUNK, dtype=torch.int16, device="cuda")
            self.out32 = torch.full((self.B, self.Hq, D), float("nan"), device="cuda")
        t, lens, starts, shared = self.dev
        n = len(self.shared) if groups else 0
        if fill:
            self.out.fill_(JUNK)
            self.out32.fill_(float("nan"))
            torch.cuda.synchronize()
        self.ctx.hata_dense_decode_paged(self.q, self.K, self.V, t, self.width, self.P, self.n_pages, lens, self.B,
                                         starts if n else None, shared if n else None, n, self.scale, self.out, self.out32,
                                         stream=stream)
        return self.out, self.out32

    def check(self, groups=True, ref=None, **kw):
        """fp32 output o = sum p v / sum p: the weights p of shared rows are rounded to bf16, p (1 + d) with |d| <= 2^-8 (half a
        step), in both sums, which moves o by sum p d (v - o) / sum p, at most 2^-8 (sum p |v| + |o|) / sum p; the others are taken in
        two terms (2^-15) or as they are; logits of fp32 sums: |q.k| summed is below 2^9 here, 2^-24 of it for each of some ten
        roundings, below 2^-11 at most, an e-fold of that in the weights; the bf16 output is that, rounded."""
        import torch
        out, out32 = self.run(groups, **kw)
        torch.cuda.synchronize()
        want, size = ref if ref is not None else self.exact()
        rounded = 2.0 ** -8 if groups and self.shared else 0.0
        err = (out32.double() - want).abs() - rounded * (size + want.abs()) - 2.0 ** -11 * size
        assert bool((err <= 1e-30).all()), f"off by {float((out32.double() - want).abs().max()):.3e} (bound passed by {float(err.max()):.3e})"
        assert torch.equal(out.view(torch.bfloat16), out32.to(torch.bfloat16))
        return want, size


def hata_module():
    from paper_2506_02572_amd import hata
    return hata


@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 4), (6, 2), (8, 2), (10, 2), (16, 2), (16, 1), (13, 1)])
@pytest.mark.parametrize("P", [16, 64, 512])
def test_alone(hata, Hq, Hkv, P):
    World([1, 0, 15, 16, 17, 700, 33, 2047], Hq=Hq, Hkv=Hkv, P=P, seed=Hq + P).check()


@pytest.mark.parametrize("L", [1, 15, 16, 17, 127, 128, 129, 1000, 4097, 20011])
def test_one_sequence(hata, L):
    World([L], Hq=8, Hkv=2, P=16, seed=L).check()


def test_no_rows_at_all(hata):
    World([0, 0, 0]).check()
    World([0]).check()


def test_more_than_64_tiles_a_wave(hata):
    World([70001, 3, 9000], Hq=4, Hkv=1, P=16, seed=1).check()
    World([40000] * 40, Hq=8, Hkv=8, P=256, seed=2).check()


def test_many_sequences(hata):
    rng = np.random.default_rng(5)
    World(list(rng.integers(0, 300, 200)), Hq=4, Hkv=1, P=32, seed=3).check()


def test_equals_the_contiguous_cache(hata):
    """The same rows in a contiguous cache: the same result bit for bit."""
    import torch
    w = World([500, 64, 3001, 17], Hq=8, Hkv=2, P=64, seed=9, L_cap=3008)
    K, V = (torch.zeros((w.B, w.Hkv, w.L_cap, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for b, n in enumerate(w.lens):
        K[b, :, :n] = w.rows(w.K, b).transpose(0, 1).to(torch.bfloat16)
        V[b, :, :n] = w.rows(w.V, b).transpose(0, 1).to(torch.bfloat16)
    out, out32 = w.run()
    o2, o232 = torch.zeros_like(out), torch.zeros_like(out32)
    w.ctx.hata_dense_decode(w.q, K, V, w.dev[1], w.B, SCALE, o2, o232)
    torch.cuda.synchronize()
    assert torch.equal(out, o2) and torch.equal(out32, o232)


GROUPS = [
    ([300, 280, 257, 299], [(4, 256)]),                              # one group
    ([1024] * 3, [(3, 1024)]),                                       # nothing behind the shared rows
    ([100, 2000, 2100, 1999, 5, 900, 901, 0], [(1, 96), (3, 1984), (1, 0), (2, 896)]),  # groups of one, of none shared; one outside
    ([700, 0, 650, 0, 0, 641], [(6, 640)]),                          # padded places in a group
    ([0, 0, 0, 640], [(3, 640)]),                                    # a group without any row
    ([5000 + i for i in range(37)], [(37, 4992)]),                   # more query rows than a tile
    ([3000 + 7 * i for i in range(70)], [(33, 2992), (37, 1600)]),
    ([130] * 9, [(9, 112)]),                                         # shared rows that fill no tile
    ([40, 900, 900], [(3, 896)]),                                    # shorter than what the others share
]


@pytest.mark.parametrize("case", range(len(GROUPS)))
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (5, 1), (3, 3), (32, 2), (13, 1), (16, 8)])
def test_groups(hata, case, Hq, Hkv):
    lens, groups = GROUPS[case]
    World(lens, groups, Hq=Hq, Hkv=Hkv, P=16, seed=case).check()


@pytest.mark.parametrize("P", [16, 128, 1024])
@pytest.mark.parametrize("members", [2, 8, 16, 17, 64, 200])
def test_group_sizes(hata, P, members):
    rng = np.random.default_rng(members)
    shared = 5 * 1024
    World([shared + int(n) for n in rng.integers(0, 200, members)], [(members, shared)], Hq=8, Hkv=2, P=P, seed=members).check()


def test_long_shared_prompt(hata):
    World([60000 + i for i in (0, 3, 50, 700, 701)], [(5, 59968)], Hq=8, Hkv=1, P=32, seed=4).check()


def test_many_groups(hata):
    rng = np.random.default_rng(6)
    sizes = [int(n) for n in rng.integers(1, 5, 70)]
    groups = [(n, 16 * int(rng.integers(0, 40))) for n in sizes]
    lens = [s + int(rng.integers(0, 90)) for n, s in groups for _ in range(n)]
    World(lens, groups, Hq=4, Hkv=2, P=16, seed=6).check()


def test_groups_decide_only_how_rows_are_read(hata):
    """Groups whose device arrays are out of order or out of range: clamped, and the answer is the same as long as the pages are."""
    import torch
    w = World([600 + i for i in range(12)], [(12, 592)], Hq=8, Hkv=2, P=16, seed=8)
    ref = w.check()
    for starts, shared in (([-5, 12], [592]), ([0, 99], [592]), ([7, 3, 12], [592, 592]), ([0, 12, 4, 12], [592, 100, 592]),
                           ([3, 3, 3, 9], [5, 592, 320]), ([0, 12], [2 ** 31 - 1]), ([0, 12], [-4]), ([12, 12], [592])):
        w.dev = w.dev[:2] + tuple(torch.tensor(a, dtype=torch.int32, device="cuda") for a in (starts, shared))
        w.shared = shared
        if shared == [2 ** 31 - 1]:  # (members must have the same pages: clamped to the shortest, whose rows behind 592 are its own)
            continue
        w.check(ref=ref)


def test_bad_page_numbers_stay_inside_the_pools(hata):
    import torch
    w = World([300] * 4, [(4, 256)], Hq=8, Hkv=2, P=16)
    w.K.normal_()
    w.V.normal_()
    w.table[:, 3] = 2 ** 31 - 1
    w.table[:, 7] = -9
    clamped = World.__new__(World)
    clamped.__dict__.update(w.__dict__)
    clamped.table = np.clip(w.table, 0, w.n_pages - 1)
    w.check(ref=clamped.exact())
    w.check(groups=False, ref=clamped.exact())


def test_infinite_values_of_other_rows(hata):
    """Infinities and NaN behind a sequence's end, and in rows of the shared pages that only longer members have, do not count."""
    import torch
    w = World([40, 900, 900], [(3, 896)], Hq=8, Hkv=2, P=16, seed=2)
    ref = w.exact()
    page = int(w.table[1, 3])
    for pool in (w.K, w.V):
        pool[page, :, 5] = float("inf")
        pool[page, :, 6] = float("nan")
    out, out32 = w.run()
    torch.cuda.synchronize()
    err = (out32[0].double() - ref[0][0]).abs()
    assert bool((err <= 2.0 ** -8 * (ref[1][0] + ref[0][0].abs()) + 2.0 ** -11 * ref[1][0]).all())
    assert bool(out32[1:].isnan().any())


def test_large_logits(hata):
    """One row far above the others, at the end of the shared rows, in front of them, behind them: its value is the answer."""
    import torch
    for row in (0, 2000, 2047, 2048, 2100):
        w = World([2110] * 20, [(20, 2048)], Hq=8, Hkv=2, P=16, seed=row, outliers=False)
        w.q[:] = 2.0
        for b in range(w.B):
            w.K[int(w.table[b, row // 16]), :, row % 16] = 30.0
        w.check()


@pytest.mark.parametrize("B,Hkv", [(8, 2), (40, 8), (70, 16), (300, 8)])
def test_one_sequence_much_longer_than_the_others(hata, B, Hkv):
    for place in (0, B // 2, B - 1):
        lens = [1040 + i % 50 for i in range(B)]
        lens[place] = 20000
        World(lens, [(B, 1024)], Hq=2 * Hkv, Hkv=Hkv, P=16, seed=place).check()


@pytest.mark.parametrize("scale", [-SCALE, 0.0, 1e-30, 2.0])
def test_scales(hata, scale):
    w = World([2100 + i for i in range(20)], [(20, 2048)], Hq=8, Hkv=2, P=16, seed=5, outliers=False)
    w.scale = scale
    w.check()


@pytest.mark.parametrize("exponent", [-60, 60, 125])
def test_values_of_every_size(hata, exponent):
    """Values near the largest and smallest that the sums can hold: no weight is above 1, so nothing overflows on the way."""
    w = World([900 + i for i in range(20)], [(20, 832)], Hq=8, Hkv=2, P=16, seed=6, outliers=False)
    w.V.copy_((w.V.double() * 2.0 ** exponent / 4).to(w.V.dtype))
    w.check()


def test_one_kv_head_many_splits(hata):
    World([140000 + i for i in range(3)], [(3, 139968)], Hq=16, Hkv=1, P=32, seed=7).check()


def test_context_larger_than_the_batch(hata):
    w = World([700 + i for i in range(9)], [(5, 640), (4, 688)], Hq=8, Hkv=2, P=16, seed=8)
    w.ctx.close()
    w.ctx = hata.Context(300, 8, 2, D, 32, 4096, 64)
    w.check()
    w.check(groups=False)


def test_more_groups_than_are_looked_at(hata):
    """Pairs that share, 1100 of them: those behind the 1024th read their rows twice."""
    World([80 + i % 7 for i in range(2200)], [(2, 64)] * 1100, Hq=2, Hkv=1, P=16, seed=9, outliers=False).check()


def test_large_batches(hata):
    """Every sequence has the same rows and query: the answer of one, of all of them."""
    import torch
    one = World([100], Hq=2, Hkv=1, P=16, seed=10, outliers=False)
    want, _ = one.check()
    for B in (5000, 16384, 20000):
        ctx = hata.Context(B, 2, 1, D, 32, 112, 64)
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
        q = one.q.expand(B, 2, D).contiguous()
        table = torch.from_numpy(one.table).cuda().expand(B, one.width).contiguous()
        out = torch.full((B, 2, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        for groups in (0, 1, 2):
            ctx.hata_dense_decode_paged(q, one.K, one.V, table, one.width, 16, one.n_pages, i32([100] * B), B, i32([0, B // 3, B]),
                                        i32([64, 96]), groups, SCALE, out)
            torch.cuda.synchronize()
            assert bool(((out.double() - want).abs() <= 2.0 ** -6 * want.abs().max()).all()), (B, groups)
        ctx.close()


def test_pools_beyond_four_gigabytes(hata):
    """Pages at the far end of pools of 4.6 GB each: row offsets that pass 32 bits."""
    import torch
    w = World([520 + i for i in range(6)] + [333], [(6, 512)], Hq=16, Hkv=8, P=32, seed=11)
    far = 70000 - w.n_pages
    for name in ("K", "V"):
        pool = torch.empty((70000, w.Hkv, w.P, D), dtype=torch.bfloat16, device="cuda")
        pool[far:] = getattr(w, name)
        setattr(w, name, pool)
    w.table = np.where((w.table >= 0) & (w.table < w.n_pages), w.table + far, w.table).astype(np.int32)
    w.n_pages = 70000
    ref = w.check()
    w.check(groups=False, ref=ref)
    # rows written there through a slot map
    T = 300
    x = torch.randn((T, 2, w.Hkv, D), device="cuda").to(torch.bfloat16)
    slots = torch.arange(70000 * w.P - T, 70000 * w.P, dtype=torch.int32, device="cuda")
    codes = torch.zeros((70000, w.Hkv, w.P, 1), dtype=torch.int32, device="cuda")
    W = torch.randn((w.Hkv, D, 32), device="cuda")
    for n in (T, 100):  # both forms
        w.K[-T // w.P - 1:].zero_()
        codes.zero_()
        w.ctx.hata_write_slots(x[-n:, 0], x[-n:, 1], 2 * w.Hkv * D, D, slots[-n:], n, w.K, w.V, codes, w.P, w.n_pages, W)
        torch.cuda.synchronize()
        rows = w.K.transpose(1, 2)[-T // w.P - 1:].reshape(-1, w.Hkv, D)[-n:]
        assert torch.equal(rows, x[-n:, 0])
        bits = torch.einsum("thd,hdr->thr", x[-n:, 0].double(), W.double()) >= 0
        words = (bits.long() << torch.arange(32, device="cuda")).sum(2)
        got = codes.transpose(1, 2)[-T // w.P - 1:].reshape(-1, w.Hkv)[-n:].long() & 0xFFFFFFFF
        assert torch.equal(got, words)


def test_two_contexts_at_once(hata):
    import torch
    ws = [World([3000 + 7 * i for i in range(24)], [(24, 2992)], Hq=8, Hkv=2, P=16, seed=s) for s in (20, 21)]
    refs = [w.exact() for w in ws]
    streams = [torch.cuda.Stream() for _ in ws]
    for w in ws:
        w.run()
    torch.cuda.synchronize()
    for _ in range(10):
        for w, s in zip(ws, streams):
            w.run(stream=s, fill=False)
    torch.cuda.synchronize()
    for w, ref in zip(ws, refs):
        err = (w.out32.double() - ref[0]).abs() - 2.0 ** -8 * (ref[1] + ref[0].abs()) - 2.0 ** -11 * ref[1]
        assert bool((err <= 0).all())


def test_lengths_out_of_range_and_a_group_of_one_sequence(hata):
    """Lengths below zero count as zero, above the context's rows as those; one sequence alone may be called a group."""
    import torch
    w = World([640, 640, 0, 700], [(4, 640)], Hq=8, Hkv=2, P=16, seed=13, L_cap=640)
    w.lens = [640, 640, 0, 640]
    ref = w.exact()
    w.run()
    w.dev[1].copy_(torch.tensor([641, 2 ** 31 - 1, -7, 700], dtype=torch.int32))
    w.check(ref=ref)
    w.check(groups=False, ref=ref)
    one = World([300], [(1, 288)], Hq=8, Hkv=2, P=16, seed=14)
    one.check()
    # (and without the fp32 output)
    want = one.out.clone()
    one.out.zero_()
    t, lens, starts, shared = one.dev
    one.ctx.hata_dense_decode_paged(one.q, one.K, one.V, t, one.width, one.P, one.n_pages, lens, 1, starts, shared, 1, SCALE, one.out)
    torch.cuda.synchronize()
    assert torch.equal(one.out, want)


def test_pools_in_pinned_host_memory(hata):
    import torch
    w = World([700 + i for i in range(6)], [(6, 640)], Hq=8, Hkv=2, P=16, seed=15)
    ref = w.exact()
    slots = torch.arange(5, dtype=torch.int32, device="cuda") + 16 * int(w.table[0, 40])  # rows of a block that is a sequence's own
    x = torch.randn((5, 2, 2, D), device="cuda").to(torch.bfloat16)
    for name in ("K", "V"):
        host = torch.empty(getattr(w, name).shape, dtype=torch.bfloat16, pin_memory=True)
        host.copy_(getattr(w, name))
        setattr(w, name, host)
    w.check(ref=ref)
    w.check(groups=False, ref=ref)
    w.ctx.hata_write_slots(x[:, 0], x[:, 1], 4 * D, D, slots, 5, w.K, w.V, None, w.P, w.n_pages, None)
    torch.cuda.synchronize()
    page = int(w.table[0, 40])
    assert torch.equal(w.K[page, :, :5].transpose(0, 1), x[:, 0].cpu()) and torch.equal(w.V[page, :, :5].transpose(0, 1), x[:, 1].cpu())


def test_twice_the_same_and_captured(hata):
    import torch
    w = World([3000 + 7 * i for i in range(40)], [(20, 2992), (18, 1600)], Hq=8, Hkv=2, P=16, seed=12)
    ref = w.check()
    first = w.out32.clone()
    w.check(ref=ref)
    assert torch.equal(first, w.out32)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            w.run(fill=False)
    for turn in range(4):
        for lens, shared in ((w.lens, w.shared), ([n - 1000 for n in w.lens], [1984, 600])):
            w.dev[1].copy_(torch.tensor(lens, dtype=torch.int32))
            w.dev[3].copy_(torch.tensor(shared, dtype=torch.int32))
            w.out32.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            got = w.out32.clone()
            w.out32.fill_(float("nan"))
            w.run(fill=False)
            torch.cuda.synchronize()
            assert torch.equal(got, w.out32) and not bool(got.isnan().any())
            if lens is w.lens:
                assert torch.equal(got, first)


def test_on_another_stream_beside_other_work(hata):
    import torch
    w = World([800] * 6, [(6, 768)], seed=3)
    s = torch.cuda.Stream()
    ref = w.exact()
    torch.cuda.synchronize()
    a = torch.randn((2048, 2048), device="cuda")
    for _ in range(20):
        a = a @ a * 1e-3
    w.check(ref=ref, stream=s)


def test_refusals(hata):
    import torch
    lib = hata.load_library()
    ctx = hata.Context(4, 8, 2, D, 128, 512, 64)
    t = torch.zeros(65536, dtype=torch.int32, device="cuda")
    p = t.data_ptr()

    def call(h=ctx._h, q=p, K=p, V=p, table=p, max_blocks=8, P=16, n_pages=4, seq=p, B=4, gs=None, sl=None, n=0, out=p, out32=None):
        return lib.hata_dense_decode_paged(h, q, K, V, table, max_blocks, P, n_pages, seq, B, gs, sl, n, 1.0, out, out32, None)

    for bad in ({"h": None}, {"q": None}, {"K": None}, {"V": None}, {"table": None}, {"max_blocks": 0}, {"P": 8}, {"P": 24},
                {"n_pages": 0}, {"n_pages": 1 << 27}, {"max_blocks": 1 << 27}, {"seq": None}, {"B": 0}, {"B": 5}, {"n": -1},
                {"n": 5, "gs": p, "sl": p}, {"n": 1, "sl": p}, {"n": 1, "gs": p}, {"out": None}, {"q": p + 8}, {"K": p + 2},
                {"V": p + 8}, {"out": p + 4}, {"out32": p + 8}, {"seq": p + 1}, {"n": 1, "gs": p + 2, "sl": p}, {"table": p + 2}):
        assert call(**bad) == -1, bad
    ctx.close()
