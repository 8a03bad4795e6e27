"""The accepted path's rows moved together (hata_keep_rows), against the same on the host; every row of the pools looked at."""
import ctypes

import numpy as np
import pytest

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]

D = 128


@pytest.fixture(scope="module")
def hata():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2506_02572_amd import hata
    return hata


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Caches:
    def __init__(self, hata, base, draft, Hkv=2, r=64, P=16, seed=0, L_cap=4096, spare=0):
        rng = np.random.default_rng(seed)
        self.hata, self.B, self.Hkv, self.P, self.Wd = hata, len(base), Hkv, P, r // 32
        self.base, self.len = np.asarray(base, np.int32), np.asarray(base, np.int32) + np.asarray(draft, np.int32)
        blocks = [-(-int(n) // P) for n in self.len]
        self.width, self.n_pages = max(max(blocks), 1) + 1, sum(blocks) + 2 + spare
        pages = list(rng.permutation(self.n_pages))
        self.table = np.where(rng.random((self.B, self.width)) < 0.5, -7, 2 ** 31 - 1).astype(np.int32)
        for b, n in enumerate(blocks):
            self.table[b, :n] = [pages.pop() for _ in range(n)]
        self.K, self.V = (rng.integers(-2 ** 15, 2 ** 15, (self.n_pages, Hkv, P, D)).astype(np.int16) for _ in range(2))
        self.codes = rng.integers(-2 ** 31, 2 ** 31, (self.n_pages, Hkv, P, self.Wd)).astype(np.int32) if r else None
        self.ctx = hata.Context(self.B, Hkv, Hkv, D, r or 32, L_cap, 64)

    def expect(self, path, n_path):
        pools = [p.copy() for p in (self.K, self.V, self.codes) if p is not None]
        before = [p.copy() for p in pools]
        kept = np.zeros(self.B, np.int32)
        for b in range(self.B):
            last, base = -1, int(self.base[b])
            for i in range(min(max(int(n_path[b]), 0), path.shape[1])):
                j = int(path[b, i])
                if j <= last or j >= int(self.len[b]) - base:
                    break
                last = j
                a, z = base + j, base + i
                for p, q in zip(pools, before):
                    p[self.table[b, z // self.P], :, z % self.P] = q[self.table[b, a // self.P], :, a % self.P]
                kept[b] = i + 1
        return pools, self.base + kept

    def call(self, path, n_path, stream=None):
        import torch
        if not hasattr(self, "dev"):
            self.dev = [None if p is None else dev(p) for p in (self.K, self.V, self.codes)]
            self.ints = [dev(p) for p in (self.table, self.base, self.len)]
            self.out = torch.full((self.B + 1,), -5, dtype=torch.int32, device="cuda")
        t, base, n = self.ints
        self.ctx.hata_keep_rows(*self.dev, t, self.width, self.P, self.n_pages, base, n, self.B, path, n_path, path.shape[1], self.out,
                                stream=stream)

    def check(self, path, n_path):
        import torch
        path, n_path = np.asarray(path, np.int32).reshape(self.B, -1), np.asarray(n_path, np.int32)
        want, lens = self.expect(path, n_path)
        self.call(dev(path), dev(n_path))
        torch.cuda.synchronize()
        got = [p.cpu().numpy() for p in self.dev if p is not None]
        assert all(np.array_equal(a, b) for a, b in zip(got, want))
        assert self.out.cpu().numpy().tolist() == lens.tolist() + [-5]


@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("r", [0, 32, 128, 256])
@pytest.mark.parametrize("Hkv", [1, 8])
def test_paths(hata, P, r, Hkv):
    rng = np.random.default_rng(P + r)
    base = [0, 1, 15, 16, 17, 63, 64, 200, 255, 300]
    draft = [40, 1, 2, 16, 5, 64, 33, 0, 256, 100]
    s = Caches(hata, base, draft, Hkv, r, P, seed=r)
    most = 40
    path, n_path = np.full((s.B, most), 9, np.int64), []
    for b, n in enumerate(draft):
        k = int(rng.integers(0, min(n, most) + 1))
        path[b, :k] = np.sort(rng.permutation(n)[:k])
        n_path.append(k)
    s.check(path, n_path)
    s.ctx.close()


@pytest.mark.parametrize("most", [1, 31, 32, 33, 64, 255, 256])
def test_long_paths(hata, most):
    """Everything, and everything but the first row (every source is the next row's target), over more than one turn of rows."""
    base, draft = [5, 250, 0, 31], [most, most + 1, 2 * most, most]
    s = Caches(hata, base, draft, r=256, seed=most)
    i = np.arange(most)
    s.check([i, i + 1, 2 * i + 1, i], [most, most, most, most])
    s.ctx.close()


def test_paths_that_break_off(hata):
    s = Caches(hata, [10] * 9 + [20], [12] * 9 + [0])
    path = [[0, 3, 3, 5], [4, 2, 6, 8], [-1, 2, 3, 4], [1, 5, 12, 13], [1, 2, 3, 4], [1, 2, 3, 4], [7, 8, 2 ** 31 - 1, 9], [-2 ** 31, 1, 2, 3],
            [11, 12, 13, 14], [0, 1, 2, 3]]
    s.check(path, [4, 4, 4, 4, -3, 100, 4, 4, 4, 4])
    s.ctx.close()


def test_pools_beyond_4_gb(hata):
    """A path in the last pages of pools of more than 2^32 bytes: as in pools that are those pages alone."""
    import torch
    s = Caches(hata, [700, 90], [60, 40], Hkv=8, r=128, P=256, seed=5)
    path = np.tile(np.arange(1, 33, dtype=np.int32), (2, 1))
    s.check(path, [32, 20])
    n, before = 9000, 9000 - s.n_pages
    big = []
    for p in (s.K, s.V, s.codes):
        t = torch.empty((n,) + p.shape[1:], dtype=dev(p).dtype, device="cuda")
        t[before:] = dev(p)
        big.append(t)
    assert big[0].numel() > 2 ** 31
    t = dev(np.where((s.table >= 0) & (s.table < s.n_pages), s.table + before, s.table).astype(np.int32))
    out = torch.full((3,), -5, dtype=torch.int32, device="cuda")
    s.ctx.hata_keep_rows(*big, t, s.width, s.P, n, s.ints[1], s.ints[2], 2, dev(path), dev(np.asarray([32, 20], np.int32)), 32, out)
    torch.cuda.synchronize()
    for a, b in zip(s.dev, big):
        assert torch.equal(a, b[before:])
    assert torch.equal(out, s.out)


def test_lengths_out_of_range(hata):
    """Lengths are clamped to the cache (base_len <= seq_len <= min(L_cap, table)), pages to the pools; nothing else is touched."""
    import torch
    s = Caches(hata, [16, 16, 16], [16, 16, 16], L_cap=64)
    path, n = dev(np.array([[1, 2], [1, 2], [1, 2]], np.int32)), dev(np.array([2, 2, 2], np.int32))
    s.call(path, n)
    torch.cuda.synchronize()
    # not granted (no rows behind base), a base above the length, a length below 0: nothing moves
    s.ints[1].copy_(dev(np.array([32, 40, 5], np.int32)))
    s.ints[2].copy_(dev(np.array([32, 20, -9], np.int32)))
    before = [p.clone() for p in s.dev]
    s.call(path, n)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(s.dev, before)) and s.out.tolist() == [32, 20, 0, -5]
    s.ints[2].copy_(dev(np.array([2 ** 31 - 1] * 3, np.int32)))  # the table has 48 rows: row 33, 34 of pages clamped to the pool
    s.ints[1].copy_(dev(np.array([32, 47, 48], np.int32)))
    s.call(path, n)
    torch.cuda.synchronize()
    assert s.out.tolist() == [34, 47, 48, -5]
    s.ctx.close()


def test_captured_and_on_another_stream(hata):
    import torch
    s = Caches(hata, [30, 5, 70], [20, 20, 20], r=128, P=16, seed=3)
    path, n_path = torch.zeros((3, 6), dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    s.call(path, n_path)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            s.call(path, n_path)
    rng = np.random.default_rng(4)
    for turn in range(5):
        s.K, s.V, s.codes = (p.cpu().numpy() for p in s.dev)
        p = np.stack([np.sort(rng.permutation(20)[:6]) for _ in range(3)]).astype(np.int32)
        n = rng.integers(0, 7, 3).astype(np.int32)
        want, lens = s.expect(p, n)
        path.copy_(dev(p)), n_path.copy_(dev(n))
        torch.cuda.synchronize()
        graph.replay() if turn != 2 else s.call(path, n_path, stream=side)
        torch.cuda.synchronize()
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(s.dev, want)) and s.out.tolist() == lens.tolist() + [-5]
    s.ctx.close()


def test_refusals(hata):
    import torch
    s = Caches(hata, [16, 16], [16, 16])
    path, n = dev(np.zeros((2, 4), np.int32)), dev(np.zeros(2, np.int32))
    s.call(path, n)
    torch.cuda.synchronize()
    t, base, length = s.ints
    lib = hata.load_library()
    p = {"K": s.dev[0].data_ptr(), "V": s.dev[1].data_ptr(), "codes": s.dev[2].data_ptr(), "table": t.data_ptr(), "width": s.width, "P": 16,
         "pages": s.n_pages, "base": base.data_ptr(), "seq": length.data_ptr(), "B": 2, "path": path.data_ptr(), "n": n.data_ptr(), "most": 4,
         "out": s.out.data_ptr()}
    call = lambda **kw: lib.hata_keep_rows(s.ctx._h, *dict(p, **kw).values(), None)
    for bad in [dict(B=0), dict(B=3), dict(width=0), dict(P=15), dict(P=24), dict(pages=0), dict(most=0), dict(most=-1), dict(width=2 ** 30)] + \
               [{k: None} for k in ("K", "V", "table", "base", "seq", "path", "n", "out")] + \
               [{k: p[k] + 8} for k in ("K", "V", "codes")] + [{k: p[k] + 2} for k in ("table", "base", "seq", "path", "n", "out")] + \
               [{"out": p[k]} for k in ("base", "seq", "n", "path")]:
        assert call(**bad) == -1, bad
    assert call(most=257) == -2
    assert call(codes=None) == 0 and call() == 0
    s.ctx.close()


def heads_of_a_workgroup(B, Hkv):
    """KV heads that a workgroup takes, so that the launch has up to 512 of them."""
    heads = 1
    while B * -(-Hkv // heads) > 512 and heads < Hkv:
        heads *= 2
    return heads


@pytest.mark.parametrize("B,Hkv,r,P,heads", [
    (256, 8, 256, 64, 4), (256, 8, 0, 16, 4),
    (200, 6, 128, 16, 4), (130, 5, 32, 16, 2),      # a tail of two heads, and of one
    (600, 3, 256, 16, 4), (520, 7, 64, 16, 8),      # all heads, no power of two, in one workgroup
    (5, 256, 256, 16, 4), (9, 100, 32, 16, 2),      # few sequences of many heads
    (40, 200, 32, 16, 32),                          # six workgroups of 32 heads and one of eight
    (129, 256, 32, 16, 128), (130, 300, 256, 16, 128),  # 128 heads: a turn in two parts of them; and a tail of 44
    (300, 140, 64, 16, 256)])                       # 140 heads, as many as 256 are laid out
def test_several_heads_a_workgroup(hata, B, Hkv, r, P, heads):
    """Batches in which a workgroup has several KV heads, some of them with fewer heads behind: paths of no row, of a few, and longer than a
    turn of rows (64 divided by the heads, but at least one)."""
    assert heads_of_a_workgroup(B, Hkv) == heads
    rng = np.random.default_rng(B + Hkv)
    draft = rng.integers(0, 13, B)
    base = rng.integers(0, 2 * P if Hkv <= 8 else 8, B)
    draft[0], base[0], draft[-1] = 12, 3, 12
    if heads <= 8:
        draft[1] = 200  # (several turns)
    s = Caches(hata, base, draft, Hkv, r, P, seed=Hkv, L_cap=64 if Hkv > 8 and heads > 8 else 1024)
    most = 100 if heads <= 8 else 12
    path, n_path = np.full((B, most), 5, np.int64), []
    for b, n in enumerate(draft):
        k = int(rng.integers(0, min(n, most) + 1)) if 1 < b < B - 1 else min(int(n), most) - (b == 0)
        path[b, :k] = np.sort(rng.permutation(n)[:k]) if b else 1 + np.arange(k)  # (the first: every source is the row behind its target)
        n_path.append(k)
    s.check(path, n_path)
    s.ctx.close()
