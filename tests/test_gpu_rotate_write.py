"""Packed rows rotated on the way into pages (hata_rotate_write_slots): keys, values, codes of the rotated keys and queries against
the formula in extended precision, every row of the pools looked at."""
import ctypes

import numpy as np
import pytest

import rotary_reference as R

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]

D, JUNK = 128, 0x7FC1


@pytest.fixture(scope="module")
def hata():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2506_02572_amd import hata
    return hata


def dev(a):
    import torch
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view({2: np.int16, 4: np.int32}[a.itemsize]) if a.dtype.kind == "u" else a).cuda()


def random_bits(rng, *shape):
    import torch
    return torch.from_numpy(rng.standard_normal(shape)).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


class Rows:
    """T packed rows of a fused projection (q, K, V heads), slots in random pages, some of them nowhere."""

    def __init__(self, hata, T, Hq=8, Hkv=2, r=128, P=16, dims=128, interleaved=False, m=1.0, seed=0, fused=True, far=100000, prepared=True):
        import torch
        rng = np.random.default_rng(seed * 7919 + T)
        self.hata, self.T, self.Hq, self.Hkv, self.r, self.P, self.interleaved, self.m = hata, T, Hq, Hkv, r, P, interleaved, m
        self.fused = fused
        self.x = random_bits(rng, T, Hq + 2 * Hkv, D)
        self.x[:, Hq:Hq + Hkv, rng.permutation(D)[:4]] = random_bits(rng, T, Hkv, 4)
        self.n_pages = -(-T // P) + 3
        self.slots = rng.permutation(self.n_pages * P)[:T].astype(np.int32)
        self.slots[rng.random(T) < 0.1] = -1
        if T > 3:
            self.slots[3], self.slots[T // 2] = self.n_pages * P, 2 ** 31 - 1  # not in the pools
        self.positions = rng.integers(-3, far, T).astype(np.int32)
        self.freq = np.asarray(hata.rotary_frequencies(dims, 10000.0)[0])
        self.rotary = hata.Rotary(dev(self.freq), interleaved, m)
        self.W = rng.standard_normal((Hkv, D, max(r, 32))).astype(np.float32) if r else None
        self.ctx = hata.Context(1, Hq, Hkv, D, r or 128, 64, 64)
        self.Wd = dev(self.W) if r else None
        if r and prepared:
            self.ctx.hata_prepare_weights(self.Wd)
        self.K = torch.full((self.n_pages, Hkv, P, D), JUNK, dtype=torch.int16, device="cuda")
        self.V = torch.full((self.n_pages, Hkv, P, D), JUNK, dtype=torch.int16, device="cuda")
        self.codes = torch.full((self.n_pages, Hkv, P, r // 32), 77, dtype=torch.int32, device="cuda") if r else None
        self.q_out = torch.full((T, Hq, D), JUNK, dtype=torch.int16, device="cuda")

    def call(self, queries=True, stream=None):
        xd, Hq, Hkv = dev(self.x), self.Hq, self.Hkv
        q, K, V = xd[:, :Hq], xd[:, Hq:Hq + Hkv], xd[:, Hq + Hkv:]
        if not self.fused:
            q, K, V = q.contiguous(), K.contiguous(), V.contiguous()
        self.ctx.hata_rotate_write_slots(q if queries else None, q.stride(0), q.stride(1), self.q_out if queries else None, K, V,
                                         K.stride(0), K.stride(1), dev(self.positions), dev(self.slots), self.T, self.rotary, self.K,
                                         self.V, self.codes, self.P, self.n_pages, self.Wd, stream=stream)
        import torch
        torch.cuda.synchronize()

    def check(self, queries=True):
        T, Hq, Hkv, P = self.T, self.Hq, self.Hkv, self.P
        rot = lambda bits: R.turn(R.values(bits), self.positions, self.freq, self.m, self.interleaved)
        host = lambda t: t.cpu().numpy().view({2: np.uint16, 4: np.uint32}[t.element_size()])
        if queries:
            R.check(host(self.q_out), *rot(self.x[:, :Hq]), "q")
        else:
            assert np.all(host(self.q_out) == JUNK)
        flat = lambda t: host(t).transpose(0, 2, 1, 3).reshape(self.n_pages * P, Hkv, -1)
        K, V = flat(self.K), flat(self.V)
        live = np.flatnonzero((self.slots >= 0) & (self.slots < self.n_pages * P))
        at = self.slots[live]
        y, size = rot(self.x[:, Hq:Hq + Hkv])
        held = R.check(K[at], y[live], size[live], "K")
        assert np.array_equal(V[at], self.x[live, Hq + Hkv:])
        rest = np.setdiff1d(np.arange(self.n_pages * P), at)
        assert np.all(K[rest] == JUNK) and np.all(V[rest] == JUNK)
        if self.r:
            codes = flat(self.codes)
            assert np.array_equal(codes[at], R.codes(held, self.W)) and np.all(codes[rest] == 77)


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 64, 128, 129, 300, 1100])
@pytest.mark.parametrize("r", [0, 32, 64, 96, 128, 256])
def test_widths_and_row_counts(hata, T, r):
    s = Rows(hata, T, r=r, seed=r)
    s.call()
    s.check()
    s.ctx.close()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dims", [16, 48, 64, 112, 128])
@pytest.mark.parametrize("T", [5, 400])
def test_layouts_of_pairs(hata, T, dims, interleaved):
    s = Rows(hata, T, dims=dims, interleaved=interleaved, m=1.3465735912322998, seed=dims)
    s.call()
    s.check()
    s.ctx.close()


@pytest.mark.parametrize("T,Hq,Hkv,r,P,fused,prepared", [
    (33, 32, 8, 128, 64, True, True), (200, 40, 8, 128, 256, False, True), (260, 32, 32, 256, 16, True, False),
    (1500, 64, 8, 128, 64, True, False), (140, 16, 1, 64, 32, False, False), (700, 8, 8, 32, 1024, True, True), (7, 24, 8, 256, 16, True, True),
    (3000, 32, 8, 128, 64, True, True), (2100, 4, 1, 256, 16, False, True),
    # many rows of few heads in one launch, few of many in two, and either side of where that changes
    (2048, 8, 1, 32, 64, True, True), (4096, 8, 1, 32, 64, True, True), (4097, 8, 1, 32, 64, False, False), (64, 32, 32, 256, 16, True, True),
    (48, 32, 32, 256, 64, False, False), (49, 32, 32, 256, 64, True, False), (17, 64, 64, 256, 16, True, True), (512, 16, 8, 64, 32, True, True),
    (513, 16, 8, 64, 32, True, True)])
def test_heads_pages_and_weights(hata, T, Hq, Hkv, r, P, fused, prepared):
    s = Rows(hata, T, Hq, Hkv, r, P, fused=fused, prepared=prepared, seed=P)
    s.call()
    s.check()
    s.ctx.close()


@pytest.mark.parametrize("T", [9, 500])
def test_without_queries_and_on_another_stream(hata, T):
    import torch
    s = Rows(hata, T, seed=4)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    s.call(queries=False, stream=side)
    s.check(queries=False)
    s.ctx.close()


@pytest.mark.parametrize("T", [40, 600])
def test_a_key_has_one_row_and_one_code(hata, T):
    """The same rows in calls of other sizes, by hata_rotate and hata_write_slots, and on top of what is there: the same bits."""
    import torch
    s = Rows(hata, T, seed=6)
    s.call()
    K, V, codes = s.K.clone(), s.V.clone(), s.codes.clone()
    s.K.fill_(JUNK), s.V.fill_(JUNK), s.codes.fill_(77)
    xd = dev(s.x)
    at = 0
    while at < T:  # in pieces
        n = min(T - at, 1 + at % 23)
        k, v = xd[at:at + n, s.Hq:s.Hq + s.Hkv], xd[at:at + n, s.Hq + s.Hkv:]
        s.ctx.hata_rotate_write_slots(None, 0, 0, None, k, v, k.stride(0), k.stride(1), dev(s.positions[at:at + n]), dev(s.slots[at:at + n]),
                                      n, s.rotary, s.K, s.V, s.codes, s.P, s.n_pages, s.Wd)
        at += n
    torch.cuda.synchronize()
    assert torch.equal(s.K, K) and torch.equal(s.V, V) and torch.equal(s.codes, codes)
    s.call()  # once more
    assert torch.equal(s.K, K) and torch.equal(s.V, V) and torch.equal(s.codes, codes)
    rows = torch.zeros((T, s.Hkv, D), dtype=torch.int16, device="cuda")
    k, v = xd[:, s.Hq:s.Hq + s.Hkv], xd[:, s.Hq + s.Hkv:].contiguous()
    s.ctx.hata_rotate(k, k.stride(0), D, s.Hkv, dev(s.positions), T, s.rotary, False, rows, s.Hkv * D, D)
    s.K.fill_(JUNK), s.V.fill_(JUNK), s.codes.fill_(77)
    s.ctx.hata_write_slots(rows, v, s.Hkv * D, D, dev(s.slots), T, s.K, s.V, s.codes, s.P, s.n_pages, s.Wd)
    torch.cuda.synchronize()
    assert torch.equal(s.K, K) and torch.equal(s.V, V) and torch.equal(s.codes, codes)
    s.ctx.close()


@pytest.mark.parametrize("T", [40, 1500])
def test_pools_beyond_4_gb(hata, T):
    """Rows in the last pages of pools of more than 2^32 bytes: as in pools that are those pages alone."""
    import torch
    few = Rows(hata, T, 32, 8, 128, 256, seed=21)
    few.slots[few.slots >= few.n_pages * 256] = -1
    few.call()
    few.check()
    many = Rows(hata, T, 32, 8, 128, 256, seed=21)
    many.n_pages = 9000
    before = many.n_pages - few.n_pages
    many.slots = np.where(few.slots >= 0, few.slots + before * 256, -1).astype(np.int32)
    held = [(t, torch.empty((many.n_pages,) + tuple(t.shape[1:]), dtype=t.dtype, device="cuda")) for t in (many.K, many.V, many.codes)]
    for small, big in held:
        big[before:] = small
    many.K, many.V, many.codes = (big for _, big in held)
    assert many.K.numel() > 2 ** 31
    many.call()
    for a, b in ((few.K, many.K), (few.V, many.V), (few.codes, many.codes)):
        assert torch.equal(a, b[before:])
    assert torch.equal(few.q_out, many.q_out)


def test_more_rows_than_a_launch_has(hata):
    """More than 2^20 rows in a call, as the same in calls of a third each."""
    import torch
    T, P, Hq, Hkv, r = (1 << 20) + 4321, 1024, 2, 1, 32
    n_pages = -(-T // P) + 1
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((T, Hq + 2 * Hkv, D), device="cuda", generator=g).to(torch.bfloat16)
    slots = torch.randperm(n_pages * P, device="cuda", generator=g)[:T].to(torch.int32)
    positions = torch.randint(0, 1 << 20, (T,), device="cuda", generator=g, dtype=torch.int32)
    W = torch.randn((Hkv, D, r), device="cuda", generator=g)
    ctx, rotary = hata.Context(1, Hq, Hkv, D, r, 64, 64), hata.Rotary.scaled(D, 10000.0)
    results = []
    for pieces in ([T], [T // 3, T // 3, T - 2 * (T // 3)]):
        K, V = (torch.zeros((n_pages, Hkv, P, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        codes, q_out = torch.zeros((n_pages, Hkv, P, r // 32), dtype=torch.int32, device="cuda"), torch.zeros((T, Hq, D), dtype=torch.bfloat16, device="cuda")
        t = 0
        for n in pieces:
            part = x[t:t + n]
            q, k, v = part[:, :Hq], part[:, Hq:Hq + Hkv], part[:, Hq + Hkv:]
            ctx.hata_rotate_write_slots(q, x.stride(0), x.stride(1), q_out[t:], k, v, x.stride(0), x.stride(1), positions[t:], slots[t:], n,
                                        rotary, K, V, codes, P, n_pages, W)
            t += n
        torch.cuda.synchronize()
        results.append((K, V, codes, q_out))
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.int16) if a.dtype == torch.bfloat16 else a, b.view(torch.int16) if b.dtype == torch.bfloat16 else b)
    assert torch.equal(results[0][1].transpose(1, 2).reshape(-1, D)[slots.long()], x[:, 3])
    ctx.close()


@pytest.mark.parametrize("T", [64, 400])
def test_values_out_of_the_ordinary(hata, T):
    """Rows of zeros, of the smallest and largest numbers and of infinities beside ordinary ones; weights of zeros."""
    s = Rows(hata, T, Hq=2, Hkv=1, seed=8, far=50)
    keys = s.x[:, 2]
    keys[0] = 0
    keys[1], keys[2] = 0x0001, 0x0100
    keys[4] = 0x7e00
    keys[5, ::2] = 0x8000
    s.slots[:6] = -1
    s.slots[[0, 1, 2, 4, 5]] = np.setdiff1d(np.arange(s.n_pages * s.P), s.slots)[:5]
    s.W[:, :, 5] = 0.0
    s.Wd.copy_(dev(s.W))
    s.ctx.hata_prepare_weights(s.Wd)
    s.call()
    s.check()
    s.ctx.close()


def test_captured_and_replayed(hata):
    """A call of few rows and one of many in one graph, replayed with other rows, with eager calls between."""
    import torch
    few, many = Rows(hata, 21, seed=10), Rows(hata, 700, seed=11)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    static = [(dev(s.x), dev(s.positions), dev(s.slots)) for s in (few, many)]

    def step(stream=None):
        for s, (x, pos, slots) in zip((few, many), static):
            q, k, v = x[:, :s.Hq], x[:, s.Hq:s.Hq + s.Hkv], x[:, s.Hq + s.Hkv:]
            s.ctx.hata_rotate_write_slots(q, x.stride(0), D, s.q_out, k, v, x.stride(0), D, pos, slots, s.T, s.rotary, s.K, s.V, s.codes,
                                          s.P, s.n_pages, s.Wd, stream=stream)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    rng = np.random.default_rng(12)
    for turn in range(5):
        for s, (x, pos, slots) in zip((few, many), static):
            s.x, s.positions = random_bits(rng, *s.x.shape), rng.integers(0, 9999, s.T).astype(np.int32)
            x.copy_(dev(s.x)), pos.copy_(dev(s.positions))
            for t in (s.K, s.V, s.q_out):
                t.fill_(JUNK)
            s.codes.fill_(77)
        torch.cuda.synchronize()
        step() if turn == 3 else graph.replay()
        torch.cuda.synchronize()
        few.check(), many.check()
    few.ctx.close(), many.ctx.close()


def test_refusals(hata):
    import torch
    s = Rows(hata, 8, seed=1)
    lib, rot = hata.load_library(), s.rotary.ref
    x = dev(s.x)
    p = {"q": x.data_ptr(), "qst": 12 * D, "qsh": D, "q_out": s.q_out.data_ptr(), "K_new": x.data_ptr(), "V_new": x.data_ptr(), "st": 12 * D,
         "sh": D, "pos": dev(s.positions).data_ptr(), "slots": dev(s.slots).data_ptr(), "n": 8, "rot": rot, "K": s.K.data_ptr(),
         "V": s.V.data_ptr(), "codes": s.codes.data_ptr(), "P": 16, "pages": s.n_pages, "W": s.Wd.data_ptr()}
    call = lambda **kw: lib.hata_rotate_write_slots(s.ctx._h, *dict(p, **kw).values(), None)
    for bad in [dict(q=None), dict(q_out=None), dict(codes=None), dict(W=None), dict(rot=None), dict(n=-1), dict(P=17), dict(P=8), dict(pages=0),
                dict(qst=-8), dict(qsh=4), dict(st=-8), dict(sh=12), dict(pages=2 ** 30)] + \
               [{k: None} for k in ("K_new", "V_new", "pos", "slots", "K", "V")] + \
               [{k: p[k] + 8} for k in ("q", "q_out", "K_new", "V_new", "K", "V", "codes", "W")] + [{k: p[k] + 2} for k in ("pos", "slots")]:
        assert call(**bad) == -1, bad
    assert call(rot=ctypes.byref(hata.hata_rotary(s.rotary.freq.data_ptr(), 120, 0, 1.0))) == -2
    assert call(n=0) == 0
    torch.cuda.synchronize()
    assert bool((s.K == JUNK).all()) and bool((s.q_out == JUNK).all())
    assert call(q=None, q_out=None, qst=-1, qsh=3) == 0  # (strides of nothing)
    s.ctx.close()
