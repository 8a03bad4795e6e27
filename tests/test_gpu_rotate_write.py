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


# ---- calls that go by two launches: rows rotated into the slots, and their codes from there on the matrix cores ----

def launches(s, queries=True):
    """One, or two where its workgroups would be more than two a compute unit: 16 rows and 64 hash columns of a KV head each (32 where
    the width is no multiple of 64), and one more for its queries."""
    columns = s.r // (64 if s.r % 64 == 0 else 32) + (1 if queries else 0)
    return 2 if s.r in (32, 64, 128, 256) and columns * s.Hkv * -(-s.T // 16) > 512 else 1


def check_all(s, queries=True):
    """As Rows.check, with rows that are not finite or overflow: infinities and NaN where the formula has them, and bits of NaN 0."""
    host = lambda t: t.cpu().numpy().view({2: np.uint16, 4: np.uint32}[t.element_size()])
    flat = lambda t: host(t).transpose(0, 2, 1, 3).reshape(s.n_pages * s.P, s.Hkv, -1)

    def held(got, bits, positions, what):
        with np.errstate(invalid="ignore"):
            y, size = R.turn(R.values(bits), positions, s.freq, s.m, s.interleaved)
        whole = np.isfinite(y)
        want = R.check(np.where(whole, got, 0).astype(np.uint16), np.where(whole, y, 0), np.where(whole, size, 1), what)
        assert not (abs(want) >= 2.0 ** 128).any()  # (no finite row here overflows)
        want = np.where(whole, want, y.astype(np.float64))
        assert np.array_equal(np.isnan(R.values(got)), np.isnan(want)) and np.array_equal(R.values(got)[~np.isnan(want)], want[~np.isnan(want)]), what
        return want
    if queries:
        held(host(s.q_out), s.x[:, :s.Hq], s.positions, "q")
    else:
        assert np.all(host(s.q_out) == JUNK)
    live = np.flatnonzero((s.slots >= 0) & (s.slots < s.n_pages * s.P))
    at = s.slots[live]
    K, V, codes = flat(s.K), flat(s.V), flat(s.codes)
    keys = held(K[at], s.x[live, s.Hq:s.Hq + s.Hkv], s.positions[live], "K")
    assert np.array_equal(V[at], s.x[live, s.Hq + s.Hkv:])
    with np.errstate(invalid="ignore"):
        want = np.stack([keys[:, h] @ s.W[h].astype(np.float64) >= 0 for h in range(s.Hkv)], 1)  # (NaN: false)
    assert np.array_equal(codes[at], np.packbits(want, axis=2, bitorder="little").view(np.uint32))
    rest = np.setdiff1d(np.arange(s.n_pages * s.P), at)
    assert np.all(K[rest] == JUNK) and np.all(V[rest] == JUNK) and np.all(codes[rest] == 77)
    return live


@pytest.mark.parametrize("T,Hq,Hkv,r", [(64, 2, 1, 128), (3000, 2, 1, 128), (3100, 4, 2, 64), (9000, 2, 1, 32), (1000, 2, 2, 256), (500, 4, 4, 256)])
@pytest.mark.parametrize("prepared", [True, False])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rows_out_of_the_ordinary_by_one_launch_and_two(hata, T, Hq, Hkv, r, prepared, interleaved):
    """Rows of zeros, of the smallest and large numbers, of infinities, of NaN, all over the workgroups' rows; columns of zero weights."""
    s = Rows(hata, T, Hq=Hq, Hkv=Hkv, r=r, seed=8, far=50, prepared=prepared, interleaved=interleaved)
    assert launches(s) == (1 if T == 64 else 2)
    rng = np.random.default_rng(T)
    s.positions[::7] = 0  # (an angle of zero: what is infinite makes its pair NaN)
    keys = s.x[:, Hq:Hq + Hkv]
    kinds = rng.permutation(T)[:max(T // 3, 18)]  # a third of the rows, some of every kind
    for i, t in enumerate(kinds):
        kind = i % 9
        if kind == 0:
            keys[t] = 0
        elif kind == 1:
            keys[t] = 0x8000
        elif kind == 2:
            keys[t] = rng.choice(np.array([0x0001, 0x8001, 0x0003, 0x0080, 0], np.uint16), keys[t].shape)  # subnormals
        elif kind == 3:
            keys[t] = 0x0100
        elif kind == 4:
            keys[t] = rng.choice(np.array([0x7e00, 0xfe00, 0x7d33], np.uint16), keys[t].shape)
        elif kind == 5:
            keys[t, :, rng.integers(D)] = 0x7f80
        elif kind == 6:
            keys[t, :, rng.integers(D)] = 0xff80
        elif kind == 7:
            keys[t, :, [3, 3 + D // 2]] = 0x7f80  # a pair of halves
            keys[t, :, [10, 11]] = 0xff80         # and of neighbours
        else:
            keys[t, :, rng.integers(D)] = 0x7fc0
    s.W[:, :, 5], s.W[:, :, r - 1] = 0.0, 0.0
    s.Wd.copy_(dev(s.W))
    if prepared:
        s.ctx.hata_prepare_weights(s.Wd)
    s.call()
    live = check_all(s)
    assert len(np.intersect1d(live, kinds)) > len(kinds) // 2
    s.ctx.close()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dims", [16, 48, 64, 112])
def test_layouts_of_pairs_by_two_launches(hata, dims, interleaved):
    s = Rows(hata, 3000, dims=dims, interleaved=interleaved, m=1.3465735912322998, seed=dims)
    assert launches(s) == 2
    s.call()
    s.check()
    s.ctx.close()


@pytest.mark.parametrize("T,Hkv,r", [(3000, 2, 128), (5000, 2, 64), (700, 8, 256), (9000, 1, 32)])
def test_without_queries_by_two_launches(hata, T, Hkv, r):
    import torch
    s = Rows(hata, T, Hkv=Hkv, r=r, seed=4)
    assert launches(s, queries=False) == 2
    torch.cuda.synchronize()
    s.call(queries=False, stream=torch.cuda.Stream())
    s.check(queries=False)
    s.ctx.close()


@pytest.mark.parametrize("T,Hkv,r,prepared", [(3000, 2, 128, True), (3000, 2, 128, False), (5000, 2, 64, True), (600, 8, 256, True), (9000, 1, 32, True)])
def test_one_launch_and_two_give_the_same_bits(hata, T, Hkv, r, prepared):
    """The same rows by one call of two launches, by calls of one launch, and by hata_rotate and hata_write_slots; projections next to
    zero among them (columns of weights that a key's first channels cancel in)."""
    import torch
    s = Rows(hata, T, Hkv=Hkv, r=r, seed=6, prepared=prepared)
    # weights of few bits against keys of few values: sums that are zero, or a unit in the last place from it
    s.W[:, :, 1::4] = np.rint(s.W[:, :, 1::4])
    s.x[::3, s.Hq:s.Hq + Hkv, 4:] = 0
    s.positions[::3] = 0
    s.Wd.copy_(dev(s.W))
    if prepared:
        s.ctx.hata_prepare_weights(s.Wd)
    assert launches(s) == 2 and launches(s, queries=False) == 2
    s.call()
    s.check()
    results = [s.K.clone(), s.V.clone(), s.codes.clone(), s.q_out.clone()]
    reset = lambda: (s.K.fill_(JUNK), s.V.fill_(JUNK), s.codes.fill_(77), s.q_out.fill_(JUNK))
    same = lambda: all(torch.equal(a, b) for a, b in zip(results, (s.K, s.V, s.codes, s.q_out)))
    reset()
    xd, pos, slots = dev(s.x), dev(s.positions), dev(s.slots)
    q, k, v = xd[:, :s.Hq], xd[:, s.Hq:s.Hq + Hkv], xd[:, s.Hq + Hkv:]
    at, piece = 0, 16 * (512 // (Hkv * (-(-r // 64) + 1)))
    while at < T:
        n = min(piece - at % 5, T - at)
        part, s.T = s.T, n
        assert launches(s) == 1
        s.T = part
        s.ctx.hata_rotate_write_slots(q[at:], xd.stride(0), D, s.q_out[at:], k[at:], v[at:], xd.stride(0), D, pos[at:], slots[at:], n, s.rotary,
                                      s.K, s.V, s.codes, s.P, s.n_pages, s.Wd)
        at += n
    torch.cuda.synchronize()
    assert same()
    s.call()  # once more, on top of what is there
    assert same()
    reset()
    rows = torch.zeros((T, Hkv, D), dtype=torch.int16, device="cuda")
    s.ctx.hata_rotate(k, xd.stride(0), D, Hkv, pos, T, s.rotary, False, rows, Hkv * D, D)
    s.ctx.hata_rotate(q, xd.stride(0), D, s.Hq, pos, T, s.rotary, False, s.q_out, s.Hq * D, D)
    s.ctx.hata_write_slots(rows, v.contiguous(), Hkv * D, D, slots, T, s.K, s.V, s.codes, s.P, s.n_pages, s.Wd)
    torch.cuda.synchronize()
    assert same()
    s.ctx.close()


def test_two_launches_captured_and_replayed(hata):
    """A call of one launch and one of two in one graph, replayed with other rows and slots, with eager calls between."""
    import torch
    few, many = Rows(hata, 21, seed=10), Rows(hata, 3000, seed=11)
    assert launches(few) == 1 and launches(many) == 2
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    static = [(dev(s.x), dev(s.positions), dev(s.slots)) for s in (few, many)]

    def step():
        for s, (x, pos, slots) in zip((few, many), static):
            q, k, v = x[:, :s.Hq], x[:, s.Hq:s.Hq + s.Hkv], x[:, s.Hq + s.Hkv:]
            s.ctx.hata_rotate_write_slots(q, x.stride(0), D, s.q_out, k, v, x.stride(0), D, pos, slots, s.T, s.rotary, s.K, s.V, s.codes,
                                          s.P, s.n_pages, s.Wd)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    rng = np.random.default_rng(12)
    for turn in range(5):
        for s, (x, pos, slots) in zip((few, many), static):
            s.x, s.positions = random_bits(rng, *s.x.shape), rng.integers(0, 9999, s.T).astype(np.int32)
            s.slots = rng.permutation(s.n_pages * s.P)[:s.T].astype(np.int32)
            s.slots[rng.random(s.T) < 0.2] = -1
            x.copy_(dev(s.x)), pos.copy_(dev(s.positions)), slots.copy_(dev(s.slots))
            for t in (s.K, s.V, s.q_out):
                t.fill_(JUNK)
            s.codes.fill_(77)
        torch.cuda.synchronize()
        step() if turn == 3 else graph.replay()
        torch.cuda.synchronize()
        few.check(), many.check()
    few.ctx.close(), many.ctx.close()
