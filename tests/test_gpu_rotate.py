"""Rotary positions of packed rows (hata_rotate) against the formula in extended precision: bits, layouts, strides, far and
negative positions, special values, the gradient, refusals."""
import ctypes

import numpy as np
import pytest

import rotary_reference as R

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]

D = 128
POSITIONS = [0, 1, -1, 2, 7, 100, 4095, 131071, 10 ** 6 + 3, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1]


@pytest.fixture(scope="module")
def hata():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2506_02572_amd import hata
    return hata


@pytest.fixture(scope="module")
def ctx(hata):
    c = hata.Context(1, 32, 8, D, 128, 64, 64)
    yield c
    c.close()


def dev(a):
    import torch
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


def random_bits(rng, *shape):
    import torch
    return torch.from_numpy(rng.standard_normal(shape)).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dims", [16, 32, 64, 96, 112, 128])
@pytest.mark.parametrize("T,heads", [(1, 1), (1, 40), (2, 3), (5, 8), (67, 9), (130, 33)])
def test_rows(hata, ctx, T, heads, dims, interleaved):
    """Heads inside wider rows, into rows of other strides; what lies between and around stays as it was."""
    import torch
    rng = np.random.default_rng(T * 1000 + heads + dims)
    x = random_bits(rng, T, heads + 3, D + 8)
    positions = np.resize(np.asarray(POSITIONS, np.int64), T)
    positions[len(POSITIONS):] = rng.integers(0, 200000, max(T - len(POSITIONS), 0))
    m = float(np.float32(1.2772588))
    freq, _ = hata.rotary_frequencies(dims, 10000.0)
    freq = np.asarray(freq)
    rotary = hata.Rotary(dev(freq), interleaved, m)
    xd, out = dev(x), torch.full((T + 1, heads + 1, D + 16), 0x1234, dtype=torch.int16, device="cuda")
    for back in (False, True):
        ctx.hata_rotate(xd[:, 1:], xd.stride(0), xd.stride(1), heads, dev(positions.astype(np.int32)), T, rotary, back, out,
                        out.stride(0), out.stride(1))
        got = out.cpu().numpy().view(np.uint16)
        part = x[:, 1:1 + heads, :D]
        y, size = R.turn(R.values(part), positions, freq, m, interleaved, back)
        R.check(got[:T, :heads, :D], y, size, f"back {back}")
        assert np.array_equal(got[:T, :heads, dims:D], part[..., dims:])
        assert np.all(got[T] == 0x1234) and np.all(got[:, heads] == 0x1234) and np.all(got[..., D:] == 0x1234)
    assert np.array_equal(xd.cpu().numpy().view(np.uint16), x)


def test_in_place_and_heads_that_share_a_row(hata, ctx):
    """out = x; and a stride of 0 between heads, one row read for all of them."""
    import torch
    rng = np.random.default_rng(5)
    x, positions = random_bits(rng, 101, 7, D), rng.integers(0, 5000, 101)
    freq = np.asarray(hata.rotary_frequencies(128, 500000.0, "bands", 8.0)[0])
    rotary = hata.Rotary(dev(freq))
    y, size = R.turn(R.values(x), positions, freq)
    xd, pd = dev(x), dev(positions.astype(np.int32))
    ctx.hata_rotate(xd, 7 * D, D, 7, pd, 101, rotary, False, xd, 7 * D, D)
    R.check(xd.cpu().numpy().view(np.uint16), y, size)
    xd, out = dev(x), torch.zeros((101, 7, D), dtype=torch.int16, device="cuda")
    ctx.hata_rotate(xd, 7 * D, 0, 7, pd, 101, rotary, False, out, 7 * D, D)
    for h in range(7):
        R.check(out[:, h].cpu().numpy().view(np.uint16), y[:, 0], size[:, 0])


@pytest.mark.parametrize("interleaved", [False, True])
def test_special_values(hata, ctx, interleaved):
    """Zeros, the smallest and largest numbers, infinities and NaN go by the formula; subnormal results are rounded like others."""
    import torch
    special = np.array([0x0000, 0x8000, 0x0001, 0x8001, 0x007f, 0x0080, 0x0081, 0x7f7f, 0xff7f, 0x3f80, 0x7f80, 0xff80, 0x7fc0], np.uint16)
    a, b = np.meshgrid(special, special)
    a, b = a.reshape(-1), b.reshape(-1)
    T = 12
    x = np.zeros((T, -(-a.size // 64), D), np.uint16)
    pa, pb = (slice(0, D, 2), slice(1, D, 2)) if interleaved else (slice(0, 64), slice(64, D))
    grid_a, grid_b = np.zeros(x.shape[1] * 64, np.uint16), np.zeros(x.shape[1] * 64, np.uint16)
    grid_a[:a.size], grid_b[:b.size] = a, b
    x[..., pa], x[..., pb] = grid_a.reshape(1, -1, 64), grid_b.reshape(1, -1, 64)
    positions = np.arange(T)
    freq = np.full(64, 0.7)
    out = torch.zeros(x.shape, dtype=torch.int16, device="cuda")
    ctx.hata_rotate(dev(x), x.shape[1] * D, D, x.shape[1], dev(positions.astype(np.int32)), T, hata.Rotary(dev(freq), interleaved), False,
                    out, x.shape[1] * D, D)
    got = out.cpu().numpy().view(np.uint16)
    with np.errstate(all="ignore"):
        y, size = R.turn(R.values(x), positions, freq, 1.0, interleaved)
        y64 = y.astype(np.float64)
        nan, huge = np.isnan(y64), ~np.isnan(y64) & (abs(y64) >= 2.0 ** 127 * (2 - 2.0 ** -8))  # (rounds to infinity)
    g = R.values(got)
    assert np.all(np.isnan(g[nan])) and np.array_equal(g[huge], np.where(y64[huge] > 0, np.inf, -np.inf))
    fine = ~nan & ~huge
    want, room = R.nearest(np.where(fine, y, 0))
    assert not np.any(fine & (g != want) & (room > size * R.EXT(2.0) ** -50))


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(hata, ctx, interleaved):
    """Back is the gradient: against the formula's by autograd in 64 bits, rounded, and against differences of the forward call."""
    import torch
    T, H, dims, m = 9, 3, 64, 1.25
    rng = np.random.default_rng(2)
    g, positions = random_bits(rng, T, H, D), rng.integers(0, 3000, T)
    freq = np.asarray(hata.rotary_frequencies(dims, 10000.0)[0])
    rotary = hata.Rotary(dev(freq), interleaved, m)
    pd = dev(positions.astype(np.int32))

    def call(bits, back):
        out = torch.zeros((T, H, D), dtype=torch.int16, device="cuda")
        ctx.hata_rotate(dev(bits), H * D, D, H, pd, T, rotary, back, out, H * D, D)
        return R.values(out.cpu().numpy().view(np.uint16))

    x = torch.zeros((T, H, D), dtype=torch.float64, requires_grad=True)
    t = torch.from_numpy(positions.astype(np.float64)[:, None] * freq)
    c, s = m * torch.cos(t)[:, None], m * torch.sin(t)[:, None]
    a, b = (x[..., 0:dims:2], x[..., 1:dims:2]) if interleaved else (x[..., :dims // 2], x[..., dims // 2:dims])
    ya, yb = a * c - b * s, a * s + b * c
    y = torch.cat([torch.stack([ya, yb], 3).flatten(2) if interleaved else torch.cat([ya, yb], 2), x[..., dims:]], 2)
    (y * torch.from_numpy(R.values(g))).sum().backward()
    got = call(g, True)
    err = np.abs(got - x.grad.numpy())
    assert np.all(err <= 2.0 ** -8 * np.abs(x.grad.numpy()) + 2.0 ** -50 * 16)  # (one rounding, half a step of bf16)
    # differences: the forward call is linear, so those of +-1 along channel i are exact but for a rounding of every output
    for i in (0, 1, 31, 32, 33, 63, 64, 127):
        e = np.zeros((T, H, D), np.float64)
        e[..., i] = 1.0
        up, down = call(R.to_bits(e), False), call(R.to_bits(-e), False)
        slope = ((up - down) / 2 * R.values(g)).sum(2)
        size = (np.abs(up) * np.abs(R.values(g))).sum(2)
        assert np.all(np.abs(slope - got[..., i]) <= 2.0 ** -8 * (size + np.abs(got[..., i])) * 1.01)


def test_large_calls(hata, ctx):
    """More rows than a launch has, with offsets above 2^31 elements."""
    import torch
    T = (1 << 20) + 3
    x = torch.zeros((T, D * 17), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    x[:, :D].normal_(generator=g)
    out = torch.zeros((T, 1, D), dtype=torch.bfloat16, device="cuda")
    positions = torch.arange(T, dtype=torch.int32, device="cuda")
    freq = np.asarray(hata.rotary_frequencies(128, 10000.0)[0])
    ctx.hata_rotate(x, x.stride(0), 0, 1, positions, T, hata.Rotary(dev(freq)), False, out, D, D)
    at = np.r_[0:50, (1 << 20) - 40:T]
    y, size = R.turn(x[at, None, :D].double().cpu().numpy(), at, freq)
    R.check(out[at].view(torch.int16).cpu().numpy().view(np.uint16), y, size)


def test_another_stream_and_a_graph(hata, ctx):
    import torch
    rng = np.random.default_rng(3)
    freq = np.asarray(hata.rotary_frequencies(128, 10000.0)[0])
    rotary = hata.Rotary(dev(freq))
    x, out = dev(random_bits(rng, 300, 40, D)), torch.zeros((300, 40, D), dtype=torch.int16, device="cuda")
    positions = dev(np.arange(300, dtype=np.int32))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            ctx.hata_rotate(x, 40 * D, D, 40, positions, 300, rotary, False, out, 40 * D, D)
    for turn in range(4):
        x.copy_(dev(random_bits(rng, 300, 40, D)))
        positions.add_(1)
        torch.cuda.synchronize()
        if turn == 2:
            ctx.hata_rotate(x, 40 * D, D, 40, positions, 300, rotary, False, out, 40 * D, D, stream=side)
        else:
            graph.replay()
        torch.cuda.synchronize()
        y, size = R.turn(R.values(x.cpu().numpy().view(np.uint16)), positions.cpu().numpy(), freq)
        R.check(out.cpu().numpy().view(np.uint16), y, size)


def test_refusals(hata, ctx):
    import torch
    lib = hata.load_library()
    x, out = torch.zeros((4, 2, D), dtype=torch.bfloat16, device="cuda"), torch.full((4, 2, D), 3.0, dtype=torch.bfloat16, device="cuda")
    pos, freq = torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(65, dtype=torch.float64, device="cuda")

    def call(x=x.data_ptr(), st=2 * D, sh=D, heads=2, pos=pos.data_ptr(), n=4, freq=freq.data_ptr(), dims=128, inter=0, out=out.data_ptr(),
             ost=2 * D, osh=D, struct=True):
        r = ctypes.byref(hata.hata_rotary(freq, dims, inter, 1.0)) if struct else None
        return lib.hata_rotate(ctx._h, x, st, sh, heads, pos, n, r, 0, out, ost, osh, None)
    assert call(n=0) == 0
    for bad in (dict(x=None), dict(x=x.data_ptr() + 2), dict(st=-8), dict(st=4), dict(sh=-8), dict(sh=12), dict(heads=0), dict(heads=70000),
                dict(pos=None), dict(pos=pos.data_ptr() + 2), dict(n=-1), dict(freq=None), dict(freq=freq.data_ptr() + 4),
                dict(inter=2), dict(inter=-1), dict(out=None), dict(out=out.data_ptr() + 8), dict(ost=-8), dict(osh=20), dict(struct=False)):
        assert call(**bad) == -1, bad
    for dims in (0, 8, 24, 136, 256, -16):
        assert call(dims=dims) == -2
    torch.cuda.synchronize()
    assert bool((out == 3.0).all())
    assert call() == 0
    with pytest.raises(hata.HataError):
        hata.Rotary(torch.zeros(64, dtype=torch.float32, device="cuda"))
    with pytest.raises(hata.HataError):
        hata.Rotary(torch.zeros(64, dtype=torch.float64))
