"""Packed rows written through a slot map (hata_write_slots): rows bit for bit, key codes equal to an evaluation in 64 bits."""
import numpy as np
import pytest

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]

D = 128
JUNK16, JUNK32 = 0x7FC1, 0x5A5A5A5A


@pytest.fixture(scope="module")
def hata():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2506_02572_amd import hata
    return hata


def to_f64(bits):
    return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def bf16(x):
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def pack(bits):
    return np.packbits(bits, axis=-1, bitorder="little").view(np.uint32)


def make(seed, T, Hkv, r, P, pad=3, spare=2):
    rng = np.random.default_rng(seed)
    K, V = (bf16(rng.standard_normal((T, Hkv, D))) for _ in range(2))
    W = (rng.standard_normal((Hkv, D, r)) / np.sqrt(D)).astype(np.float32)
    n_pages = -(-T // P) + spare
    slots = rng.permutation(n_pages * P)[:T].astype(np.int32)
    if pad and T > 2 * pad:  # rows that go nowhere: negative, behind the pools
        slots[rng.choice(T, pad, replace=False)] = [-1, n_pages * P, 2 ** 31 - 1][:pad]
    return K, V, W, slots, n_pages


def expect(K, V, W, slots, n_pages, P):
    T, Hkv, _ = K.shape
    pools = [np.full((n_pages, Hkv, P, D), JUNK16, np.uint16) for _ in range(2)]
    words = 0 if W is None else W.shape[2] // 32
    codes = np.full((n_pages, Hkv, P, words), JUNK32, np.uint32)
    live = np.flatnonzero((slots >= 0) & (slots < n_pages * P))
    page, row = slots[live] // P, slots[live] % P
    pools[0][page, :, row], pools[1][page, :, row] = K[live], V[live]
    if W is not None:
        with np.errstate(invalid="ignore"):
            for h in range(Hkv):
                codes[page, h, row] = pack(to_f64(K[live, h]) @ W[h].astype(np.float64) >= 0)
    return pools[0], pools[1], codes


def layout(torch, K, V, how):
    """The same rows in memory of another order: (K, V, stride_t, stride_h)."""
    T, Hkv, _ = K.shape
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda()
    if how == "packed":
        return dev(K), dev(V), Hkv * D, D
    if how == "heads_first":
        return dev(K.transpose(1, 0, 2)), dev(V.transpose(1, 0, 2)), D, T * D
    fused = np.full((T, 2 + 2 * Hkv, D + 8), JUNK16, np.uint16)  # (rows with a gap behind them)
    fused[:, 2:2 + Hkv, :D], fused[:, 2 + Hkv:, :D] = K, V
    x = dev(fused)
    return x[:, 2:], x[:, 2 + Hkv:], x.stride(0), x.stride(1)


def check(hata, K, V, W, slots, n_pages, P, how="packed", codes=True, prepared=False, stream=None):
    import torch
    T, Hkv, _ = K.shape
    r = W.shape[2]
    ref = expect(K, V, W if codes else None, slots, n_pages, P)
    Kd, Vd, st, sh = layout(torch, K, V, how)
    ctx = hata.Context(1, Hkv, Hkv, D, r, 64, 64)
    Wd = torch.from_numpy(W).cuda()
    if prepared:
        ctx.hata_prepare_weights(Wd)
    sd = torch.from_numpy(slots).cuda()
    pools = [torch.full((n_pages, Hkv, P, D), JUNK16, dtype=torch.int16, device="cuda") for _ in range(2)]
    cd = torch.full((n_pages, Hkv, P, r // 32), JUNK32, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    for _ in range(2):
        ctx.hata_write_slots(Kd, Vd, st, sh, sd, T, pools[0], pools[1], cd if codes else None, P, n_pages, Wd if codes else None,
                             stream=stream)
    torch.cuda.synchronize()
    assert np.array_equal(pools[0].cpu().numpy().view(np.uint16), ref[0]), "K"
    assert np.array_equal(pools[1].cpu().numpy().view(np.uint16), ref[1]), "V"
    got = cd.cpu().numpy().view(np.uint32)
    if codes:
        wrong = got != ref[2]
        assert not wrong.any(), f"{int(wrong.sum())} of {wrong.size} code words"
    else:
        assert (got == JUNK32).all()
    ctx.close()


@pytest.mark.parametrize("prepared", [False, True])
@pytest.mark.parametrize("T", [1, 2, 5, 16, 17, 63, 64, 65, 130, 257, 1000, 4099])
@pytest.mark.parametrize("Hkv,r,P", [(2, 128, 64), (1, 256, 16), (3, 64, 256), (2, 32, 16), (2, 96, 32)])
def test_rows_and_codes(hata, T, Hkv, r, P, prepared):
    check(hata, *make(T + r, T, Hkv, r, P), P, how=["packed", "heads_first", "fused"][T % 3], prepared=prepared)


@pytest.mark.parametrize("T", [1, 7, 300])
@pytest.mark.parametrize("how", ["packed", "heads_first", "fused"])
def test_without_codes(hata, T, how):
    check(hata, *make(T, T, 3, 128, 16), 16, how=how, codes=False)


@pytest.mark.parametrize("prepared", [False, True])
@pytest.mark.parametrize("T", [9, 70, 700])
@pytest.mark.parametrize("r", [32, 64, 128, 256])
def test_projections_next_to_zero(hata, T, r, prepared):
    """Every projection is zero or a few units of the last place of its products: what a 32-bit sum cannot decide."""
    K, V, W, slots, n_pages = make(T, T, 2, r, 16)
    rng = np.random.default_rng(T)
    # pairs of channels with equal keys and weights that cancel but for the last bit of the fp32 weight
    K[:, :, 1::2] = K[:, :, 0::2]
    W[:, 1::2] = -W[:, 0::2]
    up = rng.integers(-1, 2, W[:, 1::2].shape) * (rng.random(W[:, 1::2].shape) < 0.02)
    W[:, 1::2] = (W[:, 1::2].view(np.int32) + up.astype(np.int32)).view(np.float32)
    p = np.einsum("thd,hdr->thr", to_f64(K), W.astype(np.float64))
    assert (p == 0).any() and (p > 0).any() and (p < 0).any() and np.abs(p).max() < 1e-5
    check(hata, K, V, W, slots, n_pages, 16, prepared=prepared)


@pytest.mark.parametrize("prepared", [False, True])
@pytest.mark.parametrize("T", [6, 200])
def test_values_of_every_size(hata, T, prepared):
    """Keys from the smallest bf16 number to the largest, infinite ones and NaN among them (a NaN projection clears the bit)."""
    K, V, W, slots, n_pages = make(T, T, 2, 128, 16)
    rng = np.random.default_rng(T)
    e = rng.integers(-133, 128, (T, 2, 1)).astype(np.float64)
    K[:] = bf16(np.clip(to_f64(K) * 2.0 ** e, -3.38e38, 3.38e38))
    K[1, 0, 5] = 0x7F80
    K[2, 1, 7], K[2, 1, 9] = 0xFF80, 0x7F80
    K[3, 0, 11] = 0x7FC0
    K[4] = 0
    check(hata, K, V, W, slots, n_pages, 16, prepared=prepared)


def test_weights_of_every_size(hata):
    K, V, W, slots, n_pages = make(1, 150, 2, 128, 16)
    W *= 2.0 ** np.random.default_rng(1).integers(-100, 60, (2, 1, 128))
    W[0, :, 3] = 0
    W[1, 4, 5], W[1, 4, 6] = np.inf, np.nan
    check(hata, K, V, W.astype(np.float32), slots, n_pages, 16)
    check(hata, K, V, W.astype(np.float32), slots, n_pages, 16, prepared=True)


@pytest.mark.parametrize("prepared", [False, True])
@pytest.mark.parametrize("T", [6, 200])
@pytest.mark.parametrize("r", [32, 64, 128, 256])
def test_rows_of_zeros_with_weights_beyond_the_narrow_types(hata, T, r, prepared):
    """Finite weights that bf16 or fp16 hold as infinite project a row of zeros to zero all the same (the bit is set); infinite ones do not."""
    K, V, W, slots, n_pages = make(2, T, 2, r, 16)
    K[::3] = 0
    K[::6, :, 1::2] = 0x8000  # (-0)
    W[0, 7, 3] = 3.4e38
    W[1, 4, 5], W[1, 9, 6] = np.inf, -1e6
    check(hata, K, V, W, slots, n_pages, 16, prepared=prepared)


def test_one_row_for_all_and_another_stream(hata):
    import torch
    K, V, W, slots, n_pages = make(8, 40, 2, 128, 16)
    K[:], V[:] = K[:1], V[:1]
    s = torch.cuda.Stream()
    check(hata, K, V, W, slots, n_pages, 16, stream=s)
    # the same through a stride of zero
    ctx = hata.Context(1, 2, 2, D, 128, 64, 64)
    ref = expect(K, V, W, slots, n_pages, 16)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    pools = [dev(np.full((n_pages, 2, 16, D), JUNK16, np.uint16).view(np.int16)) for _ in range(2)]
    codes = dev(np.full((n_pages, 2, 16, 4), JUNK32, np.int32))
    ctx.hata_write_slots(dev(K[:1].view(np.int16)), dev(V[:1].view(np.int16)), 0, D, dev(slots), 40, pools[0], pools[1], codes, 16,
                         n_pages, dev(W))
    torch.cuda.synchronize()
    assert np.array_equal(pools[0].cpu().numpy().view(np.uint16), ref[0])
    assert np.array_equal(codes.cpu().numpy().view(np.uint32), ref[2])
    ctx.close()


def test_codes_equal_those_of_an_appended_row(hata):
    """The same keys through the decode step's append: the same code words."""
    import torch
    B, Hkv, P = 3, 2, 16
    K, V, W, _, _ = make(4, B, Hkv, 128, P)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    ctx = hata.Context(B, 4, Hkv, D, 128, 64, 16)
    pools = [torch.zeros((B, Hkv, P, D), dtype=torch.int16, device="cuda") for _ in range(2)]
    codes = [torch.zeros((B, Hkv, P, 4), dtype=torch.int32, device="cuda") for _ in range(2)]
    Wd = dev(W)
    ctx.hata_write_slots(dev(K.view(np.int16)), dev(V.view(np.int16)), Hkv * D, D, dev(np.arange(B, dtype=np.int32) * P), B,
                         pools[0], pools[1], codes[0], P, B, Wd)
    one, table = dev(np.ones(B, np.int32)), dev(np.arange(B, dtype=np.int32))
    out = torch.zeros((B, 4, D), dtype=torch.int16, device="cuda")
    q = dev(np.random.default_rng(0).integers(0x3F00, 0x4000, (B, 4, D)).astype(np.int16))
    ctx.hata_decode_step_paged(q, pools[0], pools[1], Wd, codes[1], table, 1, P, B, one, one, B, True, 0.1, out)
    torch.cuda.synchronize()
    assert torch.equal(codes[0], codes[1]) and codes[0].any()
    ctx.close()


def test_refusals(hata):
    import torch
    lib = hata.load_library()
    ctx = hata.Context(1, 2, 2, D, 128, 64, 64)
    t = torch.zeros(65536, dtype=torch.int32, device="cuda")
    p = t.data_ptr()

    def call(h=ctx._h, K=p, V=p, st=256, sh=128, slots=p, n=4, Kp=p, Vp=p, codes=p, P=16, n_pages=2, W=p):
        return lib.hata_write_slots(h, K, V, st, sh, slots, n, Kp, Vp, codes, P, n_pages, W, None)

    for bad in ({"h": None}, {"K": None}, {"V": None}, {"slots": None}, {"n": -1}, {"Kp": None}, {"Vp": None}, {"codes": None},
                {"W": None}, {"st": 100}, {"sh": 4}, {"st": -256}, {"sh": -128}, {"P": 8}, {"P": 24}, {"n_pages": 0},
                {"n_pages": 1 << 27}, {"K": p + 8}, {"Vp": p + 2}, {"codes": p + 4}, {"W": p + 4}, {"slots": p + 2}):
        assert call(**bad) == -1, bad
    assert call(n=0) == 0
    ctx.close()
