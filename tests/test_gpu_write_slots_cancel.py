"""Key codes of packed rows whose projections cancel across a wide range (hata_write_slots): a key has one code, whatever number of
rows it comes with."""
import numpy as np
import pytest

from tests.test_gpu_write_slots import D, bf16, pack, to_f64

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]
HKV, P, T = 2, 16, 300


@pytest.fixture(scope="module")
def hata():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2506_02572_amd import hata
    return hata


def codes_of(hata, K, W, prepared, rows):
    """The code words of K's rows, written `rows` at a time."""
    import torch
    r = W.shape[2]
    ctx = hata.Context(1, HKV, HKV, D, r, 64, 64)
    Kd, Wd = torch.from_numpy(K.view(np.int16)).cuda(), torch.from_numpy(W).cuda()
    n_pages = -(-K.shape[0] // P)
    slots = torch.arange(K.shape[0], dtype=torch.int32, device="cuda")
    pools = [torch.zeros((n_pages, HKV, P, D), dtype=torch.int16, device="cuda") for _ in range(2)]
    codes = torch.zeros((n_pages, HKV, P, r // 32), dtype=torch.int32, device="cuda")
    if prepared:
        ctx.hata_prepare_weights(Wd)
    for t in range(0, K.shape[0], rows):
        x = Kd[t:t + rows]
        ctx.hata_write_slots(x, x, HKV * D, D, slots[t:], x.shape[0], pools[0], pools[1], codes, P, n_pages, Wd)
    torch.cuda.synchronize()
    ctx.close()
    return codes.cpu().numpy().view(np.uint32).transpose(0, 2, 1, 3).reshape(-1, HKV, r // 32)[:K.shape[0]]


def cancelling(big, small, r):
    """A row has +-2^big in two channels and +-2^small in a third, anywhere; a column's weights are equal, so the large ones cancel."""
    rng = np.random.default_rng(big - small)
    K = np.zeros((T, HKV, D), np.float32)
    for t in range(T):
        for h in range(HKV):
            at = rng.choice(D, 3, replace=False)
            if t % 3 == 0:
                at = (8 * int(rng.integers(16)) + rng.choice(8, 3, replace=False))  # neighbours
            K[t, h, at] = 2.0 ** big * np.array([1, -1, 0]) + np.array([0, 0, 2.0 ** small]) * rng.choice([-1, 1])
    W = (rng.choice([-1, 1], (HKV, 1, r)) * (1 + rng.random((HKV, 1, r)))).astype(np.float32) * np.ones((1, D, 1), np.float32)
    return bf16(K), W


@pytest.mark.parametrize("prepared", [False, True])
@pytest.mark.parametrize("r", [32, 64, 128, 256])
@pytest.mark.parametrize("big,small", [(60, 0), (12, -50), (12, -45), (-20, -90)])
def test_one_code_for_any_number_of_rows(hata, r, big, small, prepared):
    K, W = cancelling(big, small, r)
    many = codes_of(hata, K, W, prepared, T)
    for rows in (1, 100):
        few = codes_of(hata, K, W, prepared, rows)
        assert np.array_equal(many, few), f"{int((many != few).sum())} of {many.size} code words by {rows} rows a call"


@pytest.mark.parametrize("prepared", [False, True])
@pytest.mark.parametrize("rows", [T, 100])
def test_bits_beyond_what_64_bits_round(hata, rows, prepared):
    """A sum of 128 products that are exact in 64 bits is off by at most 127 2^-53, below 2^-46, of the sum of their sizes: beyond that
    the bits are those of the exact projections (whole numbers here)."""
    K, W = cancelling(40, 10, 128)
    got = codes_of(hata, K, W, prepared, rows)
    for h in range(HKV):
        x, w = to_f64(K[:, h]), W[h].astype(np.float64)
        # (x and w are multiples of 2^3 and 2^-23: sums of their multiples of 2^-20 in Python's whole numbers)
        xi, wi = (x / 2.0 ** 3).astype(object), (w * 2.0 ** 23).astype(object)
        exact = np.array([[sum(int(a) * int(b) for a, b in zip(row, col) if a) for col in wi.T[:, :]] for row in xi], dtype=object)
        assert min(abs(int(v)) for v in exact.ravel()) * 2.0 ** -20 > 2.0 ** -46 * float((np.abs(x) @ np.abs(w)).max())
        bits = np.array([[v >= 0 for v in row] for row in exact])
        assert np.array_equal(got[:, h], pack(bits))


@pytest.mark.parametrize("prepared", [False, True])
@pytest.mark.parametrize("rows", [T, 100])
def test_infinite_keys_and_columns_of_zeros(hata, rows, prepared):
    """Weights that are all zero: a finite key projects to zero (the bit is set), an infinite one or NaN to NaN (it is not)."""
    rng = np.random.default_rng(3)
    K = bf16(rng.standard_normal((T, HKV, D)))
    W = rng.standard_normal((HKV, D, 128)).astype(np.float32)
    W[:, :, 32:64] = 0  # all columns of a code word
    W[:, :, 70] = -0.0
    K[5, 0, 3], K[6, 1, 100], K[7, :, 64], K[8, :, 1] = 0x7F80, 0xFF80, 0x7FC0, 0x7F7F  # infinite, NaN, the largest
    got = codes_of(hata, K, W, prepared, rows)
    with np.errstate(invalid="ignore"):
        want = np.stack([pack(to_f64(K[:, h]) @ W[h].astype(np.float64) >= 0) for h in range(HKV)], axis=1)
    assert np.array_equal(got, want)
