"""Host-side behaviour of the operators around drafted tokens that needs no GPU: frequencies, and calls without a context."""
import ctypes
import math

import numpy as np
import pytest

from paper_2506_02572_amd import hata


def test_calls_without_a_context_are_refused():
    lib = hata.load_library()
    p, n = ctypes.c_void_p(4096), ctypes.c_size_t(0)  # (looked at by nobody)
    r = ctypes.byref(hata.hata_rotary(4096, 128, 0, 1.0))
    assert lib.hata_rotate(None, p, 128, 128, 1, p, 1, r, 0, p, 128, 128, None) == -1
    assert lib.hata_rotate_write_slots(None, p, 128, 128, p, p, p, 128, 128, p, p, 1, r, p, p, None, 16, 4, None, None) == -1
    assert lib.hata_tree_scratch_bytes(None, 1, 1, 1, ctypes.byref(n)) == -1
    assert lib.hata_dense_tree_paged(None, p, p, p, p, 4, 16, 4, p, p, 1, p, 1, 1, None, 0, 1.0, p, None, p, 1 << 20, None) == -1
    assert lib.hata_keep_rows(None, p, p, None, p, 4, 16, 4, p, p, 1, p, p, 1, p, None) == -1


@pytest.mark.parametrize("dims", [16, 32, 96, 128])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_frequencies(dims, base):
    """Against the formulas in numpy; pow is good to a few units in the last place of fp64 on either side: 2^-48."""
    pairs = dims // 2
    i = np.arange(pairs)
    f = base ** (-2.0 * i / dims)
    near = lambda got, want: np.all(np.abs(np.asarray(got) - want) <= 2.0 ** -48 * np.abs(want))
    got, m = hata.rotary_frequencies(dims, base)
    assert near(got, f) and m == 1.0
    got, m = hata.rotary_frequencies(dims, base, "linear", 4.0)
    assert near(got, f / 4) and m == 1.0
    got, m = hata.rotary_frequencies(dims, base, "base", 8.0)
    assert near(got, (base * 8.0 ** (dims / (dims - 2))) ** (-2.0 * i / dims)) and m == 1.0
    got, m = hata.rotary_frequencies(dims, base, "bands", 8.0, 1.0, 4.0, 8192.0)
    wave = 2 * math.pi / f
    share = (8192.0 / wave - 1.0) / 3.0
    want = np.where(wave < 8192.0 / 4, f, np.where(wave > 8192.0, f / 8, (1 - share) * f / 8 + share * f))
    assert np.all(np.abs(got - want) <= 2.0 ** -44 * want) and m == 1.0  # (a difference of numbers up to 8192 / 2 pi)
    got, m = hata.rotary_frequencies(dims, base, "ramp", 16.0, 1.0, 32.0, 4096.0)
    pair_of = lambda turns: dims * math.log(4096.0 / (turns * 2 * math.pi)) / (2 * math.log(base))
    lo, hi = max(math.floor(pair_of(32.0)), 0), min(math.ceil(pair_of(1.0)), pairs - 1)
    ramp = np.clip((i - lo) / max(hi - lo, 1e-3), 0, 1)
    assert near(got, f / 16 * ramp + f * (1 - ramp)) and m == np.float32(0.1 * math.log(16.0) + 1)
    assert hata.rotary_frequencies(dims, base, "ramp", 0.5, 1.0, 32.0, 4096.0)[1] == 1.0


def test_frequencies_refused():
    lib = hata.load_library()
    freq, m = (ctypes.c_double * 64)(), ctypes.c_float()

    def call(dims=128, base=1e4, kind=0, factor=2.0, low=1.0, high=4.0, original=100.0, out=freq, mag=ctypes.byref(m)):
        s = hata.hata_rotary_scaling(kind, factor, low, high, original)
        return lib.hata_rotary_frequencies(dims, base, ctypes.byref(s), out, mag)
    assert call() == 0 and lib.hata_rotary_frequencies(16, 1e4, None, freq, ctypes.byref(m)) == 0
    assert call(out=None) == -1 and call(mag=None) == -1
    for dims in (0, -16, 8, 20, 144):
        assert call(dims=dims) == -2
    for bad in (dict(base=1.0), dict(base=0.0), dict(base=float("nan")), dict(base=float("inf")), dict(kind=5), dict(kind=-1),
                dict(kind=1, factor=0.0), dict(kind=1, factor=float("nan")), dict(kind=3, low=0.0), dict(kind=3, high=1.0),
                dict(kind=4, original=0.0), dict(kind=4, high=float("inf"))):
        assert call(**bad) == -1, bad
    assert call(kind=1, low=0.0, original=0.0) == 0  # (not of this kind)
    with pytest.raises(hata.HataError):
        hata.rotary_frequencies(128, 1e4, "other")


@pytest.mark.parametrize("dims,base,original", [(128, 10000.0, 65536.0), (128, 10000.0, 131072.0), (64, 10000.0, 65536.0), (16, 10000.0, 32768.0),
                                                (128, 500000.0, 8192.0), (16, 10.0, 100000.0), (32, 10000.0, 150.0)])
def test_ramps_that_end_behind_the_last_pair(dims, base, original):
    """Where the last pair makes more than `low` turns over the original context, the ramp goes on behind it, up to pair dims - 1, and where
    the first one makes fewer than `high` it begins at pair 0.  Every pair's share of the stretched frequency from the formula that the header
    states: what the pair's number leaves of the distance between the two ends.  (2^-45: differences of logarithms below 2^4, of which 2^-53
    each is lost, over at least one pair; and no share at all, or the whole, is exact.)"""
    factor, low, high = 16.0, 1.0, 32.0
    got = np.asarray(hata.rotary_frequencies(dims, base, "ramp", factor, low, high, original)[0])
    turns_of = lambda i: original / (2 * math.pi) * base ** (-2.0 * i / dims)
    ends = []
    for turns, way in ((high, -1), (low, 1)):
        i = 0
        while turns_of(i) > turns and i < dims - 1:  # the pair that makes so many, rounded up ..
            i += 1
        if way < 0 and turns_of(i) < turns:          # .. or down
            i = max(i - 1, 0)
        ends.append(i)
    first, last = ends
    assert last > dims // 2 - 1 or first == 0 or original == 8192.0  # (what the test is about, and one in which neither acts)
    for i in range(dims // 2):
        stretched = min(max((i - first) / max(last - first, 1e-3), 0.0), 1.0)  # (both ends the last one: all pairs turn more than `high` times)
        f = base ** (-2.0 * i / dims)
        want = f * (1 - stretched) + f / factor * stretched
        assert abs(got[i] - want) <= 2.0 ** -45 * want, (i, got[i] / want)
