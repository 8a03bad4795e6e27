"""Rows that a group of sequences shares are weighted as exactly as the sequences' own (hata_dense_decode_paged): the fp32 output
against attention in 64 bits, point by point and in the 2-norm."""
import pytest

from tests.test_gpu_dense_paged import SCALE, World

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]

# heads, KV heads, sequences: 64 query rows a workgroup, 128 and 256, groups of one head to eight
TILES = [(8, 2, 3), (3, 3, 5), (16, 2, 8), (8, 2, 20), (5, 1, 40), (2, 2, 100), (8, 2, 130), (16, 2, 70), (1, 1, 460)]


@pytest.fixture(scope="module")
def hata():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2506_02572_amd import hata
    return hata


def errors(w, groups=True):
    import torch
    out, out32 = w.run(groups)
    torch.cuda.synchronize()
    want, size = w.exact()
    assert torch.equal(out.view(torch.bfloat16), out32.to(torch.bfloat16))
    return (out32.double() - want).abs(), want, size


def largest_terms(w):
    """The largest |scale| sum |q k| of the batch."""
    G, most = w.Hq // w.Hkv, 0.0
    for b, n in enumerate(w.lens):
        if n:
            K = w.rows(w.K, b).abs()
            for h in range(w.Hkv):
                most = max(most, float((w.q[b, h * G:(h + 1) * G].double().abs() @ K[:, h].T).max()))
    return most * abs(w.scale)


def world(Hq, Hkv, members, shared, seed):
    lens = [shared + (7 * i) % 50 for i in range(members)]
    return World(lens, [(members, shared)], Hq=Hq, Hkv=Hkv, P=16, seed=seed, outliers=False)


# A weight p (1 + d) moves o = sum p v / sum p by at most |d| (sum p |v| / sum p + |o|), called |d| (S + |o|) here.  |d| is at most the sum of
#   2^-15   two bf16 terms of eight bits each, the first cut off, the second rounded or cut off,
#   2^-18   the exponential's argument, below 128: half a step of 2^-17, times ln 2; the exponential itself, 2^-22,
#   2^-19 A the logit, an fp32 sum of exact products: 32 roundings at most of 2^-24 of A = |scale| sum |q k|,
# and the fp32 sums of products, two instructions for 16 rows and some 64 steps to join them, are off by a step of 2^-23 of S each.
def bound(w, want, size, terms=2.0 ** -15 + 2.0 ** -18):
    steps = max(w.lens) // 8 + 64
    return (terms + 2.0 ** -19 * largest_terms(w)) * (size + want.abs()) + steps * 2.0 ** -23 * size


@pytest.mark.parametrize("scale", [SCALE, 0.5, -0.25])
@pytest.mark.parametrize("shared", [64, 704, 2112])
@pytest.mark.parametrize("Hq,Hkv,members", TILES)
def test_fp32_output(hata, Hq, Hkv, members, shared, scale):
    """Some logits far apart (0.5: a few rows decide) and many close together.  In the 2-norm the roundings above, of independent rows,
    stay below 2^-12 together: 2^-15, 2^-18, and 2^-19 A with A below 2^6 (a quarter of it, as roundings go, 2^-15).  Weights of one bf16 term,
    2^-8 at most and 2^-9.3 in the mean, are beyond that."""
    w = world(Hq, Hkv, members, shared, seed=shared + members)
    w.scale = scale
    err, want, size = errors(w)
    most = bound(w, want, size)
    assert bool((err <= most).all()), f"off by {float(err.max()):.3e}, {float((err / most).max()):.2f} of the bound"
    rel = float(err.norm() / want.norm())
    assert rel <= 2.0 ** -12, f"2-norm {rel:.3e}"


@pytest.mark.parametrize("shared", [64, 128, 640, 1088, 2048, 2112])
@pytest.mark.parametrize("Hq,Hkv,members", TILES)
def test_equal_weights_count_every_row_once(hata, Hq, Hkv, members, shared):
    """Scale 0: every weight is the same power of two, so nothing is rounded but the sums.  One row left out or taken twice moves an
    output by |v - o| / L, of 128 channels some above 2^-12 for L <= 2162, where the bound is 2^-15 at most."""
    w = world(Hq, Hkv, members, shared, seed=shared)
    w.scale = 0.0
    err, want, size = errors(w)
    most = bound(w, want, size, terms=0.0)
    assert bool((err <= most).all()), f"off by {float(err.max()):.3e}, {float((err / most).max()):.2f} of the bound"


@pytest.mark.parametrize("Hq,Hkv,members", TILES)
def test_as_exact_as_without_groups(hata, Hq, Hkv, members):
    """Naming the group changes how often rows are read: both answers within the same bound of the exact one."""
    w = world(Hq, Hkv, members, 1024, seed=members)
    w.scale = 0.3
    for groups in (True, False):
        err, want, size = errors(w, groups)
        assert bool((err <= bound(w, want, size)).all()), groups
