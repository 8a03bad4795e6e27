"""The paged-serving calls where their counts pass a limit inside: more packed rows than a launch takes, more new tokens than a slot map
can have, shared lengths beyond every sequence."""
import numpy as np
import pytest

from tests.test_gpu_dense_paged import World
from tests.test_gpu_plan_pages import CAP, check as check_plan

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]
D = 128
LAUNCH = 65535 * 16  # packed rows of a launch of hata_write_slots


@pytest.fixture(scope="module")
def hata():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2506_02572_amd import hata
    return hata


@pytest.mark.parametrize("r,codes", [(32, False), (32, True), (96, True)])
@pytest.mark.parametrize("T", [LAUNCH, LAUNCH + 1, LAUNCH + 1000])
def test_more_rows_than_a_launch(hata, T, r, codes):
    """Rows, slots and codes on both sides of the cut; 32 hash bits go to the matrix cores, 96 to the other form."""
    import torch
    P = 64
    n_pages = -(-T // P) + 1
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((T, 2, D), device="cuda", generator=g).to(torch.bfloat16)
    W = torch.randn((1, D, r), device="cuda", generator=g)
    slots = (n_pages * P - 1 - torch.arange(T, device="cuda")).to(torch.int32)  # from the far end
    slots[7], slots[-1] = -1, n_pages * P
    pools = [torch.full((n_pages, 1, P, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    words = torch.full((n_pages, 1, P, r // 32), -3, dtype=torch.int32, device="cuda")
    ctx = hata.Context(1, 1, 1, D, r, 64, 64)
    ctx.hata_write_slots(x[:, 0], x[:, 1], 2 * D, D, slots, T, pools[0], pools[1], words if codes else None, P, n_pages,
                         W if codes else None)
    torch.cuda.synchronize()
    live = torch.ones(T, dtype=torch.bool, device="cuda")
    live[7] = live[-1] = False
    at = slots[live].long()
    for i in (0, 1):
        want = torch.full((n_pages * P, D), 9.0, dtype=torch.bfloat16, device="cuda")
        want[at] = x[live, i]
        assert torch.equal(pools[i].view(-1, D), want)
    want = torch.full((n_pages * P, r // 32), -3, dtype=torch.int32, device="cuda")
    if codes:
        shift = torch.arange(32, device="cuda")
        for rows, to in zip(x[live, 0].split(1 << 17), at.split(1 << 17)):
            bits = (rows.double() @ W[0].double() >= 0).view(-1, r // 32, 32)
            v = (bits.long() << shift).sum(2)
            want[to] = torch.where(v >= 1 << 31, v - (1 << 32), v).to(torch.int32)
    assert torch.equal(words.view(-1, r // 32), want)
    ctx.close()


@pytest.mark.parametrize("first", [3, 900, 7000])
def test_more_new_tokens_than_a_slot_map_can_have(hata, first):
    """8000 sequences that want 32 million rows: token numbers beyond 2^23 count as that, requests up to the limit are granted, and
    requests without new rows wherever they stand."""
    rng = np.random.default_rng(first)
    now, then = [0] * 8000, [CAP] * 8000
    for b in range(first):  # some that fit in front
        then[b] = int(rng.integers(0, 3))
    for b in range(first, 8000, 7):  # some without new rows: as many rows, fewer, none
        now[b] = int(rng.integers(1, 200))
        then[b] = int(rng.integers(0, now[b] + 1))
    check_plan(hata, now, then, spare=2000, max_tokens=first + 50, repeat=1)
    check_plan(hata, now, then, spare=2000, max_tokens=20000, repeat=1)


@pytest.mark.parametrize("beyond", [2 ** 31 - 1, 2 ** 31 - 64, 641])
@pytest.mark.parametrize("members,Hq,Hkv", [(3, 8, 2), (30, 8, 2), (130, 8, 2)])
def test_shared_length_beyond_the_sequences(hata, members, Hq, Hkv, beyond):
    """More rows said to be shared than the shortest sequence has: its rows are (the others go on in pages of their own)."""
    import torch
    w = World([640] + [700 + i for i in range(members - 1)], [(members, 640)], Hq=Hq, Hkv=Hkv, P=16, seed=members)
    ref = w.check()
    want = w.out32.clone()
    w.dev[3].fill_(beyond)
    w.check(ref=ref)
    assert torch.equal(w.out32, want)
