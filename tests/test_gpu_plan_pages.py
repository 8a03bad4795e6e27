"""Block tables and slot maps from request lengths (hata_plan_pages) against requests served one after the other."""
import ctypes

import numpy as np
import pytest

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]

CAP, JUNK = 4096, -77


@pytest.fixture(scope="module")
def hata():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2506_02572_amd import hata
    return hata


def served(now, then, fork, shared, table, P, stack, n_free, max_tokens, cap):
    """The definition: requests in order; what is released is free before the first page is taken."""
    B, before = len(now), table.copy()
    table, stack = table.copy(), stack.copy()
    n_new = [max(max(t, 0) - max(n, 0), 0) for n, t in zip(now, then)]
    start = np.concatenate([[0], np.cumsum(n_new)])
    blocks = lambda n: -(-n // P)
    valid = []
    for b in range(B):
        ok = 0 <= now[b] <= cap and 0 <= then[b] <= cap and (n_new[b] == 0 or start[b + 1] <= max_tokens)
        f = fork[b]
        if f >= 0:
            ok = ok and f < B and f != b and fork[f] < 0 and now[b] % P == 0 and then[b] >= now[b]
            ok = ok and now[b] // P <= min(now[f], then[f], cap) // P
        valid.append(ok)
    pile = list(stack[:n_free])
    for b in range(B):
        if valid[b] and then[b] < now[b]:
            pile += list(before[b, max(blocks(then[b]), shared[b]):blocks(now[b])])
    slots, positions = np.full(max_tokens, -1), np.full(max_tokens, -1)
    seq, out_of_pages = [], False
    for b in range(B):
        granted = valid[b]
        if granted and blocks(then[b]) > blocks(now[b]):
            out_of_pages = out_of_pages or blocks(then[b]) - blocks(now[b]) > len(pile)
            granted = not out_of_pages
        if granted:
            if fork[b] >= 0:
                table[b, :now[b] // P] = before[fork[b], :now[b] // P]
            for i in range(blocks(now[b]), blocks(then[b])):
                table[b, i] = pile.pop()
            n = np.arange(now[b], then[b])
            positions[start[b]:start[b] + n.size] = n
            slots[start[b]:start[b] + n.size] = table[b, n // P] * P + n % P
        seq.append(then[b] if granted else 0 if fork[b] >= 0 else min(max(now[b], 0), cap))
    if len(pile) > n_free:
        stack[n_free:len(pile)] = pile[n_free:]
    return {"table": table, "free": stack, "n_free": [len(pile)], "seq": seq, "start": np.minimum(start, max_tokens),
            "slots": slots, "positions": positions}


def world(rng, now, P, width, spare):
    """Pages of the cached rows at random, `spare` free ones, junk in every other entry."""
    held = [-(-max(n, 0) // P) if n <= CAP else 0 for n in now]
    n_pages = sum(held) + spare
    pages = rng.permutation(n_pages)
    table, at = np.full((len(now), width), JUNK), 0
    for b, n in enumerate(held):
        table[b, :n] = pages[at:at + n]
        at += n
    stack = np.full(n_pages, JUNK)
    stack[:spare] = pages[at:]
    return table, stack, n_pages


def check(hata, now, then, fork=None, shared=None, P=16, spare=64, max_tokens=None, seed=0, alias=False, stream=None, repeat=2):
    import torch
    rng = np.random.default_rng(seed)
    B, width = len(now), CAP // P
    table, stack, n_pages = world(rng, now, P, width, spare)
    f = [-1] * B if fork is None else fork
    k = [0] * B if shared is None else shared
    tokens = sum(max(max(b, 0) - max(a, 0), 0) for a, b in zip(now, then))
    max_tokens = tokens if max_tokens is None else max_tokens
    ref = served(now, then, f, k, table, P, stack, spare, max_tokens, CAP)
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    ctx = hata.Context(B, 1, 1, 128, 32, CAP, 64)
    for _ in range(repeat):
        d = {"table": put(table), "free": put(stack), "now": put(now), "then": put(then), "n": put([spare])}
        seq = d["now"] if alias else put([JUNK] * B)
        n_out = d["n"] if alias else put([JUNK])
        start, slots, positions = put([JUNK] * (B + 1)), put([JUNK] * max_tokens), put([JUNK] * max_tokens)
        torch.cuda.synchronize()
        ctx.hata_plan_pages(d["now"], d["then"], B, None if fork is None else put(f), None if shared is None else put(k),
                            d["table"], width, P, n_pages, d["free"], d["n"], n_out, seq, start,
                            slots if max_tokens else None, positions if max_tokens else None, max_tokens, stream=stream)
        torch.cuda.synchronize()
        got = {"table": d["table"], "free": d["free"], "n_free": n_out, "seq": seq, "start": start, "slots": slots,
               "positions": positions}
        for name, want in ref.items():
            assert np.array_equal(got[name].cpu().numpy(), np.asarray(want)), name
    ctx.close()
    return ref


@pytest.mark.parametrize("P", [16, 64, 256])
def test_one_token_each(hata, P):
    now = [0, 1, P - 1, P, P + 1, 5 * P - 1, 5 * P, CAP - 1]
    check(hata, now, [n + 1 for n in now], P=P)


def test_single_sequence_from_nothing_to_full(hata):
    check(hata, [0], [CAP], spare=CAP // 16)
    check(hata, [0], [0])
    check(hata, [CAP], [0])
    check(hata, [CAP], [CAP])


def test_released_pages_are_taken_in_the_same_call(hata):
    # 3 free pages, 7 released, 9 wanted: all released ones are among them; then fewer wanted than released
    ref = check(hata, [112, 0, 5], [0, 130, 6], spare=3)
    assert ref["n_free"] == [1]
    ref = check(hata, [112, 0, 5], [40, 30, 6], spare=3)
    assert ref["n_free"] == [5]


def test_shared_blocks_stay(hata):
    check(hata, [100, 100, 100, 100], [0, 20, 0, 101], shared=[3, 3, 100, 3])


def test_forks(hata):
    now = [100, 96, 96, 0, 64, 48, 96]
    fork = [-1, 0, 0, 0, 0, -1, 5]
    # whole pages of sequence 0, twice, none, fewer; more of sequence 5 than it has: refused
    check(hata, now, [101, 97, 96, 40, 90, 48, 100], fork=fork, shared=[0, 6, 6, 0, 4, 0, 6])
    # refused: not whole pages, of itself, of nobody, of a fork, of a sequence that shrinks below, shrinking itself
    ref = check(hata, [100, 17, 16, 16, 16, 64, 32, 32], [101, 20, 20, 20, 20, 16, 40, 16],
                fork=[-1, 0, 2, 8, 1, -1, 5, 0])
    assert ref["seq"][1:5] == [0, 0, 0, 0] and ref["seq"][6:] == [0, 0]


def test_out_of_pages(hata):
    # the third request fails, the fourth (smaller) after it too, one that needs no page does not
    ref = check(hata, [0, 0, 0, 0, 5, 16], [32, 16, 48, 16, 9, 17], spare=4)
    assert ref["seq"] == [32, 16, 0, 0, 9, 16] and ref["n_free"] == [1]
    check(hata, [0, 5], [16, 6], spare=0)


def test_lengths_out_of_range(hata):
    ref = check(hata, [-3, 5, CAP + 1, 7, -1, 10], [4, -2, 9, CAP + 1, -1, 11])
    assert ref["seq"] == [0, 5, CAP, 7, 0, 11]


def test_packed_rows_that_do_not_fit(hata):
    ref = check(hata, [0, 0, 0, 3], [10, 10, 10, 3], max_tokens=25)
    assert ref["seq"] == [10, 10, 0, 3]
    check(hata, [0, 0], [10, 10], max_tokens=100)
    ref = check(hata, [4, 9], [5, 0], max_tokens=0)
    assert ref["seq"] == [4, 0]


@pytest.mark.parametrize("B,seed", [(1, 0), (2, 1), (63, 2), (256, 3), (257, 4), (700, 5), (3001, 6)])
@pytest.mark.parametrize("alias", [False, True])
def test_random_turns(hata, B, seed, alias):
    rng = np.random.default_rng(seed)
    P = int(rng.choice([16, 32, 128]))
    now, then, fork, shared = [], [], [], []
    for b in range(B):
        n, kind, f = int(rng.integers(0, CAP // 4)), int(rng.integers(6)), -1
        t = n + 1
        if kind == 0:
            n, t = 0, int(rng.integers(1, 300))
        elif kind == 1:
            t = int(rng.integers(0, n + 1))
        elif kind == 2 and b:
            f = int(rng.integers(b))
            n = min(n, now[f]) // P * P
            t = n + int(rng.integers(0, 50))
        elif kind == 3 and rng.random() < 0.3:
            t = int(rng.choice([-1, CAP + 1, n]))
        now.append(n); then.append(t); fork.append(f); shared.append(int(rng.integers(0, 3)) if rng.random() < 0.5 else 0)
    tokens = sum(max(max(t, 0) - n, 0) for n, t in zip(now, then))
    want = sum(max(0, -(-max(t, 0) // P) - -(-n // P)) for n, t in zip(now, then))
    # (a source may be given as the one of two: every row that is written is written once)
    check(hata, now, then, fork, shared, P, spare=int(want * rng.choice([0.0, 0.3, 1.0])) + 1, max_tokens=max(tokens - int(rng.integers(-9, 9)), 0),
          seed=seed, alias=alias)


def test_captured_turns_follow_their_inputs(hata):
    """Recorded once, replayed with other lengths: tables, lengths and the free list go on from turn to turn in place."""
    import torch
    P, B, width, n_pages, max_tokens = 16, 5, CAP // 16, 400, 64
    rng = np.random.default_rng(3)
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    table, stack = np.full((B, width), JUNK), rng.permutation(n_pages)
    now, n_free = [0] * B, n_pages
    ctx = hata.Context(B, 1, 1, 128, 32, CAP, 64)
    d_table, d_free, d_n, d_now, d_then = put(table), put(stack), put([n_free]), put(now), put([0] * B)
    start, slots, positions = put([0] * (B + 1)), put([0] * max_tokens), put([0] * max_tokens)
    args = (d_now, d_then, B, None, None, d_table, width, P, n_pages, d_free, d_n, d_n, d_now, start, slots, positions, max_tokens)
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            ctx.hata_plan_pages(*args)
    for turn in range(12):
        then = [max(0, n + int(rng.integers(-20, 13))) for n in now]
        ref = served(now, then, [-1] * B, [0] * B, table, P, stack, n_free, max_tokens, CAP)
        d_then.copy_(put(then))
        torch.cuda.synchronize()
        if turn % 3 == 2:
            ctx.hata_plan_pages(*args)
        else:
            graph.replay()
        torch.cuda.synchronize()
        for name, t in (("table", d_table), ("free", d_free), ("n_free", d_n), ("seq", d_now), ("start", start),
                        ("slots", slots), ("positions", positions)):
            assert np.array_equal(t.cpu().numpy(), np.asarray(ref[name])), (turn, name)
        table, stack, n_free, now = ref["table"], ref["free"], ref["n_free"][0], ref["seq"]
        held = [table[b, i] for b in range(B) for i in range(-(-now[b] // P))] + list(stack[:n_free])
        assert sorted(held) == list(range(n_pages))  # no page lost, none in two places
    ctx.close()


def test_what_may_be_left_out_and_what_may_be_the_same(hata):
    """No starts and positions; lengths returned where the wanted ones were; a context for more sequences and fewer rows than the
    table has room for (1000 rows, no whole number of pages)."""
    import torch
    P, width, n_pages, spare = 16, CAP // 16, 300, 90
    now, then = [17, 1000, 0, 40, 990, 3], [18, 1001, 300, 0, 1000, 20]
    rng = np.random.default_rng(1)
    table, stack, n_pages = world(rng, now, P, width, spare)
    ref = served(now, then, [-1] * 6, [0] * 6, table, P, stack, spare, 500, 1000)
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    ctx = hata.Context(40, 1, 1, 128, 32, 1000, 64)
    d = {"table": put(table), "free": put(stack), "seq": put(then), "n_free": put([spare])}
    slots = put([JUNK] * 500)
    ctx.hata_plan_pages(put(now), d["seq"], 6, None, None, d["table"], width, P, n_pages, d["free"], d["n_free"], d["n_free"],
                        d["seq"], None, slots, None, 500)
    torch.cuda.synchronize()
    for name in d:
        assert np.array_equal(d[name].cpu().numpy(), np.asarray(ref[name])), name
    assert np.array_equal(slots.cpu().numpy(), ref["slots"]) and ref["seq"][1] == 1000
    ctx.close()


def test_numbers_that_make_no_sense_stay_in_bounds(hata):
    """A free list longer than there are pages, pages that do not exist: clamped, every slot written names a row of the pools."""
    import torch
    P, B, n_pages = 16, 4, 20
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    ctx = hata.Context(B, 1, 1, 128, 32, CAP, 64)
    for n_free in (-5, 0, 20, 1 << 30):
        table, free = put(np.full((B, CAP // P), 2 ** 31 - 1)), put(np.full(n_pages + 500, -9))
        guard = put(np.full(500, 777))
        free[n_pages:] = guard  # (rows behind the list, which is n_pages long)
        n_out, seq, slots = put([0]), put([0] * B), put([0] * 200)
        ctx.hata_plan_pages(put([40, 500, 0, 16]), put([60, 0, 100, 17]), B, None, None, table, CAP // P, P, n_pages, free,
                            put([n_free]), n_out, seq, None, slots, None, 200)
        torch.cuda.synchronize()
        s = slots.cpu().numpy()
        assert ((s >= -1) & (s < n_pages * P)).all() and 0 <= int(n_out[0]) <= n_pages
        assert torch.equal(free[n_pages:], guard)
    ctx.close()


def test_the_largest_batch(hata):
    rng = np.random.default_rng(9)
    now = [int(n) for n in rng.integers(0, 200, 8191)]
    check(hata, now, [max(0, n + int(d)) for n, d in zip(now, rng.integers(-30, 9, 8191))], P=64, spare=500, repeat=1)


def test_on_another_stream(hata):
    import torch
    check(hata, [3, 16, 0], [4, 17, 50], stream=torch.cuda.Stream())


def test_refusals(hata):
    import torch
    lib = hata.load_library()
    ctx = hata.Context(4, 1, 1, 128, 32, CAP, 64)
    t = torch.zeros(4 * 256, dtype=torch.int32, device="cuda")
    p = t.data_ptr()

    def call(h=ctx._h, now=p, then=p, B=4, fork=None, shared=None, table=p, max_blocks=256, P=16, n_pages=100, free=p, n=p, n_out=p,
             seq=p, start=None, slots=p, positions=None, max_tokens=8):
        return lib.hata_plan_pages(h, now, then, B, fork, shared, table, max_blocks, P, n_pages, free, n, n_out, seq, start, slots,
                                   positions, max_tokens, None)

    for bad in ({"h": None}, {"now": None}, {"then": None}, {"B": 0}, {"B": 5}, {"table": None}, {"max_blocks": 0}, {"P": 8},
                {"P": 48}, {"P": 1 << 21}, {"n_pages": 0}, {"n_pages": 1 << 28}, {"max_blocks": 1 << 27}, {"free": None}, {"n": None},
                {"n_out": None}, {"seq": None}, {"slots": None}, {"max_tokens": -1}, {"max_tokens": (1 << 23) + 1}, {"now": p + 2},
                {"positions": p + 1}, {"fork": p + 3}, {"slots": p + 2}):
        assert call(**bad) == -1, bad
    ctx.close()
    many = hata.Context(8192, 1, 1, 128, 32, 64, 64)
    assert call(h=many._h, B=8192) == -2
    many.close()
