"""Operators of a paged key/value cache whose sequences share prompts, as cases that can be timed and compared.

Block tables and slot maps built from request lengths (``plan``), packed rows written through a slot map together
with their key codes (``write``), and dense decode attention on block tables, in which the rows that a group of
sequences shares are read once for all of them (``attend``).  ``own`` is false: the operators in elementary torch
operations, 32 bits wide (64 where a sign next to zero decides); ``own`` is true: the calls of this package.
"""
import math

import numpy as np
import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)


def plan(name=None, **kw):
    """B requests: ``decode`` of them grow by one token, ``prompts`` begin (every other one behind a shared prompt),
    the others end; ``tight``: the free pages do not suffice for the last of them."""
    c = {"kind": "plan", "B": 32, "decode": 32, "prompts": 0, "L": 32768, "prompt": 0, "page_rows": 64, "tight": False}
    c.update(kw)
    return dict(c, name=name) if name else c


def write(name=None, **kw):
    """T packed rows into pages; ``fused``: K and V are columns of one projection's output; ``r`` 0: no key codes."""
    c = {"kind": "write", "T": 64, "Hq": 32, "Hkv": 8, "r": 128, "page_rows": 64, "fused": True, "pad": 0}
    c.update(kw)
    return dict(c, name=name) if name else c


def attend(name=None, **kw):
    """B sequences in ``groups`` groups that share ``shared`` rows, up to ``rest`` rows behind them for each;
    ``alone`` sequences behind the groups' share nothing and have up to ``alone_rows``."""
    c = {"kind": "attend", "B": 1, "Hq": 32, "Hkv": 8, "groups": 0, "shared": 0, "rest": 0, "alone": 0, "alone_rows": 0,
         "ragged": True, "page_rows": 64}
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token for each of 32 users: what a server does before every decode step, launch cost alone
        plan("plan_decode_32"),
        # a scheduler's turn with everything in it: 512 users decode, prompts begin, requests end, small pages
        plan("plan_turn_512", B=704, decode=512, prompts=128, prompt=2048, page_rows=16),
        # the new rows of a decode step of 64 users, out of the fused projection
        write("write_decode_64"),
        # a prompt chunk of unequal prompts for a dense layer, which needs no codes
        write("write_chunk_dense", T=4001, r=0, page_rows=16),
        # packed prompts of a prefill batch
        write("write_prompts", T=20711),
        # a long prompt with the wide code and a KV head for every query head, rows that are padding behind it
        write("write_wide_r256", T=16384, Hkv=32, r=256, page_rows=256, fused=False, pad=100),
        # one user and a short context on one dense layer: the smallest attention
        attend("attend_one_2k", alone=1, alone_rows=2048, ragged=False),
        # continuous batching without anything shared
        attend("attend_ragged_16", B=16, alone=16, alone_rows=32768),
        # a serving batch behind one long system prompt
        attend("attend_prefix_32", B=32, groups=1, shared=32768, rest=1024),
        # three prompts of odd length and users without one, groups of eight heads, small pages
        attend("attend_groups_g8", B=72, Hq=64, groups=3, shared=11003, rest=2000, alone=7, alone_rows=16001, page_rows=16),
        # a long document that some users ask about, groups of five heads
        attend("attend_document_128k", B=12, Hq=40, groups=1, shared=131072, rest=300, page_rows=256),
        # many samples of one prompt: enough query rows a head to keep the matrix cores busy
        attend("attend_samples_256", B=256, Hq=64, groups=1, shared=16384, rest=500),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["plan", "write", "write", "attend", "attend", "attend"])
    P = rng.choice([16, 64, 256])
    if kind == "plan":
        decode, prompts, ends = log_int(rng, 1, 512), log_int(rng, 1, 128), rng.randint(0, 64)
        prompts = prompts if rng.random() < 0.7 else 0
        return plan(B=decode + prompts + ends, decode=decode, prompts=prompts, L=log_int(rng, 1024, 32768),
                    prompt=log_int(rng, 1, 2048) if prompts else 0, page_rows=P, tight=rng.random() < 0.3)
    Hq, Hkv = rng.choice([(32, 8), (32, 8), (64, 8), (40, 8), (32, 32)])
    if kind == "write":
        return write(T=log_int(rng, 1, (1 << 18) // Hkv), Hq=Hq, Hkv=Hkv, r=rng.choice([0, 64, 128, 128, 256]), page_rows=P,
                     fused=rng.random() < 0.6, pad=rng.randint(0, 64))
    # the largest listed cases' rows over all KV heads, and their products with a shared row
    rows, products = 1 << 20, 1 << 28
    alone, groups = log_int(rng, 1, 24), 0
    alone_rows = log_int(rng, 1, rows // Hkv // (2 * alone))
    if rng.random() < 0.3:
        return attend(B=alone, Hq=Hq, Hkv=Hkv, alone=alone, alone_rows=alone_rows, ragged=rng.random() < 0.7, page_rows=P)
    alone = alone if rng.random() < 0.3 else 0
    members = log_int(rng, 2, 256 * 8 // Hkv)
    groups = log_int(rng, 1, min(6, members // 2))
    shared = log_int(rng, 512, min(131072, rows // Hkv // groups, products // (members * Hq)))
    return attend(B=members + alone, Hq=Hq, Hkv=Hkv, groups=groups, shared=shared,
                  rest=log_int(rng, 1, max(1, min(2048, rows // Hkv // (2 * members)))), alone=alone,
                  alone_rows=min(alone_rows, 16384) if alone else 0, ragged=rng.random() < 0.7, page_rows=P)


# ---- shapes that follow from the case alone (work() knows them) ----

def blocks_of(n, P):
    return -(-n // P)


def requests(c):
    """Rows cached and wanted of every sequence, the sequence whose prompt it continues (-1: none), pages it does not own."""
    rng = np.random.default_rng(c["B"] * 1000003 + c["L"] + c["prompt"])
    P = c["page_rows"]
    now, then, source, shared = [], [], [], []
    for i in range(c["B"]):
        n = int(rng.integers(max(1, c["L"] // 8), c["L"] + 1))
        a, b, f = n, n + 1, -1
        if c["decode"] <= i < c["decode"] + c["prompts"]:
            a, b = 0, 1 + int(rng.integers(max(1, c["prompt"] // 2), c["prompt"] + 1))
            if i % 2:  # behind a prompt that a decoding sequence holds
                f = int(rng.integers(c["decode"]))
                a = min(now[f], 64 * P) // P * P
                b += a
        elif i >= c["decode"]:
            b = 0 if i % 3 else n // 2  # ends, or is set back
        now.append(a)
        then.append(b)
        source.append(f)
        shared.append(a // P if f >= 0 else min(2, n // P) if i % 4 == 0 else 0)
    return now, then, source, shared


def group_starts(c):
    members = c["B"] - c["alone"]
    return [members * g // c["groups"] for g in range(c["groups"] + 1)] if c["groups"] else []


def lengths(c):
    rng = np.random.default_rng(c["B"] * 1000003 + c["shared"] + c["alone_rows"])
    out = []
    for b in range(c["B"]):
        base, most = (c["shared"], c["rest"]) if b < c["B"] - c["alone"] else (0, c["alone_rows"])
        out.append(base + (int(rng.integers(1, most + 1)) if c["ragged"] and b % 8 else most))
    return out


def slot_rows(c):
    """Where packed rows lie: sequences of unequal length, one behind the other in whole pages, some rows padding."""
    T, P = c["T"], c["page_rows"]
    rng = np.random.default_rng(T * 31 + P)
    rows, at = [], 0
    while len(rows) < T:
        first, n = int(rng.integers(P)), int(rng.integers(1, max(2, T // 3 + 1)))
        rows += range(at * P + first, at * P + first + n)
        at += blocks_of(first + n, P)
    return np.asarray(rows[:T]), at


# ---- inputs ----

class Source:
    """Seeded tensors on the GPU, with four outlier channels per KV head."""

    def __init__(self, seed, Hkv):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.scale = torch.ones((Hkv, 1, D), dtype=torch.bfloat16, device="cuda")
        channels = np.argsort(np.random.default_rng(seed).random((Hkv, D)), axis=1)[:, :4]
        self.scale.scatter_(2, torch.from_numpy(channels[:, None, :].copy()).cuda(), 8.0)

    def normal(self, *shape):
        return torch.randn(shape, dtype=torch.bfloat16, device="cuda", generator=self.g)

    def rows(self, *shape):
        """[..., Hkv, n, D] bf16"""
        return self.normal(*shape).mul_(self.scale)


def ints(v):
    return torch.from_numpy(np.ascontiguousarray(v, dtype=np.int32)).cuda()


def prepare(case, seed):
    return {"plan": prepare_plan, "write": prepare_write, "attend": prepare_attend}[case["kind"]](case, seed)


def prepare_plan(c, seed):
    B, P = c["B"], c["page_rows"]
    now, then, source, shared = requests(c)
    rng = np.random.default_rng(seed)
    cap = max(max(now), max(then))
    n_new = sum(max(b - a, 0) for a, b in zip(now, then))
    width = blocks_of(cap, P)
    held = [0 if f >= 0 else blocks_of(a, P) for a, f in zip(now, source)]
    wanted = sum(max(0, blocks_of(b, P) - blocks_of(a, P)) for a, b in zip(now, then))
    gone = sum(max(0, blocks_of(a, P) - max(blocks_of(b, P), k)) for a, b, k in zip(now, then, shared) if b < a)
    free = wanted + 64
    if c["tight"]:
        free = max(0, wanted - gone - 1 - wanted // 16)
    n_pages = sum(held) + free
    pages = rng.permutation(n_pages).astype(np.int32)
    table = np.full((B, width), -1, np.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = pages[at:at + n]
        at += n
    stack = np.full(n_pages, -1, np.int32)
    stack[:free] = pages[at:]
    s = {"case": c, "P": P, "width": width, "n_pages": n_pages, "cap": cap, "tokens": n_new + n_new % 7,
         "now": ints(now), "then": ints(then), "source": ints(source), "shared": ints(shared),
         "table": ints(table), "free": ints(stack), "n_free": ints([free]), "n_free_out": ints([0]),
         "seq_len": ints([0] * B), "start": ints([0] * (B + 1))}
    s["slots"], s["positions"] = ints([0] * s["tokens"]), ints([0] * s["tokens"])
    if own:
        from paper_2506_02572_amd import hata
        s["ctx"] = hata.Context(B, 32, 8, D, 128, cap, 64)
    return s


def prepare_write(c, seed):
    T, Hq, Hkv, r, P = c["T"], c["Hq"], c["Hkv"], c["r"], c["page_rows"]
    src = Source(seed, Hkv)
    rng = np.random.default_rng(seed)
    rows, used = slot_rows(c)
    n_pages = used + 3
    pages = rng.permutation(n_pages)
    slots = np.concatenate([pages[rows // P] * P + rows % P, np.full(c["pad"], -1)])
    total = T + c["pad"]
    if c["fused"]:
        x = src.normal(total, Hq + 2 * Hkv, D)
        K, V = x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    else:
        K, V = src.normal(total, Hkv, D), src.normal(total, Hkv, D)
    K.mul_(src.scale[:, 0])
    V.mul_(src.scale[:, 0])
    s = {"case": c, "P": P, "n_pages": n_pages, "K_new": K, "V_new": V, "slots": ints(slots), "W": None, "codes": None,
         "K": torch.zeros((n_pages, Hkv, P, D), dtype=torch.bfloat16, device="cuda"),
         "V": torch.zeros((n_pages, Hkv, P, D), dtype=torch.bfloat16, device="cuda")}
    if r:
        s["W"] = torch.randn((Hkv, D, r), dtype=torch.float32, device="cuda", generator=src.g).mul_(D ** -0.5)
        s["codes"] = torch.zeros((n_pages, Hkv, P, r // 32), dtype=torch.int32, device="cuda")
    if own:
        from paper_2506_02572_amd import hata
        s["ctx"] = hata.Context(1, Hq, Hkv, D, r or 128, 4096, 64)
        if r:
            s["ctx"].hata_prepare_weights(s["W"])  # the weights are fixed once trained
    return s


def prepare_attend(c, seed):
    B, Hq, Hkv, P = c["B"], c["Hq"], c["Hkv"], c["page_rows"]
    src = Source(seed, Hkv)
    lens, starts = lengths(c), group_starts(c)
    full = c["shared"] // P  # pages that a group shares; rows behind them lie in the sequences' own pages
    first = [g for g in range(len(starts) - 1) for _ in range(starts[g], starts[g + 1])] + [-1] * c["alone"]
    own_blocks = [blocks_of(n, P) - (full if g >= 0 else 0) for n, g in zip(lens, first)]
    n_pages = c["groups"] * full + sum(own_blocks)
    pages = np.random.default_rng(seed).permutation(n_pages).astype(np.int32)
    table = np.zeros((B, max(blocks_of(n, P) for n in lens)), np.int32)
    at = c["groups"] * full
    for b, (n, g) in enumerate(zip(own_blocks, first)):
        skip = 0
        if g >= 0:
            table[b, :full] = pages[g * full:(g + 1) * full]
            skip = full
        table[b, skip:skip + n] = pages[at:at + n]
        at += n
    s = {"case": c, "P": P, "n_pages": n_pages, "lens": lens, "table": ints(table), "seq": ints(lens), "width": table.shape[1],
         "K": src.rows(n_pages, Hkv, P, D), "V": src.rows(n_pages, Hkv, P, D),
         "q": src.rows(B, Hkv, Hq // Hkv, D).reshape(B, Hq, D).contiguous(),
         "start": ints(starts) if starts else None, "shared": ints([full * P] * c["groups"]) if starts else None,
         "out": torch.zeros((B, Hq, D), dtype=torch.bfloat16, device="cuda")}
    if own:
        from paper_2506_02572_amd import hata
        s["ctx"] = hata.Context(B, Hq, Hkv, D, 128, max(max(lens), 64), 64)
    return s


# ---- one pass ----

def run(s):
    return (run_own if own else run_plain)(s)


def run_own(s):
    c, ctx = s["case"], s["ctx"]
    if c["kind"] == "plan":
        ctx.hata_plan_pages(s["now"], s["then"], c["B"], s["source"], s["shared"], s["table"], s["width"], s["P"], s["n_pages"],
                            s["free"], s["n_free"], s["n_free_out"], s["seq_len"], s["start"], s["slots"], s["positions"],
                            s["tokens"])
        return plan_outputs(s)
    if c["kind"] == "write":
        K = s["K_new"]
        ctx.hata_write_slots(K, s["V_new"], K.stride(0), K.stride(1), s["slots"], K.shape[0], s["K"], s["V"], s["codes"], s["P"],
                             s["n_pages"], s["W"])
        return write_outputs(s)
    ctx.hata_dense_decode_paged(s["q"], s["K"], s["V"], s["table"], s["width"], s["P"], s["n_pages"], s["seq"], c["B"],
                                s["start"], s["shared"], c["groups"], SCALE, s["out"])
    return s["out"]


def plan_outputs(s):
    return {"table": s["table"], "free": s["free"], "n_free": s["n_free_out"], "seq_len": s["seq_len"], "start": s["start"],
            "slots": s["slots"], "positions": s["positions"]}


def write_outputs(s):
    return {"K": s["K"], "V": s["V"]} if s["codes"] is None else {"K": s["K"], "V": s["V"], "codes": s["codes"]}


def run_plain(s):
    return {"plan": plain_plan, "write": plain_write, "attend": plain_attend}[s["case"]["kind"]](s)


def plain_plan(s):
    P, width, tokens = s["P"], s["width"], s["tokens"]
    now, then, source, shared = s["now"].long(), s["then"].long(), s["source"].long(), s["shared"].long()
    table = s["table"]
    col = torch.arange(width, device=table.device)
    have, want = (now + P - 1) // P, (then + P - 1) // P
    n_new = (then - now).clamp(min=0)
    end = torch.cumsum(n_new, 0)
    src = source.clamp(min=0)
    fork = source >= 0
    ok = (then <= s["cap"]) & (end <= tokens)
    ok &= ~fork | ((now % P == 0) & (source[src] < 0) & (now // P <= torch.minimum(now[src], then[src]) // P))
    need = torch.where(ok, (want - have).clamp(min=0), torch.zeros_like(want))
    keep = torch.maximum(want, shared)
    gone = ok[:, None] & (then < now)[:, None] & (col >= keep[:, None]) & (col < have[:, None])
    rank = torch.cumsum(gone.reshape(-1), 0).reshape(gone.shape) - 1
    n_free = s["n_free"].long()
    avail = n_free + gone.sum()
    upto = torch.cumsum(need, 0)
    granted = ok & ((need == 0) | (upto <= avail))
    left = avail - torch.where(granted & (need > 0), upto, torch.zeros_like(upto)).max()
    # the free stack with the released pages behind it
    pages = s["n_pages"]
    spot = torch.where(gone, n_free + rank, torch.full_like(rank, 2 * pages))
    stack = torch.cat([s["free"], torch.zeros(pages + 1, dtype=torch.int32, device=table.device)])
    stack[spot.reshape(-1)] = table.reshape(-1)
    new = granted[:, None] & (col >= have[:, None]) & (col < want[:, None])
    taken = avail - 1 - ((upto - need)[:, None] + col - have[:, None])
    copied = (granted & fork)[:, None] & (col < (now // P)[:, None])
    s["table"].copy_(torch.where(new, stack[taken.clamp(0, pages - 1)], torch.where(copied, table[src], table)))
    at = torch.arange(pages, device=table.device)
    s["free"].copy_(torch.where((at >= n_free) & (at < left), stack[:pages], s["free"]))
    s["n_free_out"].copy_(left)
    s["seq_len"].copy_(torch.where(granted, then, torch.where(fork, torch.zeros_like(now), now)))
    s["start"][0] = 0
    s["start"][1:] = end
    t = torch.arange(tokens, device=table.device)
    b = torch.searchsorted(end, t, right=True).clamp(max=now.numel() - 1)
    pos = now[b] + t - (end - n_new)[b]
    live = (t < end[-1]) & granted[b]
    slot = s["table"][b, (pos // P).clamp(max=width - 1)].long() * P + pos % P
    s["slots"].copy_(torch.where(live, slot, torch.full_like(slot, -1)))
    s["positions"].copy_(torch.where(live, pos, torch.full_like(pos, -1)))
    return plan_outputs(s)


def plain_write(s):
    P, slots = s["P"], s["slots"].long()
    live = slots >= 0
    page, row = slots[live] // P, slots[live] % P
    K_new = s["K_new"][live]
    s["K"][page, :, row] = K_new
    s["V"][page, :, row] = s["V_new"][live]
    if s["codes"] is not None:  # a sign next to zero decides a bit: 64 bits
        W = s["W"]
        bit = 1 << torch.arange(32, dtype=torch.int64, device=W.device)
        for h in range(W.shape[0]):
            positive = K_new[:, h].double() @ W[h].double() >= 0
            words = (positive.reshape(positive.shape[0], -1, 32) * bit).sum(2)
            s["codes"][page, h, row] = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
    return write_outputs(s)


def plain_attend(s):
    c, P = s["case"], s["P"]
    Hkv, G = c["Hkv"], c["Hq"] // c["Hkv"]
    for b, L in enumerate(s["lens"]):
        pages = s["table"][b, :blocks_of(L, P)].long()
        K = s["K"][pages].transpose(0, 1).reshape(Hkv, -1, D)[:, :L].float()
        V = s["V"][pages].transpose(0, 1).reshape(Hkv, -1, D)[:, :L].float()
        score = torch.matmul(K, s["q"][b].float().view(Hkv, G, D).transpose(1, 2).contiguous()) * SCALE  # [Hkv, L, G]
        weight = torch.exp(score - score.max(1, keepdim=True).values)
        weight = (weight / weight.sum(1, keepdim=True)).transpose(1, 2).contiguous()
        s["out"][b] = torch.matmul(weight, V).view(c["Hq"], D).to(torch.bfloat16)
    return s["out"]


# ---- the definitions in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": exact_plan, "write": exact_write, "attend": exact_attend}[case["kind"]](s)


def exact_plan(s):
    """Requests served one after the other."""
    P = s["P"]
    now, then, source, shared = [s[k].cpu().numpy().tolist() for k in ("now", "then", "source", "shared")]
    table, n_free = s["table"].cpu().numpy().astype(np.int64), int(s["n_free"][0])
    stack = s["free"].cpu().numpy().astype(np.int64)
    before = table.copy()
    B = len(now)

    def served(b):
        f = source[b]
        if then[b] > s["cap"] or sum(max(then[i] - now[i], 0) for i in range(b + 1)) > s["tokens"]:
            return False
        return f < 0 or (now[b] % P == 0 and source[f] < 0 and now[b] // P <= min(now[f], then[f]) // P)

    ok = [served(b) for b in range(B)]
    pile = list(stack[:n_free])
    for b in range(B):
        if ok[b] and then[b] < now[b]:
            pile += [int(before[b, i]) for i in range(max(blocks_of(then[b], P), shared[b]), blocks_of(now[b], P))]
    slots, positions = np.full(s["tokens"], -1, np.int64), np.full(s["tokens"], -1, np.int64)
    start, seq_len, full = [0], [], False
    for b in range(B):
        a, z = blocks_of(now[b], P), blocks_of(then[b], P)
        granted = ok[b]
        if granted and z > a:
            full = full or z - a > len(pile)
            granted = not full
        if granted:
            if source[b] >= 0:
                table[b, :now[b] // P] = before[source[b], :now[b] // P]
            for i in range(a, z):
                table[b, i] = pile.pop()
            n = np.arange(now[b], then[b])
            positions[start[b]:start[b] + n.size] = n
            slots[start[b]:start[b] + n.size] = table[b, n // P] * P + n % P
        seq_len.append(then[b] if granted else 0 if source[b] >= 0 else now[b])
        start.append(start[b] + max(then[b] - now[b], 0))
    if len(pile) > n_free:
        stack[n_free:len(pile)] = pile[n_free:]
    return {"table": table, "free": stack, "n_free": np.asarray([len(pile)]), "seq_len": np.asarray(seq_len),
            "start": np.asarray(start), "slots": slots, "positions": positions}


def exact_write(s):
    P = s["P"]
    slots = s["slots"].cpu().numpy().astype(np.int64)
    at = np.flatnonzero(slots >= 0)
    where = torch.from_numpy(slots[at]).cuda()
    out = {}
    for name in ("K", "V"):
        pool = s[name].transpose(1, 2).reshape(-1, s[name].shape[1], D).double()
        pool[where] = s[name + "_new"][torch.from_numpy(at).cuda()].double()
        out[name] = pool.view(s["n_pages"], P, -1, D).transpose(1, 2)
    if s["codes"] is not None:
        n_pages, Hkv, _, words = s["codes"].shape
        codes = np.zeros((n_pages * P, Hkv, words), np.int32)
        W = s["W"].double()
        for i in range(0, at.size, 4096):
            x = s["K_new"][torch.from_numpy(at[i:i + 4096]).cuda()].double().transpose(0, 1).contiguous()  # [Hkv, n, D]
            bits = (torch.bmm(x, W) >= 0).transpose(0, 1).cpu().numpy()
            codes[slots[at[i:i + 4096]]] = np.packbits(bits, axis=2, bitorder="little").view(np.int32)
        out["codes"] = codes.reshape(n_pages, P, Hkv, words).transpose(0, 2, 1, 3)
    return out


def exact_attend(s):
    c, P = s["case"], s["P"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    flat_K, flat_V = s["K"].view(-1, D), s["V"].view(-1, D)
    out = torch.zeros((c["B"], Hq, D), dtype=torch.float64, device="cuda")
    head = torch.arange(Hkv, device="cuda")
    for b, L in enumerate(s["lens"]):
        n = torch.arange(L, device="cuda")
        page = s["table"][b].long()[n // P]
        rows = (page[None, :] * Hkv + head[:, None]) * P + n % P  # [Hkv, L]
        q = s["q"][b].double().view(Hkv, Hq // Hkv, D)
        logit = torch.bmm(q, flat_K[rows].double().transpose(1, 2).contiguous()) * SCALE
        weight = torch.exp(logit - torch.logsumexp(logit, 2, keepdim=True))
        out[b] = torch.bmm(weight, flat_V[rows].double()).view(Hq, D)
    return out


# ---- what a pass cannot do without ----

def work(case):
    c = case
    if c["kind"] == "plan":
        now, then, source, _ = requests(c)
        P = c["page_rows"]
        tokens = sum(max(b - a, 0) for a, b in zip(now, then))
        moved = sum(abs(blocks_of(b, P) - blocks_of(a, P)) for a, b in zip(now, then))
        copied = sum(a // P for a, f in zip(now, source) if f >= 0)
        return {"bytes": 8 * tokens + 8 * moved + 8 * copied + 24 * c["B"], "flops": 0}
    if c["kind"] == "write":
        rows = c["T"] * c["Hkv"]
        return {"bytes": rows * (8 * D + c["r"] // 8) + 4 * (c["T"] + c["pad"]) + 4 * c["Hkv"] * D * c["r"],
                "flops": 2 * rows * D * c["r"]}
    lens = lengths(c)
    full = c["shared"] // c["page_rows"] * c["page_rows"]
    rows = sum(lens) - full * (c["B"] - c["alone"] - c["groups"])
    return {"bytes": rows * c["Hkv"] * 4 * D + c["B"] * c["Hq"] * 4 * D, "flops": 4 * sum(lens) * c["Hq"] * D}
