"""Operators of speculative decoding on a paged key/value cache, as cases that can be timed and compared.

Rotary positions of packed rows and their gradient (``rotate``), packed rows rotated on the way into pages, with the codes
of the rotated keys (``append``), attention of drafted trees of tokens on block tables (``tree``), and the rows of the
accepted path moved together (``keep``).  ``own`` is false: the operators in elementary torch operations, 32 bits wide
(64 for the angles of far positions, and where a value next to a border decides a rounding or a sign); ``own`` is true:
the calls of this package.
"""
import math

import numpy as np
import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)


def rotate(name=None, **kw):
    """T packed rows of ``heads`` heads inside rows of ``heads + beside``; ``scaling`` of the frequencies; ``back``: the gradient."""
    c = {"kind": "rotate", "T": 1, "heads": 40, "beside": 8, "dims": 128, "interleaved": False, "base": 10000.0, "scaling": "none",
         "far": 32768, "back": False}
    c.update(kw)
    return dict(c, name=name) if name else c


def append(name=None, **kw):
    """T packed rows of a fused projection's output, or of three; ``r`` 0: no key codes; ``pad`` rows that go nowhere."""
    c = {"kind": "append", "T": 64, "Hq": 32, "Hkv": 8, "r": 128, "page_rows": 64, "fused": True, "pad": 0, "dims": 128,
         "interleaved": False, "base": 10000.0, "scaling": "none", "far": 32768}
    c.update(kw)
    return dict(c, name=name) if name else c


def tree(name=None, **kw):
    """B sequences of up to L rows, the last ones of them up to ``draft`` drafted tokens; ``chain``: each sees the ones before."""
    c = {"kind": "tree", "B": 1, "Hq": 32, "Hkv": 8, "L": 2048, "draft": 5, "chain": False, "ragged": True, "page_rows": 64}
    c.update(kw)
    return dict(c, name=name) if name else c


def keep(name=None, **kw):
    """B sequences of up to L rows and ``draft`` drafted ones, of which a path of up to ``path`` is accepted."""
    c = {"kind": "keep", "B": 8, "Hkv": 8, "r": 128, "L": 300, "draft": 16, "path": 6, "page_rows": 16}
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the query and key heads of one user's next token: launch cost alone
        rotate("rotate_token"),
        # gradient of a chunk of prompts with frequencies scaled for long contexts, at far positions
        rotate("rotate_back_far", T=6001, heads=72, beside=0, base=500000.0, scaling="ramp", far=131072, back=True),
        # a decode step of 64 users, one token each
        append("append_decode_64"),
        # prompt chunks for a dense layer, which needs no codes; part of the head rotated, in pairs of neighbours
        append("append_dense", T=3001, Hq=64, r=0, page_rows=16, dims=64, interleaved=True),
        # packed prompts of a prefill batch
        append("append_prompts", T=16411, base=500000.0, scaling="bands", far=131072),
        # long prompts with the wide code and a KV head for every query head, rows that are padding behind them
        append("append_wide_r256", T=8192, Hkv=32, r=256, page_rows=256, fused=False, pad=100),
        # one user, a short chain of drafted tokens, a short context: the smallest attention
        tree("tree_one_2k", chain=True, ragged=False),
        # trees of unequal size over unequal contexts, groups of eight heads, small pages
        tree("tree_ragged_g8", B=16, Hq=64, L=16384, draft=33, page_rows=16),
        # two users with a long document, groups of five heads
        tree("tree_long_g5", B=2, Hq=40, L=131072, draft=48, ragged=False, page_rows=256),
        # a serving batch with wide trees: enough query rows to keep the matrix cores busy
        tree("tree_batch_32", B=32, L=8192, draft=64),
        # some users' accepted tokens
        keep("keep_8"),
        # a large batch with wide trees and the wide code
        keep("keep_256", B=256, r=256, draft=64, path=12, page_rows=64),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "append", "tree", "tree", "tree", "keep"])
    P = rng.choice([16, 64, 256])
    angles = {"dims": rng.choice([32, 64, 128, 128, 128]), "interleaved": rng.random() < 0.4, "base": rng.choice([10000.0, 500000.0]),
              "scaling": rng.choice(["none", "linear", "bands", "ramp"]), "far": log_int(rng, 1024, 131072)}
    if kind == "rotate":
        heads = rng.choice([1, 8, 32, 40, 64, 72])
        return rotate(T=log_int(rng, 1, 400000 // heads), heads=heads, beside=rng.choice([0, 0, 8, 16]), back=rng.random() < 0.4,
                      **angles)
    Hq, Hkv = rng.choice([(32, 8), (32, 8), (64, 8), (40, 8), (32, 32)])
    if kind == "append":
        return append(T=log_int(rng, 1, (1 << 17) // Hkv), Hq=Hq, Hkv=Hkv, r=rng.choice([0, 64, 128, 128, 256]), page_rows=P,
                      fused=rng.random() < 0.6, pad=rng.randint(0, 64), **angles)
    if kind == "keep":
        draft = log_int(rng, 1, 128)
        return keep(B=log_int(rng, 1, 256), Hkv=Hkv if Hkv == 8 else 4, r=rng.choice([0, 64, 128, 256]), L=log_int(rng, 1, 300),
                    draft=draft, path=rng.randint(1, min(draft, 16)), page_rows=P)
    # up to the largest listed cases' rows over all KV heads, and their products
    B, draft = log_int(rng, 1, 32), log_int(rng, 1, 256)
    most = min((1 << 21) // Hkv // B, (1 << 29) // (B * draft * Hq), 131072)
    return tree(B=B, Hq=Hq, Hkv=Hkv, L=log_int(rng, 1, max(1, most)), draft=draft, chain=rng.random() < 0.3,
                ragged=rng.random() < 0.7, page_rows=P)


# ---- shapes that follow from the case alone (work() knows them) ----

def blocks_of(n, P):
    return -(-n // P)


def lengths(c):
    """Committed rows and drafted ones of every sequence; with ``ragged`` one sequence has no committed rows."""
    rng = np.random.default_rng(c["B"] * 1000003 + c["L"] * 31 + c["draft"])
    base, n = [], []
    for b in range(c["B"]):
        full = c["kind"] == "tree" and (not c["ragged"] or b % 8 == 0)
        base.append(c["L"] if full else 0 if b % 16 == 13 else int(rng.integers(1, c["L"] + 1)))
        n.append(c["draft"] if full or c["kind"] == "keep" else int(rng.integers(1, c["draft"] + 1)))
    return base, n


def slot_rows(c):
    """Where packed rows lie: sequences of unequal length, one behind the other in whole pages, and their positions."""
    T, P = c["T"], c["page_rows"]
    rng = np.random.default_rng(T * 31 + P)
    rows, positions, at = [], [], 0
    while len(rows) < T:
        n = int(rng.integers(1, max(2, T // 3 + 1)))
        first = int(rng.integers(max(1, c["far"] - n)))
        rows += range(at * P + first % P, at * P + first % P + n)
        positions += range(first, first + n)
        at += blocks_of(first % P + n, P)
    return np.asarray(rows[:T]), np.asarray(positions[:T]), at


def frequencies(c):
    """Radians a position of every pair, and the factor of the rotated channels."""
    pairs = c["dims"] // 2
    i = np.arange(pairs, dtype=np.float64)
    f = c["base"] ** (-i / pairs)
    if c["scaling"] == "linear":
        return f / 4.0, 1.0
    if c["scaling"] == "bands":  # by the turns that a pair makes over the original context: many are kept, few are stretched
        share = np.clip((8192.0 * f / (2 * math.pi) - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return f * share + f / 8.0 * (1.0 - share), 1.0
    if c["scaling"] == "ramp":  # by the pair's number, between those that make 32 turns and one
        at = lambda turns: pairs * math.log(4096.0 / (turns * 2 * math.pi)) / math.log(c["base"])
        low, high = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), pairs - 1)
        share = 1.0 - np.clip((i - low) / max(high - low, 1e-3), 0.0, 1.0)
        return f * share + f / 16.0 * (1.0 - share), float(np.float32(0.1 * math.log(16.0) + 1.0))
    return f, 1.0


# ---- inputs ----

class Source:
    """Seeded tensors on the GPU, with four outlier channels per head."""

    def __init__(self, seed, heads):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.scale = torch.ones((heads, 1, D), dtype=torch.bfloat16, device="cuda")
        channels = np.argsort(np.random.default_rng(seed).random((heads, D)), axis=1)[:, :4]
        self.scale.scatter_(2, torch.from_numpy(channels[:, None, :].copy()).cuda(), 8.0)

    def normal(self, *shape):
        return torch.randn(shape, dtype=torch.bfloat16, device="cuda", generator=self.g)

    def rows(self, *shape):
        """[..., heads, n, D] bf16"""
        return self.normal(*shape).mul_(self.scale)


def ints(v):
    return torch.from_numpy(np.ascontiguousarray(v, dtype=np.int32)).cuda()


def angles(s, c):
    freq, magnitude = frequencies(c)
    s["freq"], s["magnitude"] = torch.from_numpy(freq).cuda(), magnitude
    if own:
        from paper_2506_02572_amd import hata
        s["rotary"] = hata.Rotary(s["freq"], c["interleaved"], magnitude)
    return s


def context(B, Hq, Hkv, r, rows):
    from paper_2506_02572_amd import hata
    return hata.Context(B, Hq, Hkv, D, r or 128, max(rows, 64), 64)


def prepare(case, seed):
    return {"rotate": prepare_rotate, "append": prepare_append, "tree": prepare_tree, "keep": prepare_keep}[case["kind"]](case, seed)


def prepare_rotate(c, seed):
    T, heads = c["T"], c["heads"]
    src = Source(seed, heads)
    x = src.normal(T, heads + c["beside"], D)[:, :heads]  # (heads of a fused projection's output)
    x.mul_(src.scale[:, 0])
    rng = np.random.default_rng(seed)
    first = rng.integers(0, c["far"], T)
    s = {"case": c, "x": x, "positions": ints(np.sort(first) if T > 64 else first),
         "out": torch.zeros((T, heads, D), dtype=torch.bfloat16, device="cuda")}
    if own:
        s["ctx"] = context(1, 32, 8, 128, 64)
    return angles(s, c)


def prepare_append(c, seed):
    T, Hq, Hkv, r, P = c["T"], c["Hq"], c["Hkv"], c["r"], c["page_rows"]
    src = Source(seed, Hkv)
    rng = np.random.default_rng(seed)
    rows, positions, used = slot_rows(c)
    n_pages = used + 3
    pages = rng.permutation(n_pages)
    nowhere = np.full(c["pad"], -1)
    total = T + c["pad"]
    if c["fused"]:
        x = src.normal(total, Hq + 2 * Hkv, D)
        q, K, V = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    else:
        q, K, V = src.normal(total, Hq, D), src.normal(total, Hkv, D), src.normal(total, Hkv, D)
    K.mul_(src.scale[:, 0])
    V.mul_(src.scale[:, 0])
    s = {"case": c, "P": P, "n_pages": n_pages, "q": q, "K_new": K, "V_new": V, "W": None, "codes": None,
         "slots": ints(np.concatenate([pages[rows // P] * P + rows % P, nowhere])), "positions": ints(np.concatenate([positions, nowhere])),
         "q_out": torch.zeros((total, Hq, D), dtype=torch.bfloat16, device="cuda"),
         "K": torch.zeros((n_pages, Hkv, P, D), dtype=torch.bfloat16, device="cuda"),
         "V": torch.zeros((n_pages, Hkv, P, D), dtype=torch.bfloat16, device="cuda")}
    if r:
        s["W"] = torch.randn((Hkv, D, r), dtype=torch.float32, device="cuda", generator=src.g).mul_(D ** -0.5)
        s["codes"] = torch.zeros((n_pages, Hkv, P, r // 32), dtype=torch.int32, device="cuda")
    if own:
        s["ctx"] = context(1, Hq, Hkv, r, 4096)
        if r:
            s["ctx"].hata_prepare_weights(s["W"])  # the weights are fixed once trained
    return angles(s, c)


def paged(c, lens, seed):
    """A block table over pages in random order, which hold the sequences' rows and a few spare ones."""
    P = c["page_rows"]
    own_blocks = [blocks_of(n, P) for n in lens]
    n_pages = sum(own_blocks) + 3
    pages = np.random.default_rng(seed).permutation(n_pages).astype(np.int32)
    table = np.zeros((c["B"], max(max(own_blocks), 1)), np.int32)
    at = 0
    for b, n in enumerate(own_blocks):
        table[b, :n] = pages[at:at + n]
        at += n
    return table, n_pages


def ancestors(rng, n):
    """Visible drafted tokens of each: itself and its ancestors in a random tree, parents before children."""
    seen = np.zeros((n, n), bool)
    for i in range(n):
        parent = int(rng.integers(max(-1, i - 8), i)) if i else -1
        if parent >= 0:
            seen[i] = seen[parent]
        seen[i, i] = True
    return seen


def prepare_tree(c, seed):
    B, Hq, Hkv, P = c["B"], c["Hq"], c["Hkv"], c["page_rows"]
    src = Source(seed, Hkv)
    base, n = lengths(c)
    lens = [a + k for a, k in zip(base, n)]
    table, n_pages = paged(c, lens, seed)
    words = blocks_of(c["draft"], 32)
    start = np.concatenate([[0], np.cumsum(n)])
    T = int(start[-1])
    rng = np.random.default_rng(seed + 1)
    seen = np.zeros((T, 32 * words), bool)
    for b in range(B):
        seen[start[b]:start[b + 1], :n[b]] = ancestors(rng, n[b])
    s = {"case": c, "P": P, "n_pages": n_pages, "base": base, "n": n, "lens": lens, "T": T, "words": words, "width": table.shape[1],
         "table": ints(table), "committed": ints(base), "seq": ints(lens), "start": ints(start),
         "mask": None if c["chain"] else ints(np.packbits(seen, axis=1, bitorder="little").view(np.int32)),
         "K": src.rows(n_pages, Hkv, P, D), "V": src.rows(n_pages, Hkv, P, D),
         "q": src.rows(T, Hkv, Hq // Hkv, D).reshape(T, Hq, D).contiguous(),
         "out": torch.zeros((T, Hq, D), dtype=torch.bfloat16, device="cuda")}
    if own:
        s["ctx"] = context(B, Hq, Hkv, 128, max(lens))
        s["scratch"] = s["ctx"].hata_tree_scratch(B, T, c["draft"])
    return s


def prepare_keep(c, seed):
    B, Hkv, P, r = c["B"], c["Hkv"], c["page_rows"], c["r"]
    src = Source(seed, Hkv)
    base, n = lengths(c)
    lens = [a + k for a, k in zip(base, n)]
    table, n_pages = paged(c, lens, seed)
    rng = np.random.default_rng(seed + 1)
    path, n_path = np.zeros((B, c["path"]), np.int64), []
    for b in range(B):
        k = int(rng.integers(0, c["path"] + 1))
        path[b, :k] = np.sort(rng.permutation(n[b])[:k])
        n_path.append(min(k, n[b]))
    s = {"case": c, "P": P, "n_pages": n_pages, "width": table.shape[1], "table": ints(table), "committed": ints(base), "seq": ints(lens),
         "path": ints(path), "n_path": ints(n_path), "seq_out": ints([0] * B),
         "K": src.rows(n_pages, Hkv, P, D), "V": src.rows(n_pages, Hkv, P, D), "codes": None}
    if r:
        s["codes"] = torch.randint(-2 ** 31, 2 ** 31, (n_pages, Hkv, P, r // 32), device="cuda", generator=src.g).to(torch.int32)
    if own:
        s["ctx"] = context(B, Hkv, Hkv, r, max(lens))
    return s


# ---- one pass ----

def run(s):
    return (run_own if own else run_plain)(s)


def run_own(s):
    c, ctx = s["case"], s["ctx"]
    if c["kind"] == "rotate":
        x, out = s["x"], s["out"]
        ctx.hata_rotate(x, x.stride(0), x.stride(1), c["heads"], s["positions"], c["T"], s["rotary"], c["back"], out, out.stride(0),
                        out.stride(1))
        return out
    if c["kind"] == "append":
        q, K = s["q"], s["K_new"]
        ctx.hata_rotate_write_slots(q, q.stride(0), q.stride(1), s["q_out"], K, s["V_new"], K.stride(0), K.stride(1), s["positions"],
                                    s["slots"], K.shape[0], s["rotary"], s["K"], s["V"], s["codes"], s["P"], s["n_pages"], s["W"])
        return append_outputs(s)
    if c["kind"] == "keep":
        ctx.hata_keep_rows(s["K"], s["V"], s["codes"], s["table"], s["width"], s["P"], s["n_pages"], s["committed"], s["seq"], c["B"],
                           s["path"], s["n_path"], c["path"], s["seq_out"])
        return keep_outputs(s)
    ctx.hata_dense_tree_paged(s["q"], s["K"], s["V"], s["table"], s["width"], s["P"], s["n_pages"], s["committed"], s["seq"], c["B"],
                              s["start"], s["T"], c["draft"], s["mask"], s["words"], SCALE, s["out"], None, s["scratch"])
    return s["out"]


def append_outputs(s):
    out = {"q": s["q_out"], "K": s["K"], "V": s["V"]}
    return out if s["codes"] is None else dict(out, codes=s["codes"])


def keep_outputs(s):
    out = {"K": s["K"], "V": s["V"], "seq_len": s["seq_out"]}
    return out if s["codes"] is None else dict(out, codes=s["codes"])


def run_plain(s):
    return {"rotate": plain_rotate, "append": plain_append, "tree": plain_tree, "keep": plain_keep}[s["case"]["kind"]](s)


def to_bf16(x):
    """Nearest, ties to even, in one rounding: a value whose nearest fp32 lies half-way between two bf16 is moved off it first."""
    f = x.float()
    bits = f.view(torch.int32)
    error = x.abs() - f.abs().double()
    half = (bits & 0xffff) == 0x8000
    bits = bits + torch.where(half & (error > 0), 1, 0) - torch.where(half & (error < 0), 1, 0)
    return bits.to(torch.int32).view(torch.float32).to(torch.bfloat16)


def rotated(x, positions, freq, magnitude, interleaved, back=False):
    """[T, heads, D] bf16"""
    pairs = freq.numel()
    t = positions.double()[:, None] * freq
    cos, sin = (torch.cos(t) * magnitude)[:, None], (torch.sin(t) * magnitude)[:, None]
    if back:
        sin = -sin
    x64 = x[:, :, :2 * pairs].double()
    a, b = (x64[:, :, 0::2], x64[:, :, 1::2]) if interleaved else (x64[:, :, :pairs], x64[:, :, pairs:])
    first, second = a * cos - b * sin, a * sin + b * cos
    y = torch.stack([first, second], 3).flatten(2) if interleaved else torch.cat([first, second], 2)
    return torch.cat([to_bf16(y), x[:, :, 2 * pairs:]], 2)


def plain_rotate(s):
    c = s["case"]
    s["out"].copy_(rotated(s["x"], s["positions"], s["freq"], s["magnitude"], c["interleaved"], c["back"]))
    return s["out"]


def plain_append(s):
    c, P, slots = s["case"], s["P"], s["slots"].long()
    live = slots >= 0
    page, row = slots[live] // P, slots[live] % P
    s["q_out"].copy_(rotated(s["q"], s["positions"], s["freq"], s["magnitude"], c["interleaved"]))
    K_new = rotated(s["K_new"][live], s["positions"][live], s["freq"], s["magnitude"], c["interleaved"])
    s["K"][page, :, row] = K_new
    s["V"][page, :, row] = s["V_new"][live]
    if s["codes"] is not None:  # a sign next to zero decides a bit: 64 bits
        W = s["W"]
        bit = 1 << torch.arange(32, dtype=torch.int64, device=W.device)
        for h in range(W.shape[0]):
            positive = K_new[:, h].double() @ W[h].double() >= 0
            words = (positive.reshape(positive.shape[0], -1, 32) * bit).sum(2)
            s["codes"][page, h, row] = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
    return append_outputs(s)


def visible(s, b):
    """[n, n] of sequence b's drafted tokens"""
    n, at = s["n"][b], sum(s["n"][:b])
    j = torch.arange(n, device=s["q"].device)
    if s["mask"] is None:
        return j[None, :] <= j[:, None]
    return (s["mask"][at:at + n][:, j // 32] >> (j % 32)) & 1 == 1


def plain_tree(s):
    c, P = s["case"], s["P"]
    Hkv, G = c["Hkv"], c["Hq"] // c["Hkv"]
    at = 0
    for b, (L, n) in enumerate(zip(s["lens"], s["n"])):
        pages = s["table"][b, :blocks_of(L, P)].long()
        K = s["K"][pages].transpose(0, 1).reshape(Hkv, -1, D)[:, :L].float()
        V = s["V"][pages].transpose(0, 1).reshape(Hkv, -1, D)[:, :L].float()
        q = s["q"][at:at + n].float().view(n, Hkv, G, D).permute(1, 3, 0, 2).reshape(Hkv, D, n * G)
        score = torch.matmul(K, q) * SCALE  # [Hkv, L, n G]
        hidden = ~visible(s, b).t()[:, :, None].expand(n, n, G).reshape(n, n * G)
        score[:, L - n:].masked_fill_(hidden, float("-inf"))
        top = score.max(1, keepdim=True).values
        weight = torch.exp(score - torch.where(top == float("-inf"), torch.zeros_like(top), top))
        total = weight.sum(1, keepdim=True)
        weight = (weight / torch.where(total == 0, torch.ones_like(total), total)).transpose(1, 2).contiguous()
        o = torch.matmul(weight, V).view(Hkv, n, G, D).transpose(0, 1)
        s["out"][at:at + n] = o.reshape(n, c["Hq"], D).to(torch.bfloat16)
        at += n
    return s["out"]


def plain_keep(s):
    c, P = s["case"], s["P"]
    base = s["committed"].long()
    i = torch.arange(c["path"], device=base.device)
    b, i = torch.nonzero(i[None, :] < s["n_path"][:, None], as_tuple=True)
    source, to = base[b] + s["path"].long()[b, i], base[b] + i
    table = s["table"].long()
    for pool in (s["K"], s["V"], s["codes"]):
        if pool is not None:
            pool[table[b, to // P], :, to % P] = pool[table[b, source // P], :, source % P]
    s["seq_out"].copy_(base + s["n_path"])
    return keep_outputs(s)


# ---- the definitions in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": exact_rotate, "append": exact_append, "tree": exact_tree, "keep": exact_keep}[case["kind"]](s)


def turned(x, positions, s, back=False):
    """Pairs as complex numbers, times those of their angles."""
    c, freq = s["case"], s["freq"]
    dims = 2 * freq.numel()
    angle = positions.double()[:, None, None] * freq
    turn = torch.polar(torch.full_like(angle, s["magnitude"]), -angle if back else angle)
    y = x.double()
    head = y[:, :, :dims].unflatten(2, (-1, 2)) if c["interleaved"] else y[:, :, :dims].unflatten(2, (2, -1)).transpose(2, 3)
    z = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn)
    y[:, :, :dims] = (z if c["interleaved"] else z.transpose(2, 3)).flatten(2)
    return y


def exact_rotate(s):
    return turned(s["x"], s["positions"], s, s["case"]["back"])


def exact_append(s):
    P = s["P"]
    slots = s["slots"].cpu().numpy().astype(np.int64)
    at = torch.from_numpy(np.flatnonzero(slots >= 0)).cuda()
    where = torch.from_numpy(slots[slots >= 0]).cuda()
    keys = turned(s["K_new"][at], s["positions"][at], s)
    out = {"q": turned(s["q"], s["positions"], s)}
    for name, rows in (("K", keys), ("V", s["V_new"][at].double())):
        pool = s[name].transpose(1, 2).reshape(-1, s[name].shape[1], D).double()
        pool[where] = rows
        out[name] = pool.view(s["n_pages"], P, -1, D).transpose(1, 2)
    if s["codes"] is not None:  # of the keys as the cache holds them: eight significant bits
        n_pages, Hkv, _, words = s["codes"].shape
        mantissa, exponent = torch.frexp(keys)
        held = torch.ldexp(torch.round(mantissa * 256.0), exponent - 8).transpose(0, 1).contiguous()
        bits = torch.bmm(held, s["W"].double()) >= 0
        packed = np.packbits(bits.transpose(0, 1).cpu().numpy(), axis=2, bitorder="little").view(np.int32)
        codes = np.zeros((n_pages * P, Hkv, words), np.int32)
        codes[where.cpu().numpy()] = packed
        out["codes"] = codes.reshape(n_pages, P, Hkv, words).transpose(0, 2, 1, 3)
    return out


def exact_tree(s):
    c, P = s["case"], s["P"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    G = Hq // Hkv
    flat_K, flat_V = s["K"].view(-1, D), s["V"].view(-1, D)
    out = torch.zeros((s["T"], Hq, D), dtype=torch.float64, device="cuda")
    head = torch.arange(Hkv, device="cuda")
    start = s["start"].cpu().numpy()
    for b, L in enumerate(s["lens"]):
        t0, t1 = int(start[b]), int(start[b + 1])
        r = torch.arange(L, device="cuda")
        rows = (s["table"][b].long()[r // P][None, :] * Hkv + head[:, None]) * P + r % P  # [Hkv, L]
        seen = torch.ones((t1 - t0, L), dtype=torch.bool, device="cuda")
        if s["mask"] is None:
            seen[:, L - (t1 - t0):] = torch.tril(seen[:, L - (t1 - t0):])
        else:
            bits = np.unpackbits(s["mask"][t0:t1].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :t1 - t0]
            seen[:, L - (t1 - t0):] = torch.from_numpy(bits.astype(bool)).cuda()
        for h in range(Hkv):
            K, V = flat_K[rows[h]].double(), flat_V[rows[h]].double()
            q = s["q"][t0:t1, h * G:(h + 1) * G].double().reshape(-1, D)
            logit = (q @ K.t().contiguous() * SCALE).view(t1 - t0, G, L)
            logit = logit.masked_fill(~seen[:, None, :], -math.inf)
            weight = torch.nan_to_num(torch.exp(logit - torch.logsumexp(logit, 2, keepdim=True)), 0.0)
            out[t0:t1, h * G:(h + 1) * G] = (weight.view(-1, L) @ V).view(t1 - t0, G, D)
    return out


def exact_keep(s):
    """Sequence by sequence, row by row."""
    c, P = s["case"], s["P"]
    table, committed, path, n_path = [s[k].cpu().numpy() for k in ("table", "committed", "path", "n_path")]
    out = {"seq_len": np.zeros(c["B"], np.int64)}
    pools = {k: s[k].view(torch.int16).cpu().numpy() for k in ("K", "V")}
    if s["codes"] is not None:
        pools["codes"] = s["codes"].cpu().numpy()
    before = {k: v.copy() for k, v in pools.items()}
    for b in range(c["B"]):
        base = int(committed[b])
        out["seq_len"][b] = base + int(n_path[b])
        for i in range(int(n_path[b])):
            a, z = base + int(path[b, i]), base + i
            for k in pools:
                pools[k][table[b, z // P], :, z % P] = before[k][table[b, a // P], :, a % P]
    for k, v in pools.items():
        out[k] = v if k == "codes" else (v.astype(np.int32) << 16).view(np.float32)
    return out


# ---- what a pass cannot do without ----

def work(case):
    c = case
    if c["kind"] == "rotate":
        rows = c["T"] * c["heads"]
        return {"bytes": rows * 4 * D + 4 * c["T"], "flops": 3 * rows * c["dims"]}
    if c["kind"] == "append":
        q, rows = (c["T"] + c["pad"]) * c["Hq"], c["T"] * c["Hkv"]
        return {"bytes": q * 4 * D + rows * (8 * D + c["r"] // 8) + 8 * (c["T"] + c["pad"]) + 4 * c["Hkv"] * D * c["r"],
                "flops": 3 * (q + rows) * c["dims"] + 2 * rows * D * c["r"]}
    base, n = lengths(c)
    if c["kind"] == "keep":  # about half of a path's longest
        moved = (c["B"] * c["path"] + 1) // 2
        return {"bytes": moved * c["Hkv"] * (8 * D + c["r"] // 4) + 12 * c["B"], "flops": 0}
    rows, products = sum(base) + sum(n), sum(k * a for a, k in zip(base, n))
    return {"bytes": rows * c["Hkv"] * 4 * D + sum(n) * c["Hq"] * 4 * D, "flops": 4 * products * c["Hq"] * D}
