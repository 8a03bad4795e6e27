"""The operators around drafted tokens together, as a server uses them: every turn pages are planned for the drafts, their keys and values
rotated into them (one layer without key codes, one with), both layers attended, the paths that the host accepts moved together, and the
pages behind them handed back by the next plan; hashed attention of one token goes on from the same caches."""
import math

import numpy as np
import pytest

import rotary_reference as R

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]

D, P, CAP, HASH = 128, 16, 1024, 64
SCALE = 1.0 / math.sqrt(D)


@pytest.fixture(scope="module")
def hata():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2506_02572_amd import hata
    return hata


class Server:
    def __init__(self, hata, B=5, Hq=8, Hkv=2, n_pages=120, max_tokens=320, max_draft=40, max_path=6, seed=0):
        import torch
        self.t, self.B, self.Hq, self.Hkv, self.n_pages, self.T = torch, B, Hq, Hkv, n_pages, max_tokens
        self.max_draft, self.max_path, self.words = max_draft, max_path, -(-max_draft // 32)
        self.rng = np.random.default_rng(seed)
        self.ctx = hata.Context(B, Hq, Hkv, D, HASH, CAP, 64)
        self.rotary = hata.Rotary.scaled(D, 10000.0, kind="bands", factor=8.0, low=1.0, high=4.0, original=256.0)
        z = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype, device="cuda")
        self.table, self.width = z(B, CAP // P), CAP // P
        self.free = torch.from_numpy(self.rng.permutation(n_pages).astype(np.int32)).cuda()
        self.n_free = torch.tensor([n_pages], dtype=torch.int32, device="cuda")
        self.now, self.then, self.seq, self.kept = z(B), z(B), z(B), z(B)
        self.start, self.slots, self.flat, self.depth = z(B + 1), z(max_tokens), z(max_tokens), z(max_tokens)
        self.mask, self.path, self.n_path = z(max_tokens, self.words), z(B, max_path), z(B)
        self.pools = [z(n_pages, Hkv, P, D, dtype=torch.bfloat16) for _ in range(4)]  # K, V of the dense layer, of the hashed one
        self.codes = z(n_pages, Hkv, P, HASH // 32)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.g, self.W = g, torch.randn((Hkv, D, HASH), device="cuda", generator=g)
        self.ctx.hata_prepare_weights(self.W)
        self.x = z(max_tokens, 2, Hq + 2 * Hkv, D, dtype=torch.bfloat16)
        self.q, self.out = z(2, max_tokens, Hq, D, dtype=torch.bfloat16), z(2, max_tokens, Hq, D, dtype=torch.bfloat16)
        self.out32 = z(2, max_tokens, Hq, D, dtype=torch.float32)
        self.scratch = self.ctx.hata_tree_scratch(B, max_tokens, max_draft)
        self.one, self.k = z(B, Hq, D, dtype=torch.bfloat16), torch.full((B,), 48, dtype=torch.int32, device="cuda")
        self.rows = [[] for _ in range(B)]  # the host's view: per sequence, row by row, (layer, K or V) [2, 2, Hkv, D] fp64

    def plan(self):
        """Pages for now -> then; behind the kept rows of the last turn."""
        self.ctx.hata_plan_pages(self.now, self.then, self.B, None, None, self.table, self.width, P, self.n_pages, self.free, self.n_free,
                                 self.n_free, self.seq, self.start, self.slots, self.flat, self.T)

    def turn(self):
        """Everything of a turn that is on the device once masks, depths and paths are there."""
        c, Hq, Hkv, x = self.ctx, self.Hq, self.Hkv, self.x
        self.plan()
        for layer, (codes, W) in enumerate(((None, None), (self.codes, self.W))):
            K, V = self.pools[2 * layer], self.pools[2 * layer + 1]
            c.hata_rotate_write_slots(x[:, layer, :Hq], x.stride(0), D, self.q[layer], x[:, layer, Hq:Hq + Hkv], x[:, layer, Hq + Hkv:],
                                      x.stride(0), D, self.depth, self.slots, self.T, self.rotary, K, V, codes, P, self.n_pages, W)
            c.hata_dense_tree_paged(self.q[layer], K, V, self.table, self.width, P, self.n_pages, self.now, self.seq, self.B, self.start,
                                    self.T, self.max_draft, self.mask, self.words, SCALE, self.out[layer], self.out32[layer], self.scratch)
            c.hata_keep_rows(K, V, codes, self.table, self.width, P, self.n_pages, self.now, self.seq, self.B, self.path, self.n_path,
                             self.max_path, self.kept)

    def draft(self, n):
        """New values, a random tree for every sequence with its depths and masks, and a path through it."""
        rng, T = self.rng, self.T
        self.x.normal_(generator=self.g)
        now = self.now.cpu().numpy()
        self.n, self.seen, self.paths = n, [], []
        depth, bits = np.zeros(T, np.int32), rng.random((T, 32 * self.words)) < 0.5
        path, n_path, at = np.full((self.B, self.max_path), -1, np.int32), np.zeros(self.B, np.int32), 0
        for b, k in enumerate(n):
            parent = [int(rng.integers(max(-1, i - 4), i)) if i else -1 for i in range(k)]
            see = np.zeros((k, k), bool)
            for i, p in enumerate(parent):
                if p >= 0:
                    see[i] = see[p]
                see[i, i] = True
            depth[at:at + k] = now[b] + see.sum(1) - 1
            bits[at:at + k, :k] = see
            nodes = np.flatnonzero(see[int(rng.integers(k))])[:self.max_path] if k else np.zeros(0, int)
            nodes = nodes[:int(rng.integers(0, len(nodes) + 1))]
            path[b, :len(nodes)], n_path[b] = nodes, len(nodes)
            self.seen.append(see)
            self.paths.append(nodes)
            at += k
        put = lambda to, a: to.copy_(self.t.from_numpy(a))
        put(self.depth, depth), put(self.path, path), put(self.n_path, n_path)
        put(self.mask, np.packbits(bits, axis=1, bitorder="little").view(np.int32))
        put(self.then, (now + np.asarray(n)).astype(np.int32))
        self.depth_host, self.now_host = depth, now

    def check(self):
        t, G, Hq, Hkv = self.t, self.Hq // self.Hkv, self.Hq, self.Hkv
        host = lambda x: x.cpu().numpy()
        freq, n = host(self.rotary.freq), int(sum(self.n))
        bits = host(self.x.view(t.int16)).view(np.uint16)[:n]
        turned = [R.turn(R.values(bits[:, layer, :Hq + Hkv]), self.depth_host[:n], freq) for layer in range(2)]
        table, at = host(self.table), 0
        codes = host(self.codes).view(np.uint32)
        held = {}
        for layer in range(2):
            q = R.check(host(self.q[layer, :n].view(t.int16)).view(np.uint16), turned[layer][0][:, :Hq], turned[layer][1][:, :Hq], "q")
            held[layer] = (q, R.nearest(turned[layer][0][:, Hq:])[0], R.values(bits[:, layer, Hq + Hkv:]))
        for b, k in enumerate(self.n):
            base = int(self.now_host[b])
            assert base == len(self.rows[b])
            for layer in range(2):
                q, key, value = (a[at:at + k] for a in held[layer])
                old = np.stack([r[layer] for r in self.rows[b]]) if base else np.zeros((0, 2, Hkv, D))
                K, V = np.concatenate([old[:, 0], key]), np.concatenate([old[:, 1], value])  # [rows, Hkv, D]
                see = np.concatenate([np.ones((k, base), bool), self.seen[b]], 1)
                for h in range(Hkv):
                    s = np.einsum("kgd,nd->kgn", q[:, h * G:(h + 1) * G], K[:, h]) * SCALE
                    s = np.where(see[:, None], s, -np.inf)
                    p = np.exp(s - s.max(2, keepdims=True)) if k else s
                    p = p / p.sum(2, keepdims=True)
                    want, size = p @ V[:, h], p @ np.abs(V[:, h])
                    got = host(self.out32[layer, at:at + k, h * G:(h + 1) * G]).astype(np.float64)
                    # weights of two bf16 terms in both sums, 2^-15; scores of sums of absolute products below 2^9: 2^-19 of 2^7 (scaled), in e^x
                    assert np.all(np.abs(got - want) <= (2.0 ** -15 + 4 * 2.0 ** -12) * (size + np.abs(want)))
                # the path's rows
                for i, j in enumerate(self.paths[b]):
                    n_row = base + i
                    page, row = table[b, n_row // P], n_row % P
                    assert np.array_equal(host(self.pools[2 * layer][page, :, row].double()), key[j])
                    assert np.array_equal(host(self.pools[2 * layer + 1][page, :, row].double()), value[j])
                    if layer:
                        assert np.array_equal(codes[page, :, row], R.codes(key[j:j + 1], host(self.W))[0])
            for j in self.paths[b]:
                self.rows[b].append(np.stack([np.stack(a) for a in ((held[0][1][at + j], held[0][2][at + j]), (held[1][1][at + j], held[1][2][at + j]))]))
            at += k
        assert host(self.kept).tolist() == [len(r) for r in self.rows]
        assert t.equal(self.out[:, :n], self.out32[:, :n].to(t.bfloat16))

    def settle(self):
        """The drafts' pages behind the kept rows go back."""
        self.now.copy_(self.seq)
        self.then.copy_(self.kept)
        self.plan()
        self.now.copy_(self.seq)
        self.t.cuda.synchronize()
        held = sum(-(-len(r) // P) for r in self.rows)
        assert held + int(self.n_free[0]) == self.n_pages and self.now.tolist() == [len(r) for r in self.rows]

    def hashed_step(self):
        """A step of one token on the hashed layer, from what is in its cache: rows selected by their codes."""
        t, G = self.t, self.Hq // self.Hkv
        self.one.normal_(generator=self.g)
        out, out32 = t.empty_like(self.one), t.empty(self.one.shape, dtype=t.float32, device="cuda")
        self.ctx.hata_decode_step_paged(self.one, self.pools[2], self.pools[3], self.W, self.codes, self.table, self.width, P, self.n_pages,
                                        self.now, self.k, self.B, False, SCALE, out, out32)
        t.cuda.synchronize()
        idx, W = self.ctx.hata_step_buffers()[2].cpu().numpy(), self.W.double().cpu().numpy()
        for b, rows in enumerate(self.rows):
            K = np.stack([r[1, 0] for r in rows]).transpose(1, 0, 2) if rows else np.zeros((self.Hkv, 0, D))
            for h in range(self.Hkv):
                q = self.one[b, h * G:(h + 1) * G].double().cpu().numpy()
                score = ((q @ W[h] >= 0)[:, None] ^ (K[h] @ W[h] >= 0)[None]).sum((0, 2))
                best = np.sort(np.lexsort((np.arange(len(rows)), score))[:48])
                assert np.array_equal(idx[b, h, :best.size], best)


def test_a_server_that_drafts(hata):
    s = Server(hata)
    for turn, n in enumerate([[39, 0, 17, 33, 1], [5, 40, 1, 16, 2], [12, 30, 0, 40, 7], [31, 1, 40, 2, 32], [40, 40, 40, 40, 40], [1, 1, 1, 1, 1], [0, 0, 9, 0, 0]]):
        s.draft(n)
        s.turn()
        s.t.cuda.synchronize()
        s.check()
        s.settle()
        s.hashed_step()
    s.ctx.close()


def test_captured_turns(hata):
    """A turn recorded once and replayed with other trees, values and paths, with eager turns and the program's own work between."""
    import torch
    s = Server(hata, seed=3)
    s.draft([20, 20, 20, 20, 20])
    s.turn()
    torch.cuda.synchronize()
    s.check(), s.settle()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            s.turn()
    for turn in range(8):
        s.draft(s.rng.integers(0, 41, 5).tolist())
        torch.cuda.synchronize()
        s.turn() if turn % 4 == 3 else graph.replay()
        torch.cuda.synchronize()
        s.check(), s.settle(), s.hashed_step()
    s.ctx.close()


def test_requests_that_are_not_granted(hata):
    """Too few pages: the drafts of the last sequences are not granted, their caches stay as they are, and they keep nothing."""
    import torch
    s = Server(hata, n_pages=10)  # 3 + 2 + 2 + 3, and none for the last
    s.draft([39, 30, 20, 33, 10])
    s.turn()
    torch.cuda.synchronize()
    granted = [b for b in range(5) if s.seq[b] > 0]
    assert granted == [0, 1, 2, 3]
    assert s.kept.tolist() == [len(p) for p in s.paths[:4]] + [0]
    s.n, s.seen[4], s.paths[4] = s.n[:4] + [0], np.zeros((0, 0), bool), []
    s.check(), s.settle(), s.hashed_step()
    s.ctx.close()
