"""The paged operators together, as a server uses them: every turn pages are planned, the packed new rows written into a dense
layer's cache and a hashed layer's (with key codes), and both layers attended, the dense one with the prompts that sequences share
read once.  Sequences begin, continue a prompt another one holds, grow by a token, are set back and end."""
import math

import numpy as np
import pytest

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]

D, P, CAP, R = 128, 16, 1024, 64
SCALE = 1.0 / math.sqrt(D)


@pytest.fixture(scope="module")
def hata():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2506_02572_amd import hata
    return hata


class Server:
    def __init__(self, hata, B=6, Hq=8, Hkv=2, n_pages=150, max_tokens=512, seed=0):
        import torch
        self.torch, self.B, self.Hq, self.Hkv, self.n_pages, self.max_tokens = torch, B, Hq, Hkv, n_pages, max_tokens
        self.ctx = hata.Context(B, Hq, Hkv, D, R, CAP, 64)
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        z = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype, device="cuda")
        self.table, self.width = z(B, CAP // P), CAP // P
        self.free = torch.randperm(n_pages, generator=self.g, device="cuda").to(torch.int32)
        self.n_free, self.now, self.then = torch.tensor([n_pages], dtype=torch.int32, device="cuda"), z(B), z(B)
        self.start, self.slots, self.positions = z(B + 1), z(max_tokens), z(max_tokens)
        self.pools = [z(n_pages, Hkv, P, D, dtype=torch.bfloat16) for _ in range(4)]  # K, V of the dense layer, of the hashed one
        self.codes = z(n_pages, Hkv, P, R // 32)
        self.W = torch.randn((Hkv, D, R), device="cuda", generator=self.g)
        self.ctx.hata_prepare_weights(self.W)
        self.k = torch.full((B,), 40, dtype=torch.int32, device="cuda")
        self.x = z(max_tokens, 2, Hq + 2 * Hkv, D, dtype=torch.bfloat16)  # both layers' fused projections of the new tokens
        self.q = z(2, B, Hq, D, dtype=torch.bfloat16)
        self.out, self.out32 = z(2, B, Hq, D, dtype=torch.bfloat16), z(2, B, Hq, D, dtype=torch.float32)
        self.rows = [[] for _ in range(B)]  # host's view: per sequence its (K, V) rows of both layers

    def new_values(self):
        self.x.normal_(generator=self.g)
        self.q.normal_(generator=self.g)

    def turn(self, fork=None, shared=None, groups=None):
        t, c = self.torch, self.ctx
        c.hata_plan_pages(self.now, self.then, self.B, fork, shared, self.table, self.width, P, self.n_pages, self.free, self.n_free,
                          self.n_free, self.now, self.start, self.slots, self.positions, self.max_tokens)
        K, V = self.x[:, :, self.Hq:self.Hq + self.Hkv], self.x[:, :, self.Hq + self.Hkv:]
        for layer, (codes, W) in enumerate(((None, None), (self.codes, self.W))):
            c.hata_write_slots(K[:, layer], V[:, layer], self.x.stride(0), D, self.slots, self.max_tokens, self.pools[2 * layer],
                               self.pools[2 * layer + 1], codes, P, self.n_pages, W)
        paging = (self.table, self.width, P, self.n_pages, self.now)
        start, common, n = groups if groups else (None, None, 0)
        c.hata_dense_decode_paged(self.q[0], self.pools[0], self.pools[1], *paging, self.B, start, common, n, SCALE, self.out[0], self.out32[0])
        c.hata_decode_step_paged(self.q[1], self.pools[2], self.pools[3], self.W, self.codes, self.table, self.width, P, self.n_pages,
                                 self.now, self.k, self.B, False, SCALE, self.out[1], self.out32[1])

    def follow(self, before, then, fork=None):
        """The host's view of the same turn (every request granted)."""
        x = self.x.double().cpu()
        at = 0
        for b, (n, m) in enumerate(zip(before, then)):
            if fork and fork[b] >= 0:
                self.rows[b] = list(self.rows[fork[b]][:n])
            self.rows[b] = self.rows[b][:m]
            for _ in range(max(m - n, 0)):
                self.rows[b].append((x[at, :, self.Hq:self.Hq + self.Hkv], x[at, :, self.Hq + self.Hkv:]))
                at += 1
            assert len(self.rows[b]) == m

    def check(self):
        t, G = self.torch, self.Hq // self.Hkv
        lens = self.now.cpu().tolist()
        assert lens == [len(r) for r in self.rows]
        table, free = self.table.cpu().numpy(), self.free.cpu().numpy()[:int(self.n_free[0])]
        held = {int(table[b, i]) for b, n in enumerate(lens) for i in range(-(-n // P))}
        assert held.isdisjoint(free.tolist()) and len(held) + len(free) == self.n_pages  # no page lost, none in use and free
        idx = self.ctx.hata_step_buffers()[2].cpu().numpy()
        codes, W = self.codes.cpu().numpy().view(np.uint32), self.W.double().cpu().numpy()
        for b, n in enumerate(lens):
            if n == 0:
                assert not self.out32[:, b].any()
                continue
            for layer in range(2):
                K = t.stack([r[0][layer] for r in self.rows[b]]).transpose(0, 1)  # [Hkv, n, D]
                V = t.stack([r[1][layer] for r in self.rows[b]]).transpose(0, 1)
                q = self.q[layer, b].double().cpu().view(self.Hkv, G, D)
                if layer == 1:  # over the rows that the step selected, whose codes lie in the pages
                    bits = np.einsum("hnd,hdr->hnr", K.numpy(), W) >= 0
                    page, row = table[b, np.arange(n) // P], np.arange(n) % P
                    for h in range(self.Hkv):
                        assert np.array_equal(codes[page, h, row], np.packbits(bits[h], axis=1, bitorder="little").view(np.uint32))
                        qbits = q[h].numpy() @ W[h] >= 0
                        score = (qbits[:, None] ^ bits[h][None]).sum((0, 2))
                        best = np.sort(np.lexsort((np.arange(n), score))[:40])
                        assert np.array_equal(idx[b, h, :best.size], best)
                        p = t.softmax(q[h] @ K[h, best].T * SCALE, 1)
                        assert (self.out32[1, b, h * G:(h + 1) * G].double().cpu() - p @ V[h, best]).abs().max() < 1e-3
                else:
                    p = t.softmax(q @ K.transpose(1, 2) * SCALE, 2)
                    want, size = (p @ V).view(self.Hq, D), (p @ V.abs()).view(self.Hq, D)
                    err = (self.out32[0, b].double().cpu() - want).abs()
                    assert bool((err <= 2.0 ** -8 * (size + want.abs()) + 2.0 ** -11 * size).all())  # (shared rows' weights are bf16)
        assert t.equal(self.out, self.out32.to(t.bfloat16))

    def run(self, then, fork=None, shared=None, groups=None):
        i32 = lambda a: None if a is None else self.torch.tensor(a, dtype=self.torch.int32, device="cuda")
        before = self.now.cpu().tolist()
        self.then.copy_(i32(then))
        self.new_values()
        self.turn(i32(fork), i32(shared), groups and (i32(groups[0]), i32(groups[1]), len(groups[1])))
        self.torch.cuda.synchronize()
        self.follow(before, then, fork)
        self.check()


def test_a_server_of_some_turns(hata):
    s = Server(hata)
    s.run([300, 0, 0, 0, 70, 0])                                    # two prompts
    s.run([301, 0, 0, 0, 71, 0])                                    # a token each
    # three sequences continue the first one's prompt: 288 rows in whole pages
    s.now[1:4] = 288
    for b in (1, 2, 3):
        s.rows[b] = s.rows[0][:288]
    own = [0, 18, 18, 18, 0, 0]
    s.run([302, 290, 350, 289, 72, 33], fork=[-1, 0, 0, 0, -1, -1], shared=own, groups=([0, 4], [288]))
    for turn in range(4):
        s.run([len(r) + 1 for r in s.rows], shared=own, groups=([0, 4, 6], [288, 0]))
    n = [len(r) for r in s.rows]
    s.run([n[0] + 1, 288, n[2] + 1, n[3] + 1, n[4] + 1, 0], shared=own, groups=([0, 4], [288]))     # set back, ended
    s.run([n[0] + 2, 289, 0, 300, n[4] + 2, 120], shared=own, groups=([0, 4], [288]))  # one of the group ends: the prompt stays
    s.run([n[0] + 3, 290, 0, 301, 0, 121], shared=own, groups=([0, 4], [288]))
    s.run([0, 0, 0, 0, 0, 0], shared=own)
    s.run([5, 6, 7, 8, 9, 10])
    s.ctx.close()


def test_captured_decode_turns(hata):
    """A turn recorded once -- lengths counted up on the device, planned, written, attended -- and replayed, with the program's own
    work and eager turns between."""
    import torch
    s = Server(hata, seed=3, max_tokens=128)
    s.run([90, 0, 0, 0, 30, 1])
    s.now[1:4] = 80
    for b in (1, 2, 3):
        s.rows[b] = s.rows[0][:80]
    own = [0, 5, 5, 5, 0, 0]
    s.run([91, 83, 81, 84, 31, 2], fork=[-1, 0, 0, 0, -1, -1], shared=own, groups=([0, 4], [80]))
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    shared, groups = i32(own), (i32([0, 4]), i32([80]), 1)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            torch.add(s.now, 1, out=s.then)
            s.turn(None, shared, groups)
    for turn in range(30):
        before = s.now.cpu().tolist()
        s.new_values()
        if turn % 5 == 4:
            torch.add(s.now, 1, out=s.then)
            s.turn(None, shared, groups)
        else:
            torch.cuda.synchronize()
            graph.replay()
        torch.cuda.synchronize()
        s.follow(before, [n + 1 for n in before])
        s.check()
    s.ctx.close()
