"""GPU: the paged cache's calls together, as a serving loop makes them, against lists of rows in 64 bits: contexts are appended, slots
forked, trees drafted, verified and compacted, pages summarised and read selectively, slots dropped and their pages handed out again."""
import math

import pytest
import torch

import paged_reference as R
from paper_2607_20457_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def attend(q, K, V, g):
    """q [Hq, d], K, V [n, Hkv, d] in 64 bits -> (O, LSE, softmax of |V|)."""
    parts = [R.softmax_attend(q[h * g:(h + 1) * g], K[:, h], V[:, h], 1 / math.sqrt(q.shape[1])) for h in range(K.shape[1])]
    return tuple(torch.cat([p[i] for p in parts]) for i in range(3))


class Loop:
    """A pool on the GPU, and beside it every slot's rows on the CPU: rows[s][layer] = (K [n, Hkv, d], V)."""

    def __init__(self, page, Hq, Hkv, d, layers, n_pages, max_pages, seed):
        self.gen = torch.Generator().manual_seed(seed)
        self.page, self.Hq, self.Hkv, self.d, self.layers = page, Hq, Hkv, d, layers
        shape = (layers, n_pages, page, Hkv, d)
        self.K, self.V = (torch.full(shape, float("nan"), dtype=BF, device=DEV) for _ in range(2))
        self.bounds = torch.full((layers, n_pages, Hkv, 2, d), float("nan"), dtype=BF, device=DEV)
        self.status = binding.new_status(DEV)
        self.table = torch.full((1, max_pages), -1, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.rows = [[(torch.zeros(0, Hkv, d, dtype=BF),) * 2 for _ in range(layers)]]

    def rand(self, *shape):
        return torch.randn(shape, generator=self.gen).to(BF)

    def fork(self, parent, reserve):
        par = None if parent is None else torch.tensor(parent, dtype=torch.int32, device=DEV)
        self.table, self.lens, self.free = binding.pulsar_pages_fork(self.table, self.lens, par, self.K, self.V, reserve, status=self.status)
        if parent is not None:
            empty = [(torch.zeros(0, self.Hkv, self.d, dtype=BF),) * 2] * self.layers
            self.rows = [list(self.rows[p]) if p >= 0 else list(empty) for p in parent]

    def append(self, counts):
        S, T = len(self.rows), max(counts)
        n = torch.tensor(counts, dtype=torch.int32, device=DEV)
        for layer in range(self.layers):
            k, v = self.rand(S, T, self.Hkv, self.d), self.rand(S, T, self.Hkv, self.d)
            binding.pulsar_pages_append(k.to(DEV), v.to(DEV), self.K[layer], self.V[layer], self.table, self.lens, n, status=self.status)
            for s in range(S):
                old = self.rows[s][layer]
                self.rows[s][layer] = (torch.cat([old[0], k[s, :counts[s]]]), torch.cat([old[1], v[s, :counts[s]]]))
        before = self.lens
        self.lens = self.lens + n
        binding.pulsar_pages_summarize(self.K, self.table, before, self.lens, self.bounds, status=self.status)

    def tree_step(self, T):
        """A random tree per slot, verified by chance: a path from a root to some node is accepted."""
        S, g = len(self.rows), self.Hq // self.Hkv
        t = torch.arange(T)
        parent = ((torch.rand(S, T, generator=self.gen) * (t + 1)).floor() - 1).int()
        n_draft = torch.randint(0, T + 1, (S,), generator=self.gen).int()
        new = []
        for layer in range(self.layers):
            q, k, v = self.rand(S, T, self.Hq, self.d), self.rand(S, T, self.Hkv, self.d), self.rand(S, T, self.Hkv, self.d)
            O, LSE = binding.pulsar_tree_attn(q.to(DEV), k.to(DEV), v.to(DEV), self.K[layer], self.V[layer], self.table, self.lens,
                                              parent.to(DEV), n_draft.to(DEV), status=self.status)
            for s in range(S):
                for u in range(int(n_draft[s])):
                    see = R.visible(parent[s], u)
                    Kh = torch.cat([self.rows[s][layer][0], k[s, see]]).double()
                    Vh = torch.cat([self.rows[s][layer][1], v[s, see]]).double()
                    R.check(O[s, u], LSE[s, u], attend(q[s, u].double(), Kh, Vh, g), f"layer {layer} slot {s} node {u}")
            new.append((k, v))
        accept = torch.full((S, T), -1, dtype=torch.int32)
        for s in range(S):
            n = int(n_draft[s])
            if n == 0:
                continue
            path = R.visible(parent[s], int(torch.randint(0, n, (1,), generator=self.gen)))[::-1]
            accept[s, :len(path)] = torch.tensor(path, dtype=torch.int32)
            for layer, (k, v) in enumerate(new):
                old = self.rows[s][layer]
                self.rows[s][layer] = (torch.cat([old[0], k[s, path]]), torch.cat([old[1], v[s, path]]))
        before = self.lens
        self.lens = binding.pulsar_pages_compact(self.K, self.V, self.table, self.lens, accept.to(DEV), status=self.status)
        binding.pulsar_pages_summarize(self.K, self.table, before, self.lens, self.bounds, status=self.status)

    def sparse_step(self, k, sink, window):
        S, g, page = len(self.rows), self.Hq // self.Hkv, self.page
        for layer in range(self.layers):
            q, kn, vn = self.rand(S, 1, self.Hq, self.d), self.rand(S, 1, self.Hkv, self.d), self.rand(S, 1, self.Hkv, self.d)
            O, LSE, sel = binding.pulsar_sparse_attn(q.to(DEV), kn.to(DEV), vn.to(DEV), self.K[layer], self.V[layer], self.bounds[layer],
                                                     self.table, self.lens, k, sink, window, status=self.status)
            for s in range(S):
                Ks, Vs = self.rows[s][layer]
                full = Ks.shape[0] // page
                bounds = R.page_bounds(Ks[:full * page].view(full, page, self.Hkv, self.d))
                for h in range(self.Hkv):
                    at = slice(h * g, (h + 1) * g)
                    want = R.select_pages(q[s, 0, at], bounds[:, h], full, k, sink, window)
                    assert sel[s, 0, h].tolist() == want + [-1] * (k - len(want))
                    rows = [r for b in want for r in range(b * page, (b + 1) * page)] + list(range(full * page, Ks.shape[0]))
                    Kh = torch.cat([Ks[rows, h], kn[s, :, h]]).double()
                    Vh = torch.cat([Vs[rows, h], vn[s, :, h]]).double()
                    R.check(O[s, 0, at], LSE[s, 0, at], R.softmax_attend(q[s, 0, at].double(), Kh, Vh, 1 / math.sqrt(self.d)), f"slot {s}")
                self.rows[s][layer] = (torch.cat([Ks, kn[s]]), torch.cat([Vs, vn[s]]))
        before = self.lens
        self.lens = self.lens + 1
        binding.pulsar_pages_summarize(self.K, self.table, before, self.lens, self.bounds, status=self.status)

    def check(self):
        assert int(self.status.item()) == 0
        table, lens = self.table.cpu().long(), self.lens.tolist()
        assert lens == [r[0][0].shape[0] for r in self.rows]
        for s, n in enumerate(lens):
            r = torch.arange(n)
            for x, i in ((self.K, 0), (self.V, 1)):
                for layer in range(self.layers):
                    got = x[layer].cpu()[table[s][r // self.page], r % self.page]
                    assert torch.equal(got.view(torch.int16), self.rows[s][layer][i].view(torch.int16)), (s, layer, i)


@pytest.mark.parametrize("page,Hq,Hkv,d", [(16, 4, 2, 64), (64, 8, 1, 128), (32, 4, 4, 128)])
def test_a_serving_loop(page, Hq, Hkv, d):
    x = Loop(page, Hq, Hkv, d, layers=2, n_pages=2400 // page, max_pages=480 // page, seed=page)
    x.fork([-1, -1, -1], 0)                                     # three requests, without pages yet,
    x.fork(None, 330)                                           # and room for their contexts
    x.append([page * 5 + 3, 0, 1])
    x.check()
    x.fork([0, 0, 0, 1, 2], 9)                                  # the first one is continued three times
    x.check()
    free = int(x.free.item())
    for T in (5, 1, 9):
        x.tree_step(T)
        x.fork(None, 9)                                         # room for the next tree
        x.check()
    x.sparse_step(2, 1, 1)
    x.check()
    x.fork([2, 0, 0, -1, 3], 0)                                 # two dropped, one continued twice, one new
    x.fork(None, 20)
    x.append([7, 0, 3, 11, 2])
    x.tree_step(7)
    x.fork(None, 1)
    x.sparse_step(3, 0, 1)
    x.check()
    x.fork([-1], 0)
    assert int(x.free.item()) == 2400 // page > free            # nobody holds a page any more


def test_a_context_that_all_slots_share():
    """The context's own attention (its retained blocks) and each slot's rows, joined by their sums: the float32 outputs are parts."""
    S, T, Hq, Hkv, d, block, g = 3, 4, 8, 2, 128, 128, 4
    gen = torch.Generator().manual_seed(7)
    ctx = [torch.randn(2 * block, Hkv, d, generator=gen).to(BF) for _ in range(2)]
    c = R.Cache([40, 0, 131], 32, Hkv, d, room=T, seed=3)
    q = torch.randn(S, T, Hq, d, generator=gen).to(BF)
    k, v = (torch.randn(S, T, Hkv, d, generator=gen).to(BF) for _ in range(2))
    out = torch.empty(S, T, Hq, d, device=DEV)
    O, LSE = binding.pulsar_tree_attn(q.to(DEV), k.to(DEV), v.to(DEV), c.K.to(DEV), c.V.to(DEV), c.table.to(DEV), c.lens.to(DEV), out=out)
    _, _, pO, pL = binding.pulsar_phase2_attn(q.view(S * T, Hq, d).to(DEV), ctx[0].to(DEV), ctx[1].to(DEV), 2, block, n_splits=1, want_partials=True)
    O, LSE = binding.pulsar_lse_merge(torch.cat([pO.view(-1, S * T * Hq, d), O.view(1, -1, d)]), torch.cat([pL.view(-1, S * T * Hq), LSE.view(1, -1)]))
    for s in range(S):
        K, V = c.rows(s, int(c.lens[s]), c.K), c.rows(s, int(c.lens[s]), c.V)
        for t in range(T):
            Kh, Vh = (torch.cat([y.double(), x, z[s, :t + 1].double()]) for y, x, z in ((ctx[0], K, k), (ctx[1], V, v)))
            R.check(O.view(S, T, Hq, d)[s, t], LSE.view(S, T, Hq)[s, t], attend(q[s, t].double(), Kh, Vh, g), f"slot {s} token {t}")


def test_selection_among_many_equal_scores_and_pages():
    """More pages than a block of threads holds, and more at the border than it keeps at hand."""
    c = R.Cache([16 * 4500 + 2], 16, 1, 64, room=1)
    gen = torch.Generator().manual_seed(1)
    q, k, v = torch.zeros(1, 1, 2, 64, dtype=BF), torch.randn(1, 1, 1, 64, generator=gen).to(BF), torch.randn(1, 1, 1, 64, generator=gen).to(BF)
    q[..., 0] = 1
    bounds = torch.zeros(c.n_pages, 1, 2, 64)
    bounds[:, 0, 1, 0] = torch.randint(0, 4, (c.n_pages,), generator=gen).float()
    bounds = bounds.to(BF)
    for n, sink, window in ((1500, 2, 3), (300, 0, 0)):
        O, LSE, sel = binding.pulsar_sparse_attn(q.to(DEV), k.to(DEV), v.to(DEV), c.K.to(DEV), c.V.to(DEV), bounds.to(DEV), c.table.to(DEV),
                                                 c.lens.to(DEV), n, sink, window)
        ref = R.sparse_attn(q, k, v, c, bounds, n, sink, window)
        assert torch.equal(sel.cpu(), ref[3])
        R.check(O, LSE, ref)


def test_wide_tables_and_short_slots():
    """Tables for far longer contexts than the slots have: what is past a slot's rows costs nothing and is -1."""
    S, page, width, Hkv, d = 5, 16, 9000, 2, 64
    x = Loop(page, 4, Hkv, d, layers=1, n_pages=200, max_pages=width, seed=4)
    x.fork([-1] * S, 0)
    x.fork(None, 100)
    x.append([100, 3, 0, 64, 17])
    x.fork([3, 0, 1, 1, -1], 20)
    used = [-(-(n + 20) // page) for n in (64, 100, 3, 3)] + [0]
    for s in range(S):
        assert bool((x.table[s, :used[s]] >= 0).all()) and bool((x.table[s, used[s]:] == -1).all())
    x.fork(None, 6)
    x.tree_step(6)
    x.fork(None, 1)
    x.sparse_step(2, 0, 0)
    x.check()
