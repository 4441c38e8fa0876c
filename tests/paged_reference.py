"""Plain 64-bit forms of the paged cache's operators, written from their definitions in include/pulsar.h, and the tensors the
tests feed them.  Everything here runs on the CPU."""
import math

import torch

BF = torch.bfloat16
U = torch.finfo(BF).eps / 2          # a rounding to bf16 is off by at most this share of the value


class Cache:
    """A pool with pages in random order and slots of the given lengths; rows past a slot's length hold NaN."""

    def __init__(self, lens, page, Hkv, d, room=0, n_layers=None, spare=2, seed=0, shared=0):
        g = torch.Generator().manual_seed(seed)
        self.page, self.lens = page, torch.tensor(lens, dtype=torch.int32)
        self.max_pages = max(1, -(-(max(lens) + room) // page))
        S, sp = len(lens), shared // page
        self.n_pages = sp + S * (self.max_pages - sp) + spare
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.table = torch.cat([order[:sp].expand(S, sp), order[sp:sp + S * (self.max_pages - sp)].view(S, -1)], 1).contiguous()
        shape = (() if n_layers is None else (n_layers,)) + (self.n_pages, page, Hkv, d)
        self.K, self.V = (torch.randn(shape, generator=g).to(BF) for _ in range(2))
        live = torch.zeros(self.n_pages, page, dtype=torch.bool)
        for s, n in enumerate(lens):
            rows = torch.arange(n)
            live[self.table[s].long()[rows // page], rows % page] = True
        self.live = live
        for x in (self.K, self.V):
            x.view(-1, self.n_pages, page, Hkv, d)[:, ~live] = float("nan")

    def rows(self, s, n, x):
        """Rows 0 .. n-1 of slot s in one layer's pool x, in 64 bits."""
        r = torch.arange(n)
        return x[self.table[s].long()[r // self.page], r % self.page].double()


def visible(parent, t):
    """Nodes that node t sees."""
    out = []
    while t >= 0:
        out.append(t)
        t = int(parent[t])
    return out


def softmax_attend(q, K, V, scale):
    """q [g, d], K, V [n, d] in 64 bits -> (O, LSE, softmax of |V|: what P's rounding can add up to)."""
    logits = q @ K.T * scale
    p = logits.softmax(-1)
    return p @ V, logits.logsumexp(-1), p @ V.abs()


def tree_attn(Q, Kn, Vn, cache, parent, n_draft=None, scale=None):
    S, T, Hq, d = Q.shape
    Hkv = Kn.shape[2]
    g, scale = Hq // Hkv, scale or 1 / math.sqrt(d)
    O, A = torch.zeros(S, T, Hq, d, dtype=torch.float64), torch.zeros(S, T, Hq, d, dtype=torch.float64)
    LSE = torch.zeros(S, T, Hq, dtype=torch.float64)
    for s in range(S):
        n = int(cache.lens[s])
        K, V = cache.rows(s, n, cache.K), cache.rows(s, n, cache.V)
        for t in range(T if n_draft is None else int(n_draft[s])):
            see = visible(parent[s], t)
            for h in range(Hkv):
                Kh = torch.cat([K[:, h], Kn[s, see, h].double()])
                Vh = torch.cat([V[:, h], Vn[s, see, h].double()])
                at = slice(h * g, (h + 1) * g)
                O[s, t, at], LSE[s, t, at], A[s, t, at] = softmax_attend(Q[s, t, at].double(), Kh, Vh, scale)
    return O, LSE, A


def page_bounds(K, valid=None):
    """[n_pages, page, Hkv, d] -> [n_pages, Hkv, 2, d]: smallest and largest component (NaN spreads)."""
    k = K.double()
    return torch.stack([k.amin(1), k.amax(1)], 2).to(BF)


def select_pages(q, bounds, n_full, k, sink, window):
    """q [g, d], bounds [n_full, 2, d]: ordinals of the selected pages, ascending."""
    q, low, high = q.double()[:, None], bounds[:, 0].double()[None], bounds[:, 1].double()[None]
    score = torch.where(q > 0, q * high, q * low).sum(-1)
    score = torch.where(score.isnan(), -math.inf, score).amax(0).tolist()
    rank = sorted(range(n_full), key=lambda b: (0 if b < sink or b >= n_full - window else 1, -score[b], b))
    return sorted(rank[:k])


def sparse_attn(Q, Kn, Vn, cache, bounds, k, sink, window, n_draft=None, scale=None):
    S, T, Hq, d = Q.shape
    Hkv = Kn.shape[2]
    g, scale, page = Hq // Hkv, scale or 1 / math.sqrt(d), cache.page
    O, A = torch.zeros(S, T, Hq, d, dtype=torch.float64), torch.zeros(S, T, Hq, d, dtype=torch.float64)
    LSE = torch.zeros(S, T, Hq, dtype=torch.float64)
    sel = torch.full((S, T, Hkv, k), -1, dtype=torch.int32)
    for s in range(S):
        n = int(cache.lens[s])
        full = n // page
        K, V = cache.rows(s, n, cache.K), cache.rows(s, n, cache.V)
        for t in range(T if n_draft is None else int(n_draft[s])):
            for h in range(Hkv):
                at = slice(h * g, (h + 1) * g)
                chosen = select_pages(Q[s, t, at], bounds[cache.table[s, :full].long(), h], full, k, sink, window)
                sel[s, t, h, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
                rows = [r for b in chosen for r in range(b * page, (b + 1) * page)] + list(range(full * page, n))
                Kh = torch.cat([K[rows, h], Kn[s, :t + 1, h].double()])
                Vh = torch.cat([V[rows, h], Vn[s, :t + 1, h].double()])
                O[s, t, at], LSE[s, t, at], A[s, t, at] = softmax_attend(Q[s, t, at].double(), Kh, Vh, scale)
    return O, LSE, A, sel


def check(O, LSE, ref, what="", rounded=True):
    """O, LSE from the GPU against (O, LSE, A): P is rounded to bf16 before the PV product (each probability off by at most U of
    itself, so U * A in all), O to bf16 (U of itself); logits are fp32 sums of d exact products and the sum and the exponentials are
    fp32 too: with operands of a few units that is below 2e-4 of A and of LSE's unit."""
    Oref, Lref, A = ref[:3]
    o, l = O.double().cpu(), LSE.double().cpu()
    bound = U * A + (U * Oref.abs() if rounded else 0) + 2e-4 * A + 1e-6
    err = (o - Oref).abs()
    assert bool((err <= bound).all()), f"{what}: {float((err / bound).max()):.2f} of the bound (NaN: {bool(o.isnan().any())})"
    assert float((l - Lref).abs().max()) <= 2e-4, f"{what}: LSE off by {float((l - Lref).abs().max()):.2e}"


def fork(table, lens, parent, n_pages, page, reserve):
    """(new_table, new_len, n_free, copies [(src, dst, rows)]) by the definition, page by page."""
    S, width = table.shape
    parent = list(range(S)) if parent is None else [int(x) for x in parent]
    new = torch.full((len(parent), width), -1, dtype=torch.int32)
    new_len = torch.zeros(len(parent), dtype=torch.int32)
    first, wants, held = {}, [], set()
    for i, p in enumerate(parent):
        if not 0 <= p < S:
            continue
        n = int(lens[p])
        new_len[i] = n
        kept = -(-n // page)
        need = min(-(-(n + reserve) // page), width)
        copied = n % page != 0 and p in first
        first.setdefault(p, i)
        for o in range(kept):
            if copied and o == kept - 1:
                wants.append((i, o, int(table[p, o]), n % page))
            else:
                new[i, o] = table[p, o] if 0 <= table[p, o] < n_pages else -1
                held.add(int(table[p, o]))
        wants += [(i, o, None, 0) for o in range(kept, need)]
    free = [p for p in range(n_pages) if p not in held]
    copies = []
    for i, o, src, rows in wants:
        if free:
            new[i, o] = free.pop(0)
            if src is not None and 0 <= src < n_pages:
                copies.append((src, int(new[i, o]), rows))
    return new, new_len, len(free), copies
