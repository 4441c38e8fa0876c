"""Operators of a paged key/value cache, as cases to time: page bookkeeping and copies, attention of drafted token
trees, and attention over the pages that a score selects for each query.

Every kind of pass is one call that a serving loop makes:

``fork``       continuations are forked, reordered and dropped: tables, copies of half-filled last pages in every layer
``compact``    the accepted nodes of verified trees move up behind their sequences, in every layer
``summarize``  per-page key bounds of an encoded context
``tree``       one layer's attention of drafted trees over the cached rows (a tree of one node: a decoding step)
``sparse``     one layer's attention of new tokens over the pages with the highest key bounds

Inputs: Q, K, V ~ N(0,1) in bf16 as everywhere in this repository, pages in random order, parents drawn among the earlier
nodes.  ``run`` computes the plain form, or calls the library where ``own`` is true.
"""
import math

import torch

own = False
DEV = "cuda"


def listed():
    return [
        # One decoding step of one short sequence: the smallest call a decoding loop makes.
        dict(name="tree_1_at_6k", kind="tree", slots=1, T=1, len_min=6001, len=6001, page=16, Hq=8, Hkv=2, d=128, ragged=False),
        # One decoding step of 32 continuations of all lengths.
        dict(name="tree_32x1_to_8k", kind="tree", slots=32, T=1, len_min=200, len=8192, page=32, Hq=32, Hkv=8, d=128, ragged=False),
        # Small trees of many sequences, ragged in everything, head dimension 64; some slots have fewer nodes or none.
        dict(name="tree_16x13_d64_ragged", kind="tree", slots=16, T=13, len_min=1, len=5003, page=16, Hq=16, Hkv=4, d=64, ragged=True),
        # Trees of 24 nodes for a few sequences with long contexts.
        dict(name="tree_4x24_to_32k", kind="tree", slots=4, T=24, len_min=20011, len=32768, page=64, Hq=32, Hkv=8, d=128, ragged=False),
        # A tree of 64 nodes behind the longest context.
        dict(name="tree_64_at_128k", kind="tree", slots=1, T=64, len_min=131072, len=131072, page=128, Hq=32, Hkv=8, d=128, ragged=False),
        # A single token that reads 32 pages of a short cache.
        dict(name="sparse_1_at_6k", kind="sparse", slots=1, T=1, len_min=6001, len=6001, page=16, Hq=8, Hkv=2, d=128, k=32, sink=1, window=2),
        # A single token against the longest context: 2048 of 131,072 keys.
        dict(name="sparse_1_at_128k", kind="sparse", slots=1, T=1, len_min=131072, len=131072, page=32, Hq=32, Hkv=8, d=128, k=64, sink=2, window=4),
        # Four tokens each of sixteen long sequences, head dimension 64.
        dict(name="sparse_16x4_to_45k_d64", kind="sparse", slots=16, T=4, len_min=20011, len=45011, page=16, Hq=16, Hkv=4, d=64, k=48, sink=1, window=2),
        # Eight short samples of one prompt, reordered.
        dict(name="fork_8", kind="fork", slots=8, len_min=905, len=1100, shared=896, page=16, reserve=1, n_layers=2, Hkv=2, d=128),
        # 64 continuations of a 16K context: a third of them is replaced.
        dict(name="fork_64_of_16k", kind="fork", slots=64, len_min=16400, len=16704, shared=16384, page=64, reserve=64, n_layers=8, Hkv=8, d=128),
        # 64 verified trees of 64 nodes.
        dict(name="compact_64x64", kind="compact", slots=64, T=64, len_min=50, len=900, page=64, n_layers=8, Hkv=8, d=128),
        # The key bounds of the longest context.
        dict(name="summarize_128k", kind="summarize", slots=1, len_min=131072, len=131072, page=32, n_layers=1, Hkv=8, d=128),
    ]


HEADS = ((4, 1), (8, 2), (16, 4), (32, 8), (8, 8), (16, 2), (16, 1))


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choices(("tree", "sparse", "fork", "compact", "summarize"), (5, 4, 2, 1, 1))[0]
    page = rng.choice((16, 32, 64, 128))
    Hq, Hkv = rng.choice(HEADS)
    d = rng.choice((64, 128, 128))
    slots = _log_int(rng, 1, 32)
    if kind == "tree":
        T = rng.choice((1, _log_int(rng, 1, 64), rng.randint(2, 64)))
        longest = _log_int(rng, 60, max(100, min(131072, 131072 * 8 // (slots * Hkv), 131072 * 64 * 32 // (slots * T * Hq))))
        return dict(kind=kind, slots=slots, T=T, len_min=rng.randint(0, longest), len=longest, page=page, Hq=Hq, Hkv=Hkv, d=d,
                    ragged=rng.random() < 0.3)
    if kind == "sparse":
        T = rng.choice((1, 1, rng.randint(1, 6)))
        longest = _log_int(rng, 500, max(1000, min(131072, 131072 * 8 // (slots * Hkv))))
        sink, window = rng.randint(0, 2), rng.randint(0, 4)
        k = max(sink + window, 1, _log_int(rng, 4, max(8, min(128, 4096 // page, 2 ** 20 // (slots * T * Hkv * page)))))
        return dict(kind=kind, slots=slots, T=T, len_min=rng.randint(longest // 2, longest), len=longest, page=page, Hq=Hq, Hkv=Hkv,
                    d=d, k=k, sink=sink, window=window)
    n_layers = rng.randint(1, 6)
    if kind == "fork":
        shared = page * _log_int(rng, 1, 4096 // page)
        longest = shared + _log_int(rng, 1, 400)
        return dict(kind=kind, slots=slots, len_min=rng.randint(shared, longest), len=longest, shared=shared, page=page,
                    reserve=rng.choice((0, 1, rng.randint(2, 64))), n_layers=n_layers, Hkv=Hkv, d=d)
    longest = _log_int(rng, 50, 1500)
    if kind == "compact":
        return dict(kind=kind, slots=slots, T=rng.randint(2, 64), len_min=rng.randint(0, longest), len=longest, page=page,
                    n_layers=n_layers, Hkv=Hkv, d=d)
    return dict(kind=kind, slots=slots, len_min=rng.randint(page, page + longest), len=page + longest, page=page, n_layers=n_layers,
                Hkv=Hkv, d=d)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _lens(c):
    """Rows in the cache per slot: from the shortest to the longest (prepare puts them in a random order)."""
    n, lo, hi = c["slots"], c["len_min"], c["len"]
    return [lo + (hi - lo) * i // (n - 1) if n > 1 else hi for i in range(n)]


def _drafts(c):
    """Nodes per slot: all, or T, T - 3, T - 6, ... and none at all."""
    T = c["T"]
    return [T if not c["ragged"] else max(0, T - 3 * (i % (T // 3 + 2))) for i in range(c["slots"])]


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    c, gen = dict(case), torch.Generator(device=DEV).manual_seed(seed)
    kind, slots, page, Hkv, d = c["kind"], c["slots"], c["page"], c["Hkv"], c["d"]
    s = dict(kind=kind, case=c)
    order = torch.randperm(slots, generator=gen, device=DEV)
    lens = s["lens"] = _ints(_lens(c))[order].contiguous()
    behind = {"fork": c.get("reserve", 0), "summarize": 0}.get(kind, c.get("T", 0))
    width = -(-(c["len"] + behind) // page)
    shared = c.get("shared", 0) // page
    own_pages = width - shared
    n_pages = shared + slots * (own_pages + (width - shared + 1 if kind == "fork" else 0)) + 3
    at = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.empty(slots, width, dtype=torch.int32, device=DEV)
    table[:, :shared] = at[:shared]
    table[:, shared:] = at[shared:shared + slots * own_pages].view(slots, own_pages)
    if kind == "fork":
        table[torch.arange(width, device=DEV) * page >= lens[:, None]] = -1
    s["table"] = table
    n_layers = (c["n_layers"],) if "n_layers" in c else ()
    s["K"] = _randn(gen, *n_layers, n_pages, page, Hkv, d)
    if kind == "summarize":
        s["summary"] = torch.zeros(*n_layers, n_pages, Hkv, 2, d, dtype=torch.bfloat16, device=DEV)
        return s
    s["V"] = _randn(gen, *n_layers, n_pages, page, Hkv, d)
    if kind == "fork":
        parent = torch.randint(0, slots, (slots,), generator=gen, device=DEV, dtype=torch.int32)
        kept = torch.rand(slots, generator=gen, device=DEV)
        same = torch.arange(slots, device=DEV, dtype=torch.int32)
        s["parent"] = torch.where(kept < 0.66, same, torch.where(kept < 0.97, parent, -1))
        return s
    T = c["T"]
    if kind == "compact":
        n = torch.randint(1, min(T, 8) + 1, (slots, 1), generator=gen, device=DEV)
        ranks = torch.rand(slots, T, generator=gen, device=DEV).argsort(1).argsort(1)
        nodes = torch.where(ranks < n, torch.arange(T, device=DEV), T).sort(1).values
        s["accept"] = torch.where(nodes < T, nodes, -1).to(torch.int32)
        return s
    Hq = c["Hq"]
    s["Q"], s["Kn"], s["Vn"] = _randn(gen, slots, T, Hq, d), _randn(gen, slots, T, Hkv, d), _randn(gen, slots, T, Hkv, d)
    if kind == "tree":
        u = torch.rand(slots, T, generator=gen, device=DEV)
        s["parent"] = ((u * torch.arange(1, T + 1, device=DEV)).floor().to(torch.int32) - 1).contiguous()
        s["drafts"] = _ints(_drafts(c))[order].contiguous()
        s["O"] = torch.zeros(slots, T, Hq, d, dtype=torch.bfloat16, device=DEV)
        s["LSE"] = torch.zeros(slots, T, Hq, dtype=torch.float32, device=DEV)
        return s
    k = s["K"].float()
    s["summary"] = torch.stack([k.amin(1), k.amax(1)], 2).to(torch.bfloat16).contiguous()      # [n_pages, Hkv, 2, d]
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------

def _plain_fork(s):
    c, table, lens, parent = s["case"], s["table"].long(), s["lens"].long(), s["parent"].long()
    page, width, slots = c["page"], table.shape[1], parent.shape[0]
    n_pages = s["K"].shape[1]
    alive = parent >= 0
    new_len = torch.where(alive, lens[parent.clamp(min=0)], 0)
    kept = (new_len + page - 1) // page
    need = torch.where(alive, ((new_len + c["reserve"] + page - 1) // page).clamp(max=width), 0)
    ordinal = torch.arange(width, device=DEV)
    earlier = torch.ones(slots, slots, dtype=torch.bool, device=DEV).tril(-1)
    first = ~((parent[:, None] == parent[None, :]) & earlier).any(1)
    copied = alive & ~first & (new_len % page != 0)
    from_parent = ordinal < kept[:, None]
    fresh = (~from_parent & (ordinal < need[:, None])) | (copied[:, None] & (ordinal == kept[:, None] - 1))
    old = torch.where(from_parent, table[parent.clamp(min=0)], -1)
    used = torch.zeros(n_pages + 1, dtype=torch.bool, device=DEV)
    used[torch.where(fresh, n_pages, torch.where(old >= 0, old, n_pages))] = True
    used = used[:n_pages]
    free = torch.argsort(used.to(torch.uint8), stable=True)                  # the free pages first, ascending
    n_free = (~used).sum()
    rank = fresh.flatten().cumsum(0).view_as(fresh) - 1
    page_of = torch.where(rank < n_free, free[rank.clamp(min=0, max=n_pages - 1)], -1)
    new = torch.where(fresh, page_of, old)
    tail = (kept - 1).clamp(min=0)[:, None]
    src, dst = old.gather(1, tail)[:, 0], new.gather(1, tail)[:, 0]
    row = torch.arange(page, device=DEV)
    rows = (copied & (src >= 0) & (dst >= 0))[:, None] & (row < (new_len % page)[:, None])
    at = lambda p: (p[:, None] * page + row)[rows]
    for_all = lambda x: x.view(x.shape[0], n_pages * page, *x.shape[3:])
    K, V = for_all(s["K"]), for_all(s["V"])
    K[:, at(dst)] = K[:, at(src)]
    V[:, at(dst)] = V[:, at(src)]
    left = (n_free - fresh.sum()).clamp(min=0)
    return new.to(torch.int32), new_len.to(torch.int32), left.to(torch.int32).view(1)


def _flat_rows(s, rows):
    """Rows of the pool where the slots' ``rows`` [slots, n] lie."""
    page = s["case"]["page"]
    return s["table"].long().gather(1, rows // page) * page + rows % page


def _plain_compact(s):
    lens, accept = s["lens"].long(), s["accept"].long()
    valid = accept >= 0
    src = _flat_rows(s, lens[:, None] + accept.clamp(min=0))[valid]
    dst = _flat_rows(s, lens[:, None] + torch.arange(accept.shape[1], device=DEV))[valid]
    K, V = (x.view(x.shape[0], -1, *x.shape[3:]) for x in (s["K"], s["V"]))
    K[:, dst] = K[:, src]
    V[:, dst] = V[:, src]
    return (lens + valid.sum(1)).to(torch.int32)


def _plain_summarize(s):
    page, table = s["case"]["page"], s["table"].long()
    full = torch.arange(table.shape[1], device=DEV) < (s["lens"].long() // page)[:, None]
    pages = table[full]
    k = s["K"][:, pages].float()
    s["summary"][:, pages] = torch.stack([k.amin(2), k.amax(2)], 3).to(torch.bfloat16)


def _append(s, valid):
    rows = _flat_rows(s, s["lens"].long()[:, None] + torch.arange(valid.shape[1], device=DEV))[valid]
    s["K"].flatten(0, 1)[rows] = s["Kn"][valid]
    s["V"].flatten(0, 1)[rows] = s["Vn"][valid]


def _softmax_values(scores, values):
    """Softmax over the keys of several parts and its value sum: scores [..., n], values [..., n, d], joined over the parts."""
    m = torch.stack([x.amax(-1) for x in scores]).amax(0)
    p = [(x - m[..., None]).exp() for x in scores]
    total = torch.stack([x.sum(-1) for x in p]).sum(0)
    out = torch.stack([(x[..., None, :] @ v).squeeze(-2) if v.dim() == x.dim() + 1 else x @ v for x, v in zip(p, values)]).sum(0)
    return out / total[..., None], m + total.log()


def _plain_tree(s):
    c, lens = s["case"], s["lens"].long()
    page, Hkv, d, T, slots = c["page"], c["Hkv"], c["d"], c["T"], c["slots"]
    g = c["Hq"] // Hkv
    node = torch.arange(T, device=DEV)
    valid = node < s["drafts"][:, None]
    _append(s, valid)
    P = -(-c["len"] // page)
    pages = s["table"][:, :P].long()
    rows = P * page
    K = s["K"][pages].view(slots, rows, Hkv, d).permute(0, 2, 1, 3).float()                 # [slots, Hkv, rows, d]
    V = s["V"][pages].view(slots, rows, Hkv, d).permute(0, 2, 1, 3).float()
    Kn, Vn = s["Kn"].permute(0, 2, 1, 3).float(), s["Vn"].permute(0, 2, 1, 3).float()
    q = s["Q"].view(slots, T, Hkv, g, d).permute(0, 2, 1, 3, 4).reshape(slots, Hkv, T * g, d).float() * d ** -0.5
    # a node's ancestors: powers of the matrix that steps from a node to its parent or stays
    step = torch.eye(T, device=DEV) + (s["parent"][:, :, None] == node)
    sees = (torch.linalg.matrix_power(step, T) > 0).repeat_interleave(g, 1)[:, None]
    cached = (torch.arange(rows, device=DEV) < lens[:, None])[:, None, None]
    scores = [(q @ K.transpose(-1, -2)).masked_fill(~cached, -math.inf), (q @ Kn.transpose(-1, -2)).masked_fill(~sees, -math.inf)]
    O, LSE = _softmax_values(scores, [V, Vn])
    back = lambda x: x.view(slots, Hkv, T, g, *x.shape[3:]).transpose(1, 2).flatten(2, 3)
    s["O"].copy_(torch.where(valid[:, :, None, None], back(O).to(torch.bfloat16), s["O"]))
    s["LSE"].copy_(torch.where(valid[:, :, None], back(LSE), s["LSE"]))
    return s["O"], s["LSE"]


def _plain_sparse(s):
    c, lens = s["case"], s["lens"].long()
    page, Hkv, d, T, slots, k = c["page"], c["Hkv"], c["d"], c["T"], c["slots"], c["k"]
    g = c["Hq"] // Hkv
    node = torch.arange(T, device=DEV)
    _append(s, torch.ones(slots, T, dtype=torch.bool, device=DEV))
    table = s["table"].long()
    n_full = lens // page
    P = c["len"] // page
    # scores of the full pages, in 64 bits: pages next to the border are told apart, equal ones are equal
    bounds = s["summary"][table[:, :P]].double().permute(0, 2, 3, 4, 1)                       # [slots, Hkv, 2, d, P]
    q = s["Q"].view(slots, T, Hkv, g, d).permute(0, 2, 1, 3, 4).flatten(2, 3)                  # [slots, Hkv, T * g, d]
    score = q.double().clamp(max=0) @ bounds[:, :, 0] + q.double().clamp(min=0) @ bounds[:, :, 1]
    score = score.view(slots, Hkv, T, g, P).amax(3)
    ordinal = torch.arange(P, device=DEV)
    full = (ordinal < n_full[:, None])[:, None, None]
    forced = ((ordinal < c["sink"]) | (ordinal >= n_full[:, None] - c["window"]))[:, None, None]
    score = score.masked_fill(forced, math.inf).masked_fill(~full, -math.inf)
    kk = min(k, P)
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :kk]
    best = torch.where(full.expand_as(score).gather(-1, best), best, P).sort(-1).values
    sel = torch.full((slots, T, Hkv, k), -1, dtype=torch.int32, device=DEV)
    sel[..., :kk] = torch.where(best < P, best, -1).transpose(1, 2)
    # attention over the selected pages, the rows after the last full page, and the new tokens
    ids = table.gather(1, best.clamp(max=P - 1).flatten(1)).view_as(best)[..., None]            # [slots, Hkv, T, kk, 1]
    place = (ids * page + torch.arange(page, device=DEV)).flatten(3)
    head = torch.arange(Hkv, device=DEV)[:, None, None]
    K, V = s["K"].view(-1, Hkv, d), s["V"].view(-1, Hkv, d)
    qf = q.view(slots, Hkv, T, g, d).float() * d ** -0.5
    taken = (best < P).repeat_interleave(page, -1)[:, :, :, None]
    scores = [(qf @ K[place, head].float().transpose(-1, -2)).masked_fill(~taken, -math.inf)]
    tail = (n_full * page)[:, None] + torch.arange(page, device=DEV)
    in_tail = tail < lens[:, None]
    rows = _flat_rows(s, torch.where(in_tail, tail, 0))
    Kt, Vt = (x[rows].permute(0, 2, 1, 3).float()[:, :, None] for x in (K, V))
    scores.append((qf @ Kt.transpose(-1, -2)).masked_fill(~in_tail[:, None, None, None], -math.inf))
    Kn, Vn = (x.permute(0, 2, 1, 3).float()[:, :, None] for x in (s["Kn"], s["Vn"]))
    scores.append((qf @ Kn.transpose(-1, -2)).masked_fill((node > node[:, None])[:, None], -math.inf))
    O, LSE = _softmax_values(scores, [V[place, head].float(), Vt, Vn])
    back = lambda x: x.transpose(1, 2).flatten(2, 3)
    return back(O).to(torch.bfloat16), back(LSE).contiguous(), sel


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(s):
    c, kind = s["case"], s["kind"]
    if own:
        from paper_2607_20457_b200 import binding
    if kind == "fork":
        if own:
            table, lens, free = binding.pulsar_pages_fork(s["table"], s["lens"], s["parent"], s["K"], s["V"], c["reserve"])
        else:
            table, lens, free = _plain_fork(s)
        return dict(table=table, lens=lens, free=free, K=s["K"], V=s["V"])
    if kind == "compact":
        if own:
            lens = binding.pulsar_pages_compact(s["K"], s["V"], s["table"], s["lens"], s["accept"])
        else:
            lens = _plain_compact(s)
        return dict(lens=lens, K=s["K"], V=s["V"])
    if kind == "summarize":
        if own:
            binding.pulsar_pages_summarize(s["K"], s["table"], None, s["lens"], s["summary"])
        else:
            _plain_summarize(s)
        return dict(summary=s["summary"])
    if kind == "tree":
        if own:
            O, LSE = binding.pulsar_tree_attn(s["Q"], s["Kn"], s["Vn"], s["K"], s["V"], s["table"], s["lens"], s["parent"],
                                              s["drafts"] if c["ragged"] else None, out=s["O"], lse_out=s["LSE"])
        else:
            O, LSE = _plain_tree(s)
        return dict(O=O, LSE=LSE, K=s["K"], V=s["V"])
    if own:
        O, LSE, sel = binding.pulsar_sparse_attn(s["Q"], s["Kn"], s["Vn"], s["K"], s["V"], s["summary"], s["table"], s["lens"],
                                                 c["k"], c["sink"], c["window"])
    else:
        O, LSE, sel = _plain_sparse(s)
    return dict(O=O, LSE=LSE, sel=sel, K=s["K"], V=s["V"])


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def exact(case, seed):
    c, kind = dict(case), case["kind"]
    if kind in ("fork", "compact"):
        return None                                         # whole numbers and copies
    s = prepare(case, seed)
    page, Hkv, d, slots = c["page"], c["Hkv"], c["d"], c["slots"]
    lens, table = s["lens"].tolist(), s["table"].long()
    if kind == "summarize":
        out = s["summary"].double()
        for i in range(slots):
            for b in table[i, :lens[i] // page].split(1024):
                out[:, b] = torch.stack([s["K"][:, b].double().min(2).values, s["K"][:, b].double().max(2).values], 3)
        return dict(summary=out)
    T, Hq = c["T"], c["Hq"]
    g = Hq // Hkv
    O = torch.zeros(slots, T, Hq, d, dtype=torch.float64, device=DEV)
    LSE = torch.zeros(slots, T, Hq, dtype=torch.float64, device=DEV)
    drafts = s["drafts"].tolist() if kind == "tree" else [T] * slots
    parents = s["parent"].tolist() if kind == "tree" else None

    def attend(q, keys, values):                            # q [.., d] of one head, keys [n, d]
        logits = q @ keys.T / math.sqrt(d)
        return logits.softmax(-1) @ values, logits.logsumexp(-1)

    for i in range(slots):
        n = lens[i]
        rows = (table[i, torch.arange(n, device=DEV) // page] * page + torch.arange(n, device=DEV) % page)
        for h in range(Hkv):
            K = s["K"].view(-1, Hkv, d)[rows, h].double()
            V = s["V"].view(-1, Hkv, d)[rows, h].double()
            kn, vn, q = s["Kn"][i, :, h].double(), s["Vn"][i, :, h].double(), s["Q"][i, :, h * g:(h + 1) * g].double()
            if kind == "tree":
                if drafts[i] == 0:
                    continue
                hidden = torch.ones(T, T, dtype=torch.bool)
                for t in range(drafts[i]):
                    a = t
                    while a >= 0:
                        hidden[t, a] = False
                        a = parents[i][a]
                logits = torch.cat([q @ K.T, (q @ kn.T).masked_fill(hidden[:, None].to(DEV), -math.inf)], -1)[:drafts[i]] / math.sqrt(d)
                O[i, :drafts[i], h * g:(h + 1) * g] = logits.softmax(-1) @ torch.cat([V, vn])
                LSE[i, :drafts[i], h * g:(h + 1) * g] = logits.logsumexp(-1)
                continue
            full = n // page
            for t in range(T):
                low, high = s["summary"][table[i, :full], h].double().unbind(1)
                value = torch.stack([torch.maximum(x * low, x * high).sum(-1) for x in q[t]]).max(0).values
                value[:c["sink"]] = math.inf
                value[max(0, full - c["window"]):] = math.inf
                chosen = torch.argsort(-value, stable=True)[:c["k"]]
                at = (chosen[:, None] * page + torch.arange(page, device=DEV)).flatten()
                at = torch.cat([at, torch.arange(full * page, n, device=DEV)])
                O[i, t, h * g:(h + 1) * g], LSE[i, t, h * g:(h + 1) * g] = attend(q[t], torch.cat([K[at], kn[:t + 1]]),
                                                                                  torch.cat([V[at], vn[:t + 1]]))
    return dict(O=O, LSE=LSE, sel=None, K=None, V=None) if kind == "sparse" else dict(O=O, LSE=LSE, K=None, V=None)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------

def work(case):
    c, kind = dict(case), case["kind"]
    row = 2 * c["Hkv"] * c["d"]                             # bytes of a row of K or V
    lens, page = _lens(c), c["page"]
    if kind == "fork":                                       # tables in and out; about a third of the slots gets a copy of its last page
        entries = 8 * sum(-(-n // page) for n in lens)
        return dict(bytes=entries + 4 * row * c["n_layers"] * sum(n % page for n in lens) // 3, flops=0)
    if kind == "compact":
        return dict(bytes=c["slots"] * (min(c["T"], 8) + 1) // 2 * 4 * row * c["n_layers"], flops=0)
    if kind == "summarize":
        full = sum(n // page for n in lens)
        return dict(bytes=c["n_layers"] * row * (full * page + 2 * full), flops=2 * c["n_layers"] * full * page * c["Hkv"] * c["d"])
    drafts = _drafts(c) if kind == "tree" else [c["T"]] * c["slots"]
    token = 4 * c["Hq"] * c["d"] + 4 * c["Hq"] + 4 * row     # Q, O, LSE; new K and V in, and to their pages
    if kind == "tree":
        keys = sum(n for n, t in zip(lens, drafts) if t)
        pairs = sum(t * (n + t // 2) for n, t in zip(lens, drafts))
        return dict(bytes=2 * row * keys + token * sum(drafts), flops=4 * c["d"] * c["Hq"] * pairs)
    full = [n // page for n in lens]
    read = sum(2 * row * f for f in full)                    # key bounds of the full pages
    keys = [min(c["k"], f) * page + n - f * page for f, n in zip(full, lens)]
    # (tokens and heads choose their own pages: at most all rows of the cache are read)
    rows = sum(min(c["T"] * (m - m % page) + m % page, n) for m, n in zip(keys, lens))
    flops = 4 * c["d"] * c["Hq"] * c["T"] * sum(keys) + 2 * c["d"] * c["Hq"] * c["T"] * sum(full)
    return dict(bytes=read + 2 * row * rows + token * c["T"] * c["slots"], flops=flops)
