"""GPU parity: attention of drafted trees over a paged cache against its definition in 64 bits."""
import pytest
import torch

import paged_reference as R
from paper_2607_20457_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def drafts(S, T, Hq, Hkv, d, seed=0, scale=1.0, shape="random"):
    g = torch.Generator().manual_seed(seed)
    Q = (torch.randn(S, T, Hq, d, generator=g) * scale).to(BF)
    Kn, Vn = (torch.randn(S, T, Hkv, d, generator=g).to(BF) for _ in range(2))
    t = torch.arange(T, dtype=torch.int32)
    if shape == "chain":
        parent = (t - 1).expand(S, T)
    elif shape == "star":
        parent = torch.where(t == 0, -1, 0).expand(S, T)
    elif shape == "forest":
        parent = torch.full((S, T), -1)
    else:
        parent = (torch.rand(S, T, generator=g) * (t + 1)).floor() - 1
    return Q, Kn, Vn, parent.to(torch.int32).contiguous()


def run(c, Q, Kn, Vn, parent, n_draft=None, scale=0.0, f32=False, expect=0, ref_parent=None, ref_cache=None, what=""):
    S, T, Hq, d = Q.shape
    K, V = c.K.to(DEV), c.V.to(DEV)
    status = binding.new_status(DEV)
    out = torch.full(Q.shape, 77.0, dtype=torch.float32 if f32 else BF, device=DEV)
    lse = torch.full((S, T, Hq), 77.0, device=DEV)
    nd = None if n_draft is None else torch.tensor(n_draft, dtype=torch.int32, device=DEV)
    O, LSE = binding.pulsar_tree_attn(Q.to(DEV), Kn.to(DEV), Vn.to(DEV), K, V, c.table.to(DEV), c.lens.to(DEV),
                                      None if parent is None else parent.to(DEV), nd, scale, out=out, lse_out=lse, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == expect
    counts = [T] * S if n_draft is None else [min(max(n, 0), T) for n in n_draft]
    par = ref_parent if ref_parent is not None else parent if parent is not None else (torch.arange(T) - 1).expand(S, T)
    ref = R.tree_attn(Q, Kn, Vn, ref_cache or c, par, counts, scale or None)
    used = torch.arange(T) < torch.tensor(counts)[:, None]
    assert bool((O.cpu()[~used] == 77.0).all()) and bool((LSE.cpu()[~used] == 77.0).all())
    if used.any():
        R.check(O.cpu()[used], LSE.cpu()[used], [x[used] for x in ref], what, rounded=not f32)
    if expect == 0:                                       # the nodes' rows are in the pages, all others as they were
        for x, new, old in ((K, Kn, c.K.clone()), (V, Vn, c.V.clone())):
            for s in range(S):
                r = int(c.lens[s]) + torch.arange(counts[s])
                old[c.table[s].long()[r // c.page], r % c.page] = new[s, :counts[s]]
            assert torch.equal(x.cpu().view(torch.int16), old.view(torch.int16))
    return O, LSE


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 1), (8, 8), (8, 4), (16, 2), (16, 1)])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_heads_pages_and_lengths(d, Hq, Hkv, page):
    lens = [0, 1, 15, 16, 17, 100, 127, 128, 129, 311]
    for T in (1, 2, 5):
        c = R.Cache(lens, page, Hkv, d, room=T, seed=T)
        run(c, *drafts(len(lens), T, Hq, Hkv, d, seed=T), what=f"T={T}")


@pytest.mark.parametrize("T", [3, 8, 16, 17, 31, 32, 33, 48, 63, 64])
@pytest.mark.parametrize("shape", ["random", "chain", "star", "forest"])
def test_trees(T, shape):
    for Hq, Hkv, d, page in ((8, 2, 128, 16), (4, 4, 64, 64)):
        c = R.Cache([0, 40, 200], page, Hkv, d, room=T, seed=T)
        run(c, *drafts(3, T, Hq, Hkv, d, seed=T, shape=shape), what=f"d={d}")


@pytest.mark.parametrize("Hq,Hkv,d,page", [(16, 1, 128, 16), (32, 2, 64, 128), (16, 4, 128, 32)])
def test_many_rows_per_head(Hq, Hkv, d, page):
    c = R.Cache([500, 3, 129], page, Hkv, d, room=64)
    run(c, *drafts(3, 40, Hq, Hkv, d))


def test_slots_with_fewer_nodes_or_none():
    c = R.Cache([30, 0, 64, 5, 90], 16, 2, 64, room=9)
    run(c, *drafts(5, 9, 8, 2, 64), n_draft=[9, 0, 1, 4, -3])
    run(c, *drafts(5, 9, 8, 2, 64), n_draft=[0, 0, 0, 0, 0])
    run(c, *drafts(5, 9, 8, 2, 64)[:3], None, n_draft=[3, 9, 20, 8, 1])


def test_ragged_batch_of_long_and_short_slots():
    lens = [0, 5000, 3, 1, 900, 2500, 16, 0, 33]
    c = R.Cache(lens, 32, 2, 128, room=6)
    run(c, *drafts(len(lens), 6, 8, 2, 128))
    run(c, *drafts(len(lens), 6, 8, 2, 128, seed=9), n_draft=[6, 1, 0, 2, 6, 3, 0, 5, 6])


def test_many_slots():
    g = torch.Generator().manual_seed(4)
    lens = torch.randint(0, 120, (300,), generator=g).tolist()
    c = R.Cache(lens, 16, 1, 64, room=2)
    run(c, *drafts(300, 2, 2, 1, 64))


@pytest.mark.parametrize("Hq,Hkv,T", [(8, 2, 1), (8, 2, 20)])
def test_peaked_and_scaled_logits(Hq, Hkv, T):
    c = R.Cache([700, 44], 16, Hkv, 128, room=T)
    Q, Kn, Vn, parent = drafts(2, T, Hq, Hkv, 128, scale=1.0)
    run(c, Q, Kn, Vn, parent, scale=0.3)
    run(c, Q, Kn, Vn, parent, scale=1e-3)


def test_float32_output_joins_a_context_that_all_slots_share():
    """Continuations of one encoded context: Phase 2 over the shared context and the trees' own pages are parts of one softmax."""
    L, S, T, Hq, Hkv, d = 1500, 3, 4, 8, 2, 128
    c = R.Cache([20, 0, 77], 16, Hkv, d, room=T)
    Q, Kn, Vn, parent = drafts(S, T, Hq, Hkv, d)
    O1, LSE1 = run(c, Q, Kn, Vn, parent, f32=True)
    g = torch.Generator().manual_seed(6)
    K, V = (torch.randn(L, Hkv, d, generator=g).to(BF) for _ in range(2))
    _, _, part_O, part_L = binding.pulsar_phase2_attn(Q.view(S * T, Hq, d).to(DEV), K.to(DEV), V.to(DEV), 1, L, n_splits=2, want_partials=True)
    O, LSE = binding.pulsar_lse_merge(torch.cat([part_O.view(2, -1, d), O1.view(1, -1, d)]).contiguous(),
                                      torch.cat([part_L.view(2, -1), LSE1.view(1, -1)]).contiguous())
    both = R.Cache([L + 20, L, L + 77], 16, Hkv, d)
    for s, n in enumerate((20, 0, 77)):
        for x, y, pool in ((both.K, K, c.K), (both.V, V, c.V)):
            rows = torch.cat([y.double(), c.rows(s, n, pool)]).to(BF)
            r = torch.arange(len(rows))
            x[both.table[s].long()[r // 16], r % 16] = rows
    Oref, Lref, A = R.tree_attn(Q, Kn, Vn, both, parent)
    R.check(O.view(S, T, Hq, d).cpu(), LSE.view(S, T, Hq).cpu(), (Oref, Lref, A))


def test_bad_parents_pages_and_lengths_are_reported():
    c = R.Cache([40, 40], 16, 2, 64, room=6)
    Q, Kn, Vn, parent = drafts(2, 6, 8, 2, 64)
    bad = parent.clone()
    bad[0, 2], bad[1, 3], bad[1, 5] = 2, -9, 7
    good = bad.clone()
    good[0, 2] = good[1, 3] = good[1, 5] = -1
    run(c, Q, Kn, Vn, bad, ref_parent=good, expect=binding.DEV_BAD_TREE)
    # a page that does not exist: its 16 rows count as absent
    for page_id in (-1, c.n_pages, 1 << 30):
        b = R.Cache([40, 40], 16, 2, 64, room=6)
        b.table[0, 1] = page_id
        without = R.Cache([40, 40], 16, 2, 64, room=6)
        for x in (without.K, without.V):                  # rows 32..39 move up to 16..23
            x[without.table[0, 1], :8] = x[without.table[0, 2], :8].clone()
        without.lens[0] = 24
        run(b, Q, Kn, Vn, parent, ref_cache=without, expect=binding.DEV_BAD_PAGE)
    # the table ends inside the tree: attended to, not written
    e = R.Cache([44, 40], 16, 2, 64)
    run(e, Q, Kn, Vn, parent, expect=binding.DEV_BAD_LENGTH)
    e.lens[0] = 1000
    f = R.Cache([48, 40], 16, 2, 64)
    for x, y in ((e.K, f.K), (e.V, f.V)):
        x.copy_(torch.where(x.isnan(), torch.ones_like(x), x))
        y.copy_(x)
    run(e, Q, Kn, Vn, parent, ref_cache=f, expect=binding.DEV_BAD_LENGTH)


def test_infinities_and_nan_stay_with_who_sees_them():
    """A NaN key of a node reaches its descendants and nobody else; unwritten rows (NaN here) reach nobody."""
    c = R.Cache([50], 16, 1, 64, room=8)
    Q, Kn, Vn, _ = drafts(1, 8, 4, 1, 64)
    parent = torch.tensor([[-1, 0, 0, 1, 2, -1, 5, 3]], dtype=torch.int32)
    Vn[0, 1] = float("nan")
    O, _ = binding.pulsar_tree_attn(*(x.to(DEV) for x in (Q, Kn, Vn, c.K, c.V, c.table, c.lens, parent)))
    assert [bool(x) for x in O.isnan().flatten(2).any(2)[0].cpu()] == [False, True, False, True, False, False, False, True]
    ref = R.tree_attn(Q, Kn, Vn, c, parent)
    clean = [0, 2, 4, 5, 6]
    LSE = torch.zeros(1, 8, 4)
    R.check(O.cpu()[:, clean], ref[1][:, clean], [x[:, clean] for x in ref])


def test_chain_equals_the_generation_step():
    L, gen_len, n, Hq, Hkv, d = 4096, 40, 3, 8, 2, 128
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g).to(BF).to(DEV)
    K, V, Kg, Vg = rnd(L, Hkv, d), rnd(L, Hkv, d), rnd(128, Hkv, d), rnd(128, Hkv, d)
    Q, Kn, Vn = rnd(n, Hq, d), rnd(n, Hkv, d), rnd(n, Hkv, d)
    pool = torch.cat([K, Kg]).view(-1, 32, Hkv, d).contiguous(), torch.cat([V, Vg]).view(-1, 32, Hkv, d).contiguous()
    table = torch.arange(pool[0].shape[0], dtype=torch.int32, device=DEV)[None].contiguous()
    length = torch.tensor([L + gen_len], dtype=torch.int32, device=DEV)
    O, LSE = binding.pulsar_tree_attn(Q[None], Kn[None], Vn[None], *pool, table, length)
    O2, LSE2 = binding.pulsar_phase2_generate_step(Q, Kn, Vn, K, V, 1, L, Kg, Vg, gen_len)
    assert float((O[0].float() - O2.float()).abs().max()) <= 2e-3 and float((LSE[0] - LSE2).abs().max()) <= 2e-5
    assert torch.equal(pool[0].view(-1, Hkv, d)[L:L + 128], Kg) and torch.equal(pool[1].view(-1, Hkv, d)[L:L + 128], Vg)


@pytest.mark.parametrize("T", [1, 24])
def test_offsets_past_32_bits(T):
    """Pages whose elements lie beyond 2^31 (and bytes beyond 2^32) from the pool's first."""
    Hkv, Hq, d, page = 8, 32, 128, 128
    n_pages = (1 << 31) // (page * Hkv * d) + 40
    K, V = (torch.empty(n_pages, page, Hkv, d, dtype=BF, device=DEV) for _ in range(2))
    c = R.Cache([600, 77], page, Hkv, d, room=T)
    table = c.table + (n_pages - c.n_pages)
    K[n_pages - c.n_pages:], V[n_pages - c.n_pages:] = c.K.to(DEV), c.V.to(DEV)
    Q, Kn, Vn, parent = drafts(2, T, Hq, Hkv, d)
    O, LSE = binding.pulsar_tree_attn(*(x.to(DEV) for x in (Q, Kn, Vn)), K, V, table.to(DEV), c.lens.to(DEV), parent.to(DEV))
    R.check(O, LSE, R.tree_attn(Q, Kn, Vn, c, parent))
    row = K[table[0, 600 // page], 600 % page:600 % page + 1]
    assert torch.equal(row.cpu()[0], Kn[0, 0])


@pytest.mark.parametrize("Hq,Hkv,d,T", [(32, 8, 128, 1), (32, 8, 128, 24), (8, 1, 64, 40)])
def test_long_caches_on_the_device(Hq, Hkv, d, T):
    """Lengths at which every CTA has a part: compared with 64-bit products on the GPU."""
    lens, page = [30011, 9000], 64
    g = torch.Generator(device=DEV).manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV).to(BF)
    width = -(-(max(lens) + T) // page)
    K, V = rnd(2 * width, page, Hkv, d), rnd(2 * width, page, Hkv, d)
    table = torch.randperm(2 * width, generator=g, device=DEV).to(torch.int32).view(2, width).contiguous()
    Q, Kn, Vn, parent = drafts(2, T, Hq, Hkv, d)
    length = torch.tensor(lens, dtype=torch.int32, device=DEV)
    O, LSE = binding.pulsar_tree_attn(Q.to(DEV), Kn.to(DEV), Vn.to(DEV), K, V, table, length, parent.to(DEV))
    again = binding.pulsar_tree_attn(Q.to(DEV), Kn.to(DEV), Vn.to(DEV), K, V, table, length, parent.to(DEV))
    assert torch.equal(O, again[0]) and torch.equal(LSE, again[1])           # the order of the joins does not depend on timing
    for s, n in enumerate(lens):
        r = torch.arange(n, device=DEV)
        Kc, Vc = (x[table[s].long()[r // page], r % page].double() for x in (K, V))
        hidden = torch.ones(T, T, dtype=torch.bool)
        for t in range(T):
            hidden[t, R.visible(parent[s], t)] = False
        q = Q[s].to(DEV).double().view(T, Hkv, Hq // Hkv, d)
        cat = lambda x, y: torch.cat([x, y[s].to(DEV).double()])
        Kc, Vc = cat(Kc, Kn), cat(Vc, Vn)
        logits = torch.einsum("thgd,nhd->thgn", q, Kc) / d ** 0.5
        logits[..., n:] = logits[..., n:].masked_fill(hidden[:, None, None].to(DEV), float("-inf"))
        p = logits.softmax(-1)
        ref = [torch.einsum("thgn,nhd->thgd", p, v).reshape(T, Hq, d).cpu() for v in (Vc, Vc.abs())]
        R.check(O[s].cpu(), LSE[s].cpu(), (ref[0], logits.logsumexp(-1).view(T, Hq).cpu(), ref[1]))


def test_captured_step_follows_the_lengths_on_the_device():
    T, Hq, Hkv, d = 5, 8, 2, 128
    c = R.Cache([400, 0, 63], 16, Hkv, d, room=200)
    for x in (c.K, c.V):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(8)).to(BF))
    Q, Kn, Vn, parent = (x.to(DEV) for x in drafts(3, T, Hq, Hkv, d))
    K, V, table, length = c.K.to(DEV), c.V.to(DEV), c.table.to(DEV), c.lens.to(DEV)
    ws = torch.empty(binding.tree_attn_workspace_bytes(3, T, Hq, Hkv, d), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty_like(Q), torch.empty(3, T, Hq, device=DEV)
    step = lambda: binding.pulsar_tree_attn(Q, Kn, Vn, K, V, table, length, parent, out=out, lse_out=lse, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([400, 0, 63], [17, 555, 1], [0, 0, 0]):
        length.copy_(torch.tensor(lens, dtype=torch.int32))
        ws.fill_(255)                                      # nothing in the workspace is kept from call to call
        graph.replay()
        c.lens, c.K, c.V = length.cpu(), K.cpu(), V.cpu()
        R.check(out, lse, R.tree_attn(Q.cpu(), Kn.cpu(), Vn.cpu(), c, parent.cpu()), str(lens))


def test_two_streams_at_once():
    c = R.Cache([3000, 2000], 16, 2, 128, room=4)
    sets, ref = [], []
    for seed in range(2):
        Q, Kn, Vn, parent = drafts(2, 4, 8, 2, 128, seed=seed)
        sets.append([x.to(DEV) for x in (Q, Kn, Vn, c.K, c.V, c.table, c.lens, parent)])
        ref.append(R.tree_attn(Q, Kn, Vn, c, parent))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in sets], []
    for _ in range(20):
        for st, x in zip(streams, sets):
            with torch.cuda.stream(st):
                got.append(binding.pulsar_tree_attn(*x))
    torch.cuda.synchronize()
    for i, (O, LSE) in enumerate(got):
        R.check(O, LSE, ref[i % 2])


def test_what_the_binding_refuses():
    c = R.Cache([40, 40], 16, 2, 64, room=6)
    Q, Kn, Vn, parent = drafts(2, 6, 8, 2, 64)
    good = [x.to(DEV) for x in (Q, Kn, Vn, c.K, c.V, c.table, c.lens, parent)]
    for i, wrong in ((0, good[0][:1]), (0, good[0][:, :5].contiguous()), (0, good[0][..., :32].contiguous()), (1, good[1][:, :5].contiguous()),
                     (2, good[2][:1]), (3, good[3][:, :, :1].contiguous()), (4, good[4][:3].contiguous()), (5, good[5][0]), (6, good[6][:1]),
                     (7, good[7][:, :3].contiguous())):
        args = list(good)
        args[i] = wrong
        with pytest.raises((ValueError, TypeError)):
            binding.pulsar_tree_attn(*args)
    for i in range(8):
        args = list(good)
        args[i] = good[i].float() if i < 5 else good[i].long()
        with pytest.raises(TypeError):
            binding.pulsar_tree_attn(*args)
        args[i] = good[i].cpu()
        with pytest.raises(TypeError):
            binding.pulsar_tree_attn(*args)
    with pytest.raises(TypeError):
        binding.pulsar_tree_attn(good[0].transpose(1, 2), *good[1:])
    with pytest.raises(TypeError):
        binding.pulsar_tree_attn(*good, out=torch.empty(2, 6, 8, 64, dtype=torch.float16, device=DEV))
    with pytest.raises(binding.PulsarError) as e:
        binding.pulsar_tree_attn(*good, workspace=torch.empty(1024, dtype=torch.uint8, device=DEV))
    assert e.value.status == 4


@pytest.mark.parametrize("T,Hq,Hkv,d", [(2, 4, 1, 64), (2, 8, 2, 128), (5, 4, 1, 64), (13, 16, 4, 64), (16, 8, 2, 128), (24, 8, 2, 128),
                                        (30, 4, 1, 64), (64, 8, 2, 64), (40, 16, 1, 128)])
def test_values_that_are_not_finite_reach_who_sees_them(T, Hq, Hkv, d):
    """An infinite component and a NaN one of two nodes' values, in every form that a call can take: the outputs of the nodes that see
    them are what the definition says, component by component, and everybody else's are as if they were not there."""
    c = R.Cache([150, 0], 16, Hkv, d, room=T)
    Q, Kn, Vn, parent = drafts(2, T, Hq, Hkv, d, seed=T)
    Vn[0, 1, :, 3], Vn[1, T // 2, :, d - 1], Vn[1, 0, 0, 5] = float("inf"), float("nan"), float("-inf")
    O, LSE = binding.pulsar_tree_attn(*(x.to(DEV) for x in (Q, Kn, Vn, c.K, c.V, c.table, c.lens, parent)))
    Oref, Lref, A = R.tree_attn(Q, Kn, Vn, c, parent)
    o = O.double().cpu()
    assert torch.equal(o.isnan(), Oref.isnan()) and torch.equal(o.isinf(), Oref.isinf()) and bool((o[o.isinf()] == Oref[o.isinf()]).all())
    fine = Oref.isfinite()
    assert not bool(fine.all())
    zero = torch.zeros_like(Oref)
    R.check(torch.where(fine, o, zero), LSE, (torch.where(fine, Oref, zero), Lref, torch.where(fine, A, zero)))


@pytest.mark.parametrize("T,Hq,Hkv,d", [(1, 8, 2, 128), (6, 8, 2, 128), (13, 16, 4, 64), (24, 8, 2, 128), (64, 8, 2, 64)])
def test_logits_that_rise_by_powers_of_two(T, Hq, Hkv, d):
    """Tiles whose largest logits lie 2^20 to 2^200 above those of the tiles before: what has been summed up so far is rescaled, in the
    middle of a tile and between tiles.  (Keys are multiples of the queries' mean direction, so the logits rise along the cache.)"""
    c = R.Cache([900, 385], 16, Hkv, d, room=T)
    Q, Kn, Vn, parent = drafts(2, T, Hq, Hkv, d, seed=T)
    g = torch.Generator().manual_seed(2)
    u = torch.randn(Hkv, d, generator=g)
    u /= u.norm(dim=-1, keepdim=True)
    Q = (Q.float() * 0.05 + u.repeat_interleave(Hq // Hkv, 0)).to(BF)
    rise = {0: 0.0, 70: 20.0, 200: 45.0, 300: 130.0, 301: 140.0, 500: 230.0, 800: 238.0}
    for s, n in enumerate((900, 385)):
        h = 0.0
        for r in range(n):
            h = rise.get(r, h)
            at = c.table[s, r // 16], r % 16
            c.K[at] = (c.K[at].float() * 0.05 + u * h * 0.6931).to(BF)
    run(c, Q, Kn, Vn, parent, scale=1.0)
