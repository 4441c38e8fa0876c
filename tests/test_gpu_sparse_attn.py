"""GPU parity: attention over the pages that each query selects, against its definition in 64 bits; the selection is exact."""
import pytest
import torch

import paged_reference as R
from paper_2607_20457_b200 import binding
from test_gpu_tree_attn import drafts

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def run(c, Q, Kn, Vn, k, sink=0, window=0, n_draft=None, scale=0.0, bounds=None, expect=0, what=""):
    S, T, Hq, d = Q.shape
    Hkv = Kn.shape[2]
    K, V = c.K.to(DEV), c.V.to(DEV)
    bounds = R.page_bounds(c.K) if bounds is None else bounds
    status = binding.new_status(DEV)
    out, lse = torch.full(Q.shape, 77.0, dtype=BF, device=DEV), torch.full((S, T, Hq), 77.0, device=DEV)
    sel = torch.full((S, T, Hkv, k), 77, dtype=torch.int32, device=DEV)
    nd = None if n_draft is None else torch.tensor(n_draft, dtype=torch.int32, device=DEV)
    binding.pulsar_sparse_attn(Q.to(DEV), Kn.to(DEV), Vn.to(DEV), K, V, bounds.to(DEV), c.table.to(DEV), c.lens.to(DEV), k, sink, window, nd,
                               scale, out=out, lse_out=lse, sel_out=sel, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == expect
    counts = [T] * S if n_draft is None else [min(max(n, 0), T) for n in n_draft]
    O, LSE, A, want = R.sparse_attn(Q, Kn, Vn, c, bounds, k, sink, window, counts, scale or None)
    used = torch.arange(T) < torch.tensor(counts)[:, None]
    assert torch.equal(sel.cpu()[used], want[used]), what
    for x in (out, lse, sel):
        assert bool((x.cpu()[~used] == 77).all())
    if used.any():
        R.check(out.cpu()[used], lse.cpu()[used], (O[used], LSE[used], A[used]), what)
    for x, new, old in ((K, Kn, c.K.clone()), (V, Vn, c.V.clone())):
        for s in range(S):
            r = int(c.lens[s]) + torch.arange(counts[s])
            old[c.table[s].long()[r // c.page], r % c.page] = new[s, :counts[s]]
        assert torch.equal(x.cpu().view(torch.int16), old.view(torch.int16))
    return sel


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 1), (4, 4), (4, 2), (16, 2), (16, 1)])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_heads_pages_and_lengths(d, Hq, Hkv, page):
    lens = [0, 1, page - 1, page, 3 * page, 9 * page + 3, 12 * page - 1, 20 * page + 16]
    for T, k, sink, window in ((1, 4, 1, 1), (3, 3, 0, 0), (2, 6, 2, 4)):
        c = R.Cache(lens, page, Hkv, d, room=T, seed=k)
        run(c, *drafts(len(lens), T, Hq, Hkv, d, seed=T)[:3], k, sink, window, what=f"T={T} k={k}")


@pytest.mark.parametrize("k,sink,window", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (7, 0, 0), (64, 3, 5), (400, 10, 10)])
def test_many_pages(k, sink, window):
    c = R.Cache([16 * 700 + 5, 16 * 64, 16 * 65], 16, 2, 64, room=2)
    run(c, *drafts(3, 2, 8, 2, 64)[:3], k, sink, window)


def test_equal_scores_go_to_the_lower_page():
    c = R.Cache([16 * 90 + 3, 16 * 40], 16, 1, 64, room=1)
    bounds = torch.zeros(c.n_pages, 1, 2, 64)
    g = torch.Generator().manual_seed(1)
    bounds[:, 0, 1, 0] = torch.randint(0, 3, (c.n_pages,), generator=g).float()    # three scores only
    Q, Kn, Vn, _ = drafts(2, 1, 2, 1, 64)
    Q[...] = 0
    Q[..., 0] = 1
    with pytest.raises(binding.PulsarError):                # a page for each of three forced ones is asked for
        run(c, Q, Kn, Vn, 1, 1, 2, bounds=bounds.to(BF))
    for k in (1, 5, 33):
        run(c, Q, Kn, Vn, k, min(k - 1, 1), min(k - 1, 2), bounds=bounds.to(BF))
    Q[...] = 0                                              # all equal
    run(c, Q, Kn, Vn, 5, bounds=bounds.to(BF))


def test_scores_next_to_each_other_are_told_apart():
    """Page scores that differ in the 40th bit only: the sum of a large product and a small one."""
    c = R.Cache([16 * 60], 16, 1, 64, room=1)
    bounds = torch.zeros(c.n_pages, 1, 2, 64)
    bounds[:, 0, :, 0] = 256.0
    g = torch.Generator().manual_seed(2)
    for o, x in enumerate(torch.randperm(60, generator=g).tolist()):
        bounds[c.table[0, o], 0, :, 1] = (x + 1) * 2.0 ** -32
    Q, Kn, Vn, _ = drafts(1, 1, 1, 1, 64)
    Q[...] = 0
    Q[..., :2] = 1
    run(c, Q, Kn, Vn, 9, bounds=bounds.to(BF))


def test_bounds_that_are_infinite_or_no_numbers():
    c = R.Cache([16 * 30], 16, 1, 64, room=1)
    bounds = R.page_bounds(torch.where(c.K.isnan(), torch.zeros_like(c.K), c.K))
    t = c.table[0].long()
    bounds[t[3], 0, :, 5] = float("nan")
    bounds[t[4], 0, 1, 6], bounds[t[4], 0, 0, 6] = float("inf"), float("inf")
    bounds[t[5], 0, 0, 7], bounds[t[5], 0, 1, 7] = float("-inf"), float("-inf")
    Q, Kn, Vn, _ = drafts(1, 1, 4, 1, 64)
    Q[0, 0, :, 6], Q[0, 0, :, 7] = 1.0, 1.0
    sel = run(c, Q, Kn, Vn, 8, bounds=bounds).cpu()[0, 0, 0].tolist()
    assert 4 in sel and 3 not in sel and 5 not in sel
    run(c, Q, Kn, Vn, 29, bounds=bounds)


def test_slots_with_fewer_tokens_or_none():
    c = R.Cache([200, 0, 64, 333], 16, 2, 64, room=6)
    run(c, *drafts(4, 6, 8, 2, 64)[:3], 4, 1, 1, n_draft=[6, 3, 0, 1])
    run(c, *drafts(4, 6, 8, 2, 64)[:3], 4, 1, 1, n_draft=[0, 0, 0, 0])


def test_tokens_at_the_most():
    c = R.Cache([200, 777], 16, 1, 64, room=64)
    run(c, *drafts(2, 64, 2, 1, 64)[:3], 5, 1, 1)


def test_all_pages_selected_is_the_whole_cache():
    c = R.Cache([333, 1000], 32, 2, 128, room=1)
    Q, Kn, Vn, _ = drafts(2, 1, 8, 2, 128)
    args = [x.to(DEV) for x in (Q, Kn, Vn, c.K, c.V)]
    bounds = R.page_bounds(c.K).to(DEV)
    O, LSE, sel = binding.pulsar_sparse_attn(*args, bounds, c.table.to(DEV), c.lens.to(DEV), 40)
    O2, LSE2 = binding.pulsar_tree_attn(*args, c.table.to(DEV), c.lens.to(DEV))
    assert float((O.float() - O2.float()).abs().max()) <= 1e-2 and float((LSE - LSE2).abs().max()) <= 2e-5
    assert sel[0, 0, 0].cpu().tolist() == list(range(10)) + [-1] * 30


def test_bad_pages_are_reported():
    c = R.Cache([16 * 20 + 4], 16, 1, 64, room=1)
    bounds = R.page_bounds(c.K).to(DEV)
    table = c.table.clone()
    table[0, 7], table[0, 0] = -1, c.n_pages
    Q, Kn, Vn, _ = drafts(1, 1, 4, 1, 64)
    for sink in (0, 1):                                     # ranked last, or selected all the same: its rows count as absent
        status = binding.new_status(DEV)
        O, _, sel = binding.pulsar_sparse_attn(*(x.to(DEV) for x in (Q, Kn, Vn, c.K, c.V)), bounds, table.to(DEV), c.lens.to(DEV), 6, sink,
                                               status=status)
        assert int(status.item()) == binding.DEV_BAD_PAGE and bool(O.isfinite().all())
        assert (0 in sel.cpu().flatten().tolist()) == (sink == 1) and 7 not in sel.cpu().flatten().tolist()


def test_captured_step_follows_the_lengths_on_the_device():
    T, Hq, Hkv, d, k = 2, 8, 2, 64, 5
    c = R.Cache([500, 100], 16, Hkv, d, room=600)
    for x in (c.K, c.V):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(8)).to(BF))
    bounds = R.page_bounds(c.K)
    Q, Kn, Vn, _ = (x.to(DEV) for x in drafts(2, T, Hq, Hkv, d))
    K, V, B, table, length = (x.to(DEV) for x in (c.K, c.V, bounds, c.table, c.lens))
    ws = torch.empty(binding.sparse_attn_workspace_bytes(2, T, c.max_pages, k, Hq, Hkv, d), dtype=torch.uint8, device=DEV)
    out, lse, sel = torch.empty_like(Q), torch.empty(2, T, Hq, device=DEV), torch.empty(2, T, Hkv, k, dtype=torch.int32, device=DEV)
    step = lambda: binding.pulsar_sparse_attn(Q, Kn, Vn, K, V, B, table, length, k, 1, 1, out=out, lse_out=lse, sel_out=sel, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([500, 100], [17, 1055], [0, 79]):
        length.copy_(torch.tensor(lens, dtype=torch.int32))
        ws.fill_(255)
        graph.replay()
        c.lens, c.K, c.V = length.cpu(), K.cpu(), V.cpu()
        O, LSE, A, want = R.sparse_attn(Q.cpu(), Kn.cpu(), Vn.cpu(), c, bounds, k, 1, 1)
        assert torch.equal(sel.cpu(), want)
        R.check(out, lse, (O, LSE, A), str(lens))


def test_scores_that_are_equal_infinite_or_far_apart_everywhere():
    """What the fp32 scores cannot tell: all equal, more equal ones at the border than are kept at hand, and sizes beyond fp32."""
    c = R.Cache([16 * 900 + 1], 16, 1, 64, room=1)
    Q, Kn, Vn, _ = drafts(1, 1, 4, 1, 64)
    g = torch.Generator().manual_seed(5)
    bounds = R.page_bounds(torch.where(c.K.isnan(), torch.zeros_like(c.K), c.K))
    run(c, Q, Kn, Vn, 40, 1, 1, bounds=torch.ones_like(bounds))
    two = torch.where(torch.rand(c.n_pages, 1, 1, 1, generator=g) < 0.5, 1.0, 0.0).expand_as(bounds).to(BF).contiguous()
    run(c, Q, Kn, Vn, 700, 0, 3, bounds=two)
    huge = (bounds.float() * 1e37).to(BF)
    run(c, (Q.float() * 1e3).to(BF), Kn, Vn, 33, bounds=huge, scale=1e-6)
    tiny = (bounds.float() * 1e-38).to(BF)
    run(c, Q, Kn, Vn, 33, bounds=tiny)
    some = bounds.clone()
    some[c.table[0, 7:300:13].long()] = float("nan")
    run(c, Q, Kn, Vn, 33, 2, 2, bounds=some)


@pytest.mark.parametrize("T,Hq,Hkv", [(40, 8, 2), (9, 16, 1), (33, 1, 1)])
def test_more_query_rows_than_a_tile(T, Hq, Hkv):
    c = R.Cache([16 * 80 + 9, 16 * 130], 16, Hkv, 128, room=T)
    run(c, *drafts(2, T, Hq, Hkv, 128)[:3], 7, 1, 2)


def test_more_pages_than_a_thread_block_holds():
    c = R.Cache([16 * 5000 + 3], 16, 1, 64, room=1)
    run(c, *drafts(1, 1, 2, 1, 64)[:3], 50, 1, 2)
