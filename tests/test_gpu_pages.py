"""GPU parity: fork, compact, append and summarise on a paged cache against their definitions."""
import pytest
import torch

import paged_reference as R
from paper_2607_20457_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def bits(x):
    return x.cpu().view(torch.int16)


def run_fork(c, parent, reserve, table=None, expect=0):
    table = c.table if table is None else table
    K, V = c.K.to(DEV), c.V.to(DEV)
    status = binding.new_status(DEV)
    par = None if parent is None else torch.tensor(parent, dtype=torch.int32, device=DEV)
    got = binding.pulsar_pages_fork(table.to(DEV), c.lens.to(DEV), par, K, V, reserve, status=status)
    new, new_len, n_free, copies = R.fork(table, c.lens, parent, c.n_pages, c.page, reserve)
    assert int(status.item()) == expect
    assert torch.equal(got[0].cpu(), new) and torch.equal(got[1].cpu(), new_len) and int(got[2].item()) == n_free
    for x, ref in ((K, c.K.clone()), (V, c.V.clone())):
        for src, dst, rows in copies:
            ref[:, dst, :rows] = ref[:, src, :rows]
        assert torch.equal(bits(x), bits(ref))
    return got


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("Hkv,d,n_layers", [(2, 64, 3), (1, 128, 1), (8, 128, 2)])
@pytest.mark.parametrize("reserve", [0, 1, 70])
def test_fork_shares_copies_and_reserves(page, Hkv, d, n_layers, reserve):
    lens = [0, 1, page - 1, page, page + 1, 3 * page + 5]
    c = R.Cache(lens, page, Hkv, d, room=page + 80, n_layers=n_layers, spare=60)
    for parent in (None, [5, 5, 1, -1, 3, 3, 5, 2, 4, 0], [1], [4] * 12, [-1, -1], [0, 1, 2, 3, 4, 5]):
        run_fork(c, parent, reserve)


def test_fork_of_slots_that_share_a_context():
    c = R.Cache([100, 97, 128, 96], 32, 2, 64, room=40, n_layers=2, shared=96, spare=9)
    run_fork(c, [0, 0, 1, 2, 2, 3, 3, -1, 0], 10)


def test_pages_of_dropped_slots_are_handed_out_in_the_same_call():
    c = R.Cache([64, 64, 64], 16, 1, 64, n_layers=1, room=64, spare=0)
    table = c.table.clone()
    table[:, 4:] = -1
    run_fork(c, [0, 0], 48, table=table)                 # 12 of 24 pages were live; 4 + 4 shared, 3 + 3 new ones


def test_fork_many_slots_and_wide_tables():
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 2600, (70,), generator=g).tolist()
    c = R.Cache(lens, 16, 1, 64, n_layers=1, room=30, spare=500)
    run_fork(c, torch.randint(-1, 70, (150,), generator=g).tolist(), 17)
    lens = [20000, 40, 0, 16399]                         # more entries than a CTA has threads
    c = R.Cache(lens, 16, 1, 64, n_layers=1, room=30, spare=70000)
    run_fork(c, [3, 0, 0, 1, 3], 100 - 70, )


def test_fork_without_enough_pages_or_room():
    c = R.Cache([20, 20], 16, 1, 64, n_layers=1, room=100, spare=0)
    new, *_ = run_fork(c, [0] * 14, 16, expect=binding.DEV_NO_PAGES)
    assert int((new == -1).sum()) > 0
    c = R.Cache([20, 30], 16, 1, 64, n_layers=1, spare=9)            # two entries per slot
    run_fork(c, [0, 1], 13, expect=binding.DEV_NO_PAGES)


def test_fork_with_bad_entries():
    c = R.Cache([40, 40, 33], 16, 1, 64, n_layers=1, spare=5)
    table = c.table.clone()
    table[1, 0], table[2, 2] = -7, c.n_pages
    run_fork(c, [0, 1, 2, 2], 3, table=table, expect=binding.DEV_BAD_PAGE)
    run_fork(c, [0, 3, -2, 1], 0, expect=binding.DEV_BAD_TREE)
    c.lens[1] = 1000
    par = torch.tensor([1], dtype=torch.int32, device=DEV)
    status = binding.new_status(DEV)
    _, length, _ = binding.pulsar_pages_fork(c.table.to(DEV), c.lens.to(DEV), par, c.K.to(DEV), c.V.to(DEV), status=status)
    assert int(status.item()) == binding.DEV_BAD_LENGTH and int(length.item()) == 48


@pytest.mark.parametrize("page,Hkv,d,n_layers", [(16, 2, 64, 3), (64, 8, 128, 2), (128, 1, 128, 1), (32, 5, 64, 2)])
def test_compact(page, Hkv, d, n_layers):
    T = 64
    lists = [[0, 1, 2], [63], [1, 2, 3, 4], list(range(64)), [], list(range(0, 64, 2)), [0, 2, 3, 40, 62], list(range(1, 64)), [5]]
    lens = [0, 1, page - 1, page, 7, 3 * page - 3, 50, 2 * page + 1, 31]
    c = R.Cache(lens, page, Hkv, d, room=T, n_layers=n_layers)
    gen = torch.Generator().manual_seed(1)
    for x in (c.K, c.V):
        x.copy_(torch.randn(x.shape, generator=gen).to(BF))
    accept = torch.full((len(lens), T), -1, dtype=torch.int32)
    for s, l in enumerate(lists):
        accept[s, :len(l)] = torch.tensor(l, dtype=torch.int32)
    K, V, status = c.K.to(DEV), c.V.to(DEV), binding.new_status(DEV)
    new_len = binding.pulsar_pages_compact(K, V, c.table.to(DEV), c.lens.to(DEV), accept.to(DEV), status=status)
    assert int(status.item()) == 0
    assert new_len.cpu().tolist() == [n + len(l) for n, l in zip(lens, lists)]
    for x, ref in ((K, c.K), (V, c.V)):
        want = ref.clone()
        for s, l in enumerate(lists):
            at = lambda r: (c.table[s].long()[r // page], r % page)
            for j, a in enumerate(l):
                (p0, o0), (p1, o1) = at(lens[s] + a), at(lens[s] + j)
                want[:, p1, o1] = ref[:, p0, o0]
        assert torch.equal(bits(x), bits(want))


def test_compact_of_lists_that_are_none():
    c = R.Cache([10, 10, 10, 10], 16, 1, 64, room=8, n_layers=1)
    accept = torch.tensor([[1, 1, -1, -1], [2, -1, 3, -1], [4, -1, -1, -1], [1, 3, -5, -1]], dtype=torch.int32)
    status = binding.new_status(DEV)
    K, V = c.K.to(DEV), c.V.to(DEV)
    new_len = binding.pulsar_pages_compact(K, V, c.table.to(DEV), c.lens.to(DEV), accept.to(DEV), status=status)
    assert int(status.item()) == binding.DEV_BAD_TREE and new_len.cpu().tolist() == [11, 11, 10, 12]
    c.table[0, 0] = -1
    status = binding.new_status(DEV)
    accept = torch.tensor([[3, -1], [-1, -1], [-1, -1], [0, 1]], dtype=torch.int32)
    binding.pulsar_pages_compact(K, V, c.table.to(DEV), c.lens.to(DEV), accept.to(DEV), status=status)
    assert int(status.item()) == binding.DEV_BAD_TREE      # node 3 of a tree of two: nothing moves


def test_compact_where_a_page_is_missing():
    c = R.Cache([10, 10], 16, 1, 64, room=8, n_layers=1)
    c.table[0, 0] = -1
    K, V, status = c.K.to(DEV), c.V.to(DEV), binding.new_status(DEV)
    accept = torch.tensor([[1, 3, -1, -1], [-1] * 4], dtype=torch.int32)
    new_len = binding.pulsar_pages_compact(K, V, c.table.to(DEV), c.lens.to(DEV), accept.to(DEV), status=status)
    assert int(status.item()) == binding.DEV_BAD_PAGE and new_len.cpu().tolist() == [12, 10]
    assert torch.equal(bits(K), bits(c.K)) and torch.equal(bits(V), bits(c.V))


@pytest.mark.parametrize("page,Hkv,d", [(16, 2, 64), (128, 8, 128), (32, 3, 128)])
def test_append(page, Hkv, d):
    lens, T = [0, 5, page, 2 * page - 1], 3 * page + 7
    c = R.Cache(lens, page, Hkv, d, room=T)
    gen = torch.Generator().manual_seed(2)
    Kn, Vn = (torch.randn(4, T, Hkv, d, generator=gen).to(BF) for _ in range(2))
    for n_new in (None, [T, 0, 1, T - 1]):
        K, V, status = c.K.to(DEV), c.V.to(DEV), binding.new_status(DEV)
        n_d = None if n_new is None else torch.tensor(n_new, dtype=torch.int32, device=DEV)
        binding.pulsar_pages_append(Kn.to(DEV), Vn.to(DEV), K, V, c.table.to(DEV), c.lens.to(DEV), n_d, status=status)
        assert int(status.item()) == 0
        for x, new, ref in ((K, Kn, c.K.clone()), (V, Vn, c.V.clone())):
            for s in range(4):
                r = torch.arange(T if n_new is None else n_new[s])
                row = lens[s] + r
                ref[c.table[s].long()[row // page], row % page] = new[s, r]
            assert torch.equal(bits(x), bits(ref))
    status = binding.new_status(DEV)                       # rows past the table are dropped
    full = torch.full((4,), c.max_pages * page - 1, dtype=torch.int32, device=DEV)
    binding.pulsar_pages_append(Kn.to(DEV), Vn.to(DEV), K, V, c.table.to(DEV), full, status=status)
    assert int(status.item()) == binding.DEV_BAD_LENGTH


@pytest.mark.parametrize("page,Hkv,d,n_layers", [(16, 2, 64, 3), (128, 8, 128, 1), (32, 5, 128, 2), (64, 1, 64, 1)])
def test_summarize(page, Hkv, d, n_layers):
    lens = [0, page - 1, page, 5 * page + 3, 3 * page]
    c = R.Cache(lens, page, Hkv, d, n_layers=n_layers)
    c.K[0, c.table[4, 1], 3, 0, 5] = float("nan")
    c.K[0, c.table[3, 2], 0, 0, 7] = float("inf")
    before = torch.randn(n_layers, c.n_pages, Hkv, 2, d).to(BF)
    for begin in (None, [0, 0, 1, 2 * page + 1, 3 * page]):
        S, status = before.to(DEV), binding.new_status(DEV)
        b = None if begin is None else torch.tensor(begin, dtype=torch.int32, device=DEV)
        binding.pulsar_pages_summarize(c.K.to(DEV), c.table.to(DEV), b, c.lens.to(DEV), S, status=status)
        assert int(status.item()) == 0
        want = before.clone()
        for s, n in enumerate(lens):
            for o in range((begin[s] if begin else 0) // page, n // page):
                p = int(c.table[s, o])
                for layer in range(n_layers):
                    want[layer, p] = R.page_bounds(c.K[layer, p:p + 1])[0]
        got = S.cpu()
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(got[~got.isnan()], want[~want.isnan()])


def test_pages_calls_are_captured_and_replayed():
    """A step of a serving loop (compact, fork with reserved pages, summarise) recorded once; replays follow the device's tables."""
    lens = [30, 47, 16, 5]
    c = R.Cache(lens, 16, 2, 64, room=64, n_layers=2, spare=40)
    K, V, table, length = c.K.to(DEV), c.V.to(DEV), c.table.to(DEV), c.lens.to(DEV)
    parent = torch.tensor([0, 0, 1, 3], dtype=torch.int32, device=DEV)
    accept = torch.tensor([[0, 2, -1], [1, -1, -1], [-1, -1, -1], [0, 1, 2]], dtype=torch.int32, device=DEV)
    S = torch.zeros(2, c.n_pages, 2, 2, 64, dtype=BF, device=DEV)
    mid = torch.empty_like(length)
    out = (torch.empty_like(table), torch.empty_like(length), torch.empty(1, dtype=torch.int32, device=DEV))
    ws = torch.empty(binding.load_library().pulsar_pages_fork_workspace_bytes(4, c.n_pages), dtype=torch.uint8, device=DEV)

    def step():
        binding.pulsar_pages_compact(K, V, table, length, accept, out=mid)
        binding.pulsar_pages_fork(table, mid, parent, K, V, 20, out=out, workspace=ws)
        binding.pulsar_pages_summarize(K, out[0], None, out[1], S)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for parents in ([0, 0, 1, 3], [3, 2, 2, 2]):
        for x, y in ((K, c.K), (V, c.V)):
            x.copy_(y)
        parent.copy_(torch.tensor(parents, dtype=torch.int32))
        graph.replay()
        got = [x.clone() for x in (K, V, S, *out)]
        for x, y in ((K, c.K), (V, c.V)):
            x.copy_(y)
        step()
        for x, y in zip(got, (K, V, S, *out)):
            assert torch.equal(x.view(torch.int16) if x.dtype == BF else x, y.view(torch.int16) if y.dtype == BF else y)
