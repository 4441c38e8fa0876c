"""Arguments of the paged cache's calls that are refused on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

import paged_reference as R
from paper_2607_20457_b200 import _build, binding

OK, INVALID, SHAPE, ALIGNMENT, WORKSPACE = 0, 1, 2, 3, 4


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return binding.load_library()


def at(i):
    return ctypes.c_void_p(i << 20)               # never read: validation fails first


def refused(fn, good, **change):
    args = dict(good)
    args.update(change)
    return fn(*args.values())


FORK = dict(table=at(1), len=at(2), n_slots=4, max_pages=8, parent=at(3), n_new=4, K=at(4), V=at(5), layers=2, n_pages=64, page=16,
            Hkv=2, d=64, reserve=1, new_table=at(6), new_len=at(7), n_free=at(8), ws=at(9), ws_bytes=1 << 16, status=None, stream=None)
COMPACT = dict(K=at(4), V=at(5), layers=2, n_pages=64, page=16, Hkv=2, d=64, table=at(1), len=at(2), n_slots=4, max_pages=8, accept=at(3),
               T=4, new_len=at(7), status=None, stream=None)
APPEND = dict(Kn=at(1), Vn=at(2), T=4, n_new=None, K=at(4), V=at(5), n_pages=64, page=16, Hkv=2, d=64, table=at(6), len=at(7), n_slots=4,
              max_pages=8, status=None, stream=None)
SUMMARIZE = dict(K=at(1), layers=1, n_pages=64, page=16, Hkv=2, d=64, table=at(2), begin=None, end=at(3), n_slots=4, max_pages=8,
                 summary=at(4), status=None, stream=None)
TREE = dict(Q=at(1), Kn=at(2), Vn=at(3), T=4, K=at(4), V=at(5), n_pages=64, page=16, table=at(6), len=at(7), n_slots=4, max_pages=8,
            parent=at(8), n_draft=None, Hq=8, Hkv=2, d=64, scale=0.0, O=at(9), f32=0, LSE=None, ws=at(10), ws_bytes=1 << 30, status=None,
            stream=None)
SPARSE = dict(Q=at(1), Kn=at(2), Vn=at(3), T=4, K=at(4), V=at(5), summary=at(11), n_pages=64, page=16, table=at(6), len=at(7), n_slots=4,
              max_pages=8, n_draft=None, k=4, sink=1, window=1, Hq=8, Hkv=2, d=64, scale=0.0, O=at(9), LSE=None, sel=at(12), ws=at(10),
              ws_bytes=1 << 30, status=None, stream=None)
CALLS = {"pulsar_pages_fork": FORK, "pulsar_pages_compact": COMPACT, "pulsar_pages_append": APPEND, "pulsar_pages_summarize": SUMMARIZE,
         "pulsar_tree_attn": TREE, "pulsar_sparse_attn": SPARSE}


@pytest.mark.parametrize("name", CALLS)
def test_shapes_that_no_kernel_covers(lib, name):
    fn, good = getattr(lib, name), CALLS[name]
    for change in (dict(page=8), dict(page=48), dict(page=256), dict(d=96), dict(Hkv=0), dict(n_slots=0), dict(n_slots=1025),
                   dict(max_pages=0), dict(max_pages=(1 << 26) + 1), dict(n_pages=0), dict(n_pages=1 << 24)):
        assert refused(fn, good, **change) == SHAPE, change
    more = {"pulsar_pages_fork": (dict(n_new=0), dict(n_new=1025), dict(reserve=-1), dict(layers=0)),
            "pulsar_pages_compact": (dict(T=0), dict(T=65)), "pulsar_pages_append": (dict(T=-1),),
            "pulsar_pages_summarize": (dict(layers=0), dict(layers=65536), dict(max_pages=1 << 26, n_slots=1, Hkv=1024)), "pulsar_tree_attn": (dict(T=0), dict(T=65), dict(Hq=7), dict(Hq=6), dict(Hq=64)),
            "pulsar_sparse_attn": (dict(T=0), dict(T=65), dict(Hq=7), dict(k=0), dict(k=65537), dict(sink=-1), dict(window=-1),
                                   dict(sink=3, window=2))}[name]
    for change in more:
        assert refused(fn, good, **change) == SHAPE, change


@pytest.mark.parametrize("name", CALLS)
def test_pointers(lib, name):
    fn, good = getattr(lib, name), CALLS[name]
    optional = {"parent", "n_new", "n_draft", "begin", "LSE", "status", "stream"}
    for key, value in good.items():
        if not isinstance(value, ctypes.c_void_p):
            continue
        if key not in optional:
            assert refused(fn, good, **{key: None}) == INVALID, key
        assert refused(fn, good, **{key: ctypes.c_void_p(value.value + 2)}) == ALIGNMENT, key
    if "ws" in good:
        assert refused(fn, good, ws=ctypes.c_void_p(good["ws"].value + 16)) == ALIGNMENT


def test_fork_refuses_results_in_the_place_of_its_inputs(lib):
    for change in (dict(new_table=at(1)), dict(new_len=at(2)), dict(new_len=at(3)), dict(n_free=at(1)),
                   dict(new_table=ctypes.c_void_p((1 << 20) + 4 * 8 * 4 - 4)), dict(parent=None, n_new=3)):
        assert refused(lib.pulsar_pages_fork, FORK, **change) == INVALID, change
    assert refused(lib.pulsar_pages_compact, COMPACT, new_len=at(2)) == INVALID


def test_workspaces(lib):
    size = lib.pulsar_pages_fork_workspace_bytes(4, 64)
    assert size > 64 and refused(lib.pulsar_pages_fork, FORK, ws_bytes=size - 1) == WORKSPACE
    size = lib.pulsar_tree_attn_workspace_bytes(4, 4, 8, 2, 64)
    assert size > 0 and refused(lib.pulsar_tree_attn, TREE, ws_bytes=size - 1) == WORKSPACE
    more = lib.pulsar_sparse_attn_workspace_bytes(4, 4, 8, 4, 8, 2, 64)
    assert more > 0 and refused(lib.pulsar_sparse_attn, SPARSE, ws_bytes=more - 1) == WORKSPACE
    assert lib.pulsar_pages_fork_workspace_bytes(0, 64) == 0 and lib.pulsar_pages_fork_workspace_bytes(4, 1 << 24) == 0
    assert lib.pulsar_tree_attn_workspace_bytes(4, 65, 8, 2, 64) == 0 and lib.pulsar_tree_attn_workspace_bytes(4, 4, 8, 2, 96) == 0
    assert lib.pulsar_sparse_attn_workspace_bytes(4, 4, 8, 0, 8, 2, 64) == 0


def test_binding_refuses_what_is_no_cuda_tensor(lib):
    c = R.Cache([5], 16, 1, 64)
    with pytest.raises(TypeError):
        binding.pulsar_pages_fork(c.table, c.lens, None, c.K[None], c.V[None])
    q = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        binding.pulsar_tree_attn(q, q, q, c.K, c.V, c.table, c.lens)


# ---- the plain forms that the kernels are compared with, on cases that can be worked out by hand ---------------------------------

def test_reference_fork_by_hand():
    table = torch.tensor([[7, 3, 5, -1], [2, 6, -1, -1]], dtype=torch.int32)
    lens = torch.tensor([40, 32], dtype=torch.int32)                       # pages of 16: two and a half, two
    new, new_len, n_free, copies = R.fork(table, lens, [0, 0, 1, -1], 9, 16, 1)
    # slot 0 keeps 5, slot 1 gets a copy in the lowest free page (0), slot 2 is full: one more page (1)
    assert new.tolist() == [[7, 3, 5, -1], [7, 3, 0, -1], [2, 6, 1, -1], [-1] * 4]
    assert new_len.tolist() == [40, 40, 32, 0] and n_free == 2 and copies == [(5, 0, 8)]


def test_reference_tree_and_selection_by_hand():
    assert R.visible([-1, 0, 0, 1], 3) == [3, 1, 0]
    c = R.Cache([0], 16, 1, 64, room=4)
    Q, Kn = torch.zeros(1, 3, 1, 64).to(R.BF), torch.randn(1, 3, 1, 64).to(R.BF)
    Vn = torch.arange(3.).view(1, 3, 1, 1).expand(1, 3, 1, 64).to(R.BF)
    O, LSE, _ = R.tree_attn(Q, Kn, Vn, c, [[-1, -1, 0]])                    # zero queries: the mean over what a node sees
    assert O[0, :, 0, 0].tolist() == [0.0, 1.0, 1.0] and torch.allclose(LSE[0, :, 0].exp(), torch.tensor([1., 1., 2.]).double())
    bounds = torch.zeros(5, 2, 64)
    bounds[:, 1, 0] = torch.tensor([1., 5., 3., 5., 0.])
    q = torch.zeros(2, 64)
    q[0, 0] = 1.
    assert R.select_pages(q, bounds, 5, 2, 0, 0) == [1, 3] and R.select_pages(q, bounds, 5, 1, 0, 0) == [1]
    assert R.select_pages(q, bounds, 5, 3, 1, 1) == [0, 1, 4]


@pytest.mark.parametrize("name,pairs", [
    ("pulsar_pages_fork", [("K", "V")]), ("pulsar_pages_compact", [("K", "V"), ("len", "new_len")]),
    ("pulsar_pages_append", [("K", "V"), ("Kn", "K"), ("Vn", "K"), ("Kn", "V"), ("Vn", "V")]), ("pulsar_pages_summarize", [("K", "summary")]),
    ("pulsar_tree_attn", [("K", "V"), ("O", "Q"), ("O", "Kn"), ("O", "Vn"), ("O", "K"), ("O", "V"), ("Kn", "K"), ("Vn", "V"), ("Q", "K")]),
    ("pulsar_sparse_attn", [("K", "V"), ("O", "Q"), ("O", "Kn"), ("O", "Vn"), ("O", "K"), ("O", "V"), ("Kn", "K"), ("Vn", "V"), ("Q", "V"),
                            ("summary", "K"), ("O", "summary"), ("sel", "O"), ("sel", "Q")])])
def test_tensors_that_share_memory(lib, name, pairs):
    fn, good = getattr(lib, name), CALLS[name]
    for one, other in pairs:
        for change in (good[other], ctypes.c_void_p(good[other].value + 256)):       # the same place, and a part of it
            if one in ("len",) and change is not good[other]:
                continue
            assert refused(fn, good, **{one: change}) == INVALID, (one, other)


# Every tensor of a call with what it takes up: (bytes, whether the call writes it).
POOL, TABLE, SLOTS = 64 * 16 * 2 * 64 * 2, 4 * 8 * 4, 4 * 4
FRESH, QUERY, SUMMARY = 16 * 2 * 64 * 2, 16 * 8 * 64 * 2, 64 * 2 * 2 * 64 * 2
ALL = {
    "pulsar_pages_fork": dict(K=(2 * POOL, 1), V=(2 * POOL, 1), new_table=(TABLE, 1), new_len=(SLOTS, 1), n_free=(4, 1), status=(4, 1),
                              table=(TABLE, 0), len=(SLOTS, 0), parent=(SLOTS, 0)),
    "pulsar_pages_compact": dict(K=(2 * POOL, 1), V=(2 * POOL, 1), new_len=(SLOTS, 1), status=(4, 1), table=(TABLE, 0), len=(SLOTS, 0),
                                 accept=(64, 0)),
    "pulsar_pages_append": dict(K=(POOL, 1), V=(POOL, 1), status=(4, 1), Kn=(FRESH, 0), Vn=(FRESH, 0), n_new=(SLOTS, 0), table=(TABLE, 0),
                                len=(SLOTS, 0)),
    "pulsar_pages_summarize": dict(summary=(SUMMARY, 1), status=(4, 1), K=(POOL, 0), table=(TABLE, 0), begin=(SLOTS, 0), end=(SLOTS, 0)),
    "pulsar_tree_attn": dict(O=(QUERY, 1), K=(POOL, 1), V=(POOL, 1), LSE=(512, 1), status=(4, 1), Q=(QUERY, 0), Kn=(FRESH, 0), Vn=(FRESH, 0),
                             table=(TABLE, 0), len=(SLOTS, 0), parent=(64, 0), n_draft=(SLOTS, 0)),
    "pulsar_sparse_attn": dict(O=(QUERY, 1), K=(POOL, 1), V=(POOL, 1), LSE=(512, 1), sel=(512, 1), status=(4, 1), Q=(QUERY, 0), Kn=(FRESH, 0),
                               Vn=(FRESH, 0), summary=(SUMMARY, 0), table=(TABLE, 0), len=(SLOTS, 0), n_draft=(SLOTS, 0)),
}


@pytest.mark.parametrize("name", ALL)
def test_nothing_that_is_written_shares_memory_with_anything(lib, name):
    """Whatever a call writes, beside every other tensor of it: at the same place, at its last word, and with its own last word at the
    other's first; and one word further off, where it is the workspace or the alignment that is refused."""
    fn, tensors = getattr(lib, name), ALL[name]
    good = dict(CALLS[name])
    for i, key in enumerate(tensors):
        good[key] = at(20 + 2 * i)
    if "ws" in good:
        good["ws"], good["ws_bytes"] = at(200), 1 << 30
    place = lambda base, by: ctypes.c_void_p(good[base].value + by)
    # (an odd address or a workspace of no bytes ends a call behind these checks)
    last = dict(ws_bytes=0) if "ws" in good else dict(len=place("len", 2)) if "len" in good else dict(end=place("end", 2))
    assert refused(fn, good, **last) == (WORKSPACE if "ws" in good else ALIGNMENT)
    for one, (size, written) in tensors.items():
        if not written:
            continue
        for other, (other_size, _) in tensors.items():
            if other == one:
                continue
            for by in {0, other_size - 4, 4 - size}:
                assert refused(fn, good, **{one: place(other, by)}) == INVALID, (one, other, by)
            for by in (other_size, -size):
                if other not in last and one not in last:
                    assert refused(fn, good, **{one: place(other, by)}, **last) in (WORKSPACE, ALIGNMENT), (one, other, by)
    if "ws" in good:
        for other, (size, _) in tensors.items():
            assert refused(fn, good, ws=ctypes.c_void_p(good[other].value // 256 * 256)) == INVALID, other
            good_ws = dict(good, ws=at(19), ws_bytes=1 << 30)
            assert refused(fn, good_ws, **{other: ctypes.c_void_p(at(19).value + 256)}) == INVALID, other
