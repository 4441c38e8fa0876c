"""GPU parity: values and keys that are not finite, in the rows of a paged cache and in new tokens, in every form that an attention call
can take (16, 32 and 64 rows per KV head, 128, 256, selected pages)."""
import pytest
import torch

import paged_reference as R
from paper_2607_20457_b200 import binding
from test_gpu_tree_attn import drafts

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")
FORMS = [(1, 8, 2, 128), (3, 4, 1, 64), (5, 8, 2, 128), (13, 16, 4, 64), (16, 8, 2, 128), (24, 8, 2, 128), (30, 4, 1, 64), (64, 8, 2, 64)]


def plant(c, s, row, comp, value, x=None, head=slice(None)):
    x = c.V if x is None else x
    x[c.table[s, row // c.page], row % c.page, head, comp] = value


def agrees(O, LSE, ref):
    """Infinities and NaN of the definition, component by component; what is finite within the usual bounds.  Every weight here is
    above 2^-100, so that its 32 bits are not zero."""
    Oref, Lref, A = ref[:3]
    o = O.double().cpu()
    fine = Oref.isfinite()
    assert not bool(fine.all())
    assert torch.equal(o.isnan(), Oref.isnan()) and torch.equal(o.isinf(), Oref.isinf()) and bool((o[o.isinf()] == Oref[o.isinf()]).all())
    zero = torch.zeros_like(Oref)
    R.check(torch.where(fine, o, zero), LSE, (torch.where(fine, Oref, zero), Lref, torch.where(fine, A, zero)))


def tree(c, Q, Kn, Vn, parent, scale=0.0):
    return binding.pulsar_tree_attn(*(x.to(DEV) for x in (Q, Kn, Vn, c.K, c.V, c.table, c.lens, parent)), softmax_scale=scale)


@pytest.mark.parametrize("T,Hq,Hkv,d", FORMS)
def test_cached_values(T, Hq, Hkv, d):
    """Everybody sees the cached rows: one infinity is an infinity of its sign, two of either sign or a NaN are a NaN."""
    c = R.Cache([150, 40, 0, 129], 16, Hkv, d, room=T)
    Q, Kn, Vn, parent = drafts(4, T, Hq, Hkv, d, seed=T)
    plant(c, 0, 7, 3, INF)
    plant(c, 0, 130, 9, -INF)
    plant(c, 0, 20, 11, NAN)
    plant(c, 0, 5, 12, INF)
    plant(c, 0, 140, 12, -INF)
    plant(c, 1, 39, 0, INF, head=Hkv - 1)
    plant(c, 3, 128, d - 1, -INF)
    agrees(*tree(c, Q, Kn, Vn, parent), R.tree_attn(Q, Kn, Vn, c, parent))


@pytest.mark.parametrize("T,Hq,Hkv,d", [(1, 8, 2, 128), (2, 8, 1, 64), (3, 16, 1, 64)])
def test_cached_values_of_items_that_one_thread_block_has(T, Hq, Hkv, d):
    c = R.Cache([60] * 170, 16, Hkv, d, room=T)
    Q, Kn, Vn, parent = drafts(170, T, Hq, Hkv, d)
    for s in range(0, 170, 3):
        plant(c, s, s % 60, s % d, INF if s % 2 else -INF)
    agrees(*tree(c, Q, Kn, Vn, parent), R.tree_attn(Q, Kn, Vn, c, parent))


@pytest.mark.parametrize("T,Hq,Hkv,d", [(1, 8, 4, 128), (13, 16, 4, 64), (24, 8, 2, 128)])
def test_cached_values_where_the_maximum_moves(T, Hq, Hkv, d):
    """The infinity has been summed up when larger logits come: it is rescaled with the rest."""
    n = 6000
    c = R.Cache([n], 32, Hkv, d, room=T)
    Q, Kn, Vn, parent = drafts(1, T, Hq, Hkv, d)
    g = torch.Generator().manual_seed(3)
    u = torch.randn(Hkv, d, generator=g)
    u /= u.norm(dim=-1, keepdim=True)
    Q = (Q.float() * 0.05 + u.repeat_interleave(Hq // Hkv, 0)).to(R.BF)
    for r in range(n):                                      # logits 9 log2 units up in each of the last five tiles
        at = c.table[0, r // 32], r % 32
        c.K[at] = (c.K[at].float() * 0.05 + u * 9 * 0.6931 * max(0, r // 128 - 42)).to(R.BF)
    plant(c, 0, 5500, 2, INF)
    plant(c, 0, 5770, 4, -INF)
    agrees(*tree(c, Q, Kn, Vn, parent, 1.0), R.tree_attn(Q, Kn, Vn, c, parent, scale=1.0))


@pytest.mark.parametrize("T,Hq,Hkv,d", [(1, 8, 2, 128), (3, 4, 1, 64), (2, 16, 1, 128)])
@pytest.mark.parametrize("k", [6, 40])
def test_values_of_selected_pages(T, Hq, Hkv, d, k):
    """Cached values, those of the rows after the last full page and those of new tokens."""
    c = R.Cache([16 * 20 + 5, 16 * 9, 7], 16, Hkv, d, room=T)
    Q, Kn, Vn, _ = drafts(3, T, Hq, Hkv, d, seed=k)
    for b in range(20):
        plant(c, 0, 16 * b + b % 16, b, INF if b % 2 else -INF)
    plant(c, 0, 16 * 20 + 2, 30, -INF)
    plant(c, 1, 16 * 8 + 3, 31, NAN)
    plant(c, 2, 0, d - 1, INF)
    Vn[2, T - 1, :, 5] = INF
    bounds = R.page_bounds(c.K)
    O, LSE, sel = binding.pulsar_sparse_attn(*(x.to(DEV) for x in (Q, Kn, Vn, c.K, c.V, bounds, c.table, c.lens)), k, 1, 2)
    *ref, want = R.sparse_attn(Q, Kn, Vn, c, bounds, k, 1, 2)
    assert torch.equal(sel.cpu(), want)
    agrees(O, LSE, ref)


def close(O, LSE, ref, rows, rounded=False):
    """Within what the weights' roundings and fp32 sums leave, for queries of a quarter (so that the products of a logit add up to less than
    3 in magnitude after scaling): 2^-16 of A = softmax of |V| up to 64 rows per KV head, R.U of A with more.  fp32: a logit is a sum of up
    to 128 products, off by less than 128 * 2^-23 * 3 = 4.6e-5, and so are two of them in a weight; the sums over up to 128 rows by
    as little; 2e-4 of A covers them."""
    Oref, Lref, A = ref[:3]
    bound = (2.0 ** -16 if rows <= 64 else R.U) * A + 2e-4 * A + 1e-6 + (R.U * Oref.abs() if rounded else 0)
    err = (O.double().cpu() - Oref).abs()
    assert bool((err <= bound).all()), f"{float((err / bound).max()):.2f} of the bound"
    assert float((LSE.double().cpu() - Lref).abs().max()) <= 2e-4


@pytest.mark.parametrize("T,Hq,Hkv,d", [f for f in FORMS if f[0] > 1])
def test_finite_components_beside_one_that_is_not(T, Hq, Hkv, d):
    """A node's value with an infinity in one component: the others count with their full weight, to float32 outputs.  Up to 64 rows
    per KV head a weight is two bf16 numbers, within 2^-16 of itself; with more rows it is one, within R.U."""
    c = R.Cache([6, 20], 16, Hkv, d, room=T)
    Q, Kn, Vn, parent = drafts(2, T, Hq, Hkv, d, seed=T, scale=0.25)
    Vn[0, 1, :, 3], Vn[1, 0, :, d - 1], Vn[1, T // 2, 0, 7] = INF, -INF, NAN
    out = torch.empty(2, T, Hq, d, device=DEV)
    O, LSE = binding.pulsar_tree_attn(*(x.to(DEV) for x in (Q, Kn, Vn, c.K, c.V, c.table, c.lens, parent)), out=out)
    Oref, Lref, A = R.tree_attn(Q, Kn, Vn, c, parent)
    fine = Oref.isfinite()
    o = O.double().cpu()
    assert torch.equal(o.isfinite(), fine) and not bool(fine.all())
    zero = torch.zeros_like(Oref)
    close(torch.where(fine, o, zero), LSE, (torch.where(fine, Oref, zero), Lref, torch.where(fine, A, zero)), T * Hq // Hkv)


@pytest.mark.parametrize("T,Hq,Hkv,d", [f for f in FORMS if f[0] > 1])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
def test_keys_of_new_tokens(T, Hq, Hkv, d, value):
    """A node's key that is not finite reaches the nodes that see it, by outputs and LSE, and nobody else.  (A logit of +infinity makes the
    softmax NaN; one of -infinity is a weight of 0.)"""
    c = R.Cache([50, 129], 16, Hkv, d, room=T)
    Q, Kn, Vn, parent = drafts(2, T, Hq, Hkv, d, seed=T)
    Kn[0, 1, :, 3], Kn[1, T // 2, 0, d - 1] = value, value
    O, LSE = tree(c, Q, Kn, Vn, parent)
    Oref, Lref, A = R.tree_attn(Q, Kn, Vn, c, parent)
    o, l = O.double().cpu(), LSE.double().cpu()
    fine = Oref.isfinite()
    assert not bool(fine.all()) or value == -INF
    assert torch.equal(o.isfinite(), fine) and bool(o[~fine].isnan().all())
    row = fine.all(-1)
    assert torch.equal(fine.any(-1), row) and not bool(l[~row].isfinite().any())
    R.check(o[row], l[row], (Oref[row], Lref[row], A[row]))


@pytest.mark.parametrize("T,Hq,Hkv,d", FORMS)
def test_cached_keys(T, Hq, Hkv, d):
    """A NaN in a cached key is everybody's NaN for that KV head alone."""
    c = R.Cache([300, 40], 16, Hkv, d, room=T)
    Q, Kn, Vn, parent = drafts(2, T, Hq, Hkv, d, seed=T)
    plant(c, 0, 7, 3, NAN, c.K, head=Hkv - 1)
    O, LSE = tree(c, Q, Kn, Vn, parent)
    g = Hq // Hkv
    assert bool(O[0, :, -g:].isnan().all()) and bool(LSE[0, :, -g:].isnan().all())
    clean = torch.ones(2, T, Hq, dtype=torch.bool)
    clean[0, :, -g:] = False
    R.check(O.cpu()[clean], LSE.cpu()[clean], [x[clean] for x in R.tree_attn(Q, Kn, Vn, c, parent)])
