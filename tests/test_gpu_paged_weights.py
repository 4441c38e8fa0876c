"""GPU parity: how far attention over a paged cache may be off where its weights are kept as two bf16 numbers (up to 64 query rows per KV
head, and selected pages), against the definition in 64 bits."""
import pytest
import torch

import paged_reference as R
from paper_2607_20457_b200 import binding
from test_gpu_paged_not_finite import close
from test_gpu_tree_attn import drafts

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


@pytest.mark.parametrize("T,Hq,Hkv,d", [(1, 8, 2, 128), (1, 4, 4, 64), (3, 4, 1, 64), (5, 8, 2, 128), (8, 4, 1, 64), (13, 16, 4, 64), (16, 8, 2, 128),
                                        (24, 8, 2, 128), (64, 8, 2, 64)])
@pytest.mark.parametrize("page", [16, 64])
def test_weights_have_16_bits_up_to_64_rows(T, Hq, Hkv, d, page):
    """Float32 outputs over few rows, where a weight that is rounded once shows: with both parts of P they are within 2^-16 of A."""
    lens = [0, 1, 5, 17, 40]
    c = R.Cache(lens, page, Hkv, d, room=T, seed=T)
    Q, Kn, Vn, parent = drafts(len(lens), T, Hq, Hkv, d, seed=T, scale=0.25)
    out = torch.empty(len(lens), T, Hq, d, device=DEV)
    O, LSE = binding.pulsar_tree_attn(*(x.to(DEV) for x in (Q, Kn, Vn, c.K, c.V, c.table, c.lens, parent)), out=out)
    close(O, LSE, R.tree_attn(Q, Kn, Vn, c, parent), T * Hq // Hkv)
    if T > 1:                                              # and with fewer nodes
        n = torch.tensor([T, 1, T - 1, 1, T], dtype=torch.int32)
        O, LSE = binding.pulsar_tree_attn(*(x.to(DEV) for x in (Q, Kn, Vn, c.K, c.V, c.table, c.lens, parent, n)), out=out)
        used = torch.arange(T) < n[:, None]
        close(O.cpu()[used], LSE.cpu()[used], [x[used] for x in R.tree_attn(Q, Kn, Vn, c, parent, n)], T * Hq // Hkv)


@pytest.mark.parametrize("T,Hq,Hkv,d", [(1, 8, 2, 128), (6, 8, 2, 128), (13, 16, 4, 64), (16, 4, 1, 128)])
def test_both_parts_are_rescaled(T, Hq, Hkv, d):
    """Logits that rise by 9 to 10 log2 units a step: what both parts of P have summed up is rescaled, and still counts.  The first
    slot's six tiles are a thread block's share of the batch."""
    lens = [700] + [128 * 3] * 320
    c = R.Cache(lens, 16, Hkv, d, room=T)
    Q, Kn, Vn, parent = drafts(len(lens), T, Hq, Hkv, d, seed=T)
    g = torch.Generator().manual_seed(2)
    u = torch.randn(Hkv, d, generator=g)
    u /= u.norm(dim=-1, keepdim=True)
    Q = (Q.float() * 0.05 + u.repeat_interleave(Hq // Hkv, 0)).to(BF)
    rise = {0: 0.0, 70: 9.0, 200: 18.5, 300: 28.0, 500: 37.5, 690: 39.0}
    h = 0.0
    for r in range(700):
        h = rise.get(r, h)
        at = c.table[0, r // 16], r % 16
        c.K[at] = (c.K[at].float() * 0.05 + u * h * 0.6931).to(BF)
    out = torch.empty(Q.shape, device=DEV)
    O, LSE = binding.pulsar_tree_attn(*(x.to(DEV) for x in (Q, Kn, Vn, c.K, c.V, c.table, c.lens, parent)), softmax_scale=1.0, out=out)
    # A logit is a sum of up to 128 products that add up to less than 2 * 39 * 0.6931 = 54; an fp32 product of 16 terms at a time rounds eight
    # sums: 8 * 2^-23 * 54 = 5.2e-5, twice in a weight.
    n = [T] + [0] * 320
    Oref, Lref, A = (x[0] for x in R.tree_attn(Q, Kn, Vn, c, parent, n, 1.0))
    err, bound = (O[0].double().cpu() - Oref).abs(), (2.0 ** -16 + 2e-4) * A + 1e-6
    assert bool((err <= bound).all()), f"{float((err / bound).max()):.2f} of the bound"
    assert float((LSE[0].double().cpu() - Lref).abs().max()) <= 2e-4


@pytest.mark.parametrize("T,Hq,Hkv,d", [(1, 8, 2, 128), (3, 4, 1, 64)])
def test_selected_pages(T, Hq, Hkv, d):
    c = R.Cache([16 * 9 + 5, 16, 3], 16, Hkv, d, room=T)
    Q, Kn, Vn, _ = drafts(3, T, Hq, Hkv, d, seed=T, scale=0.25)
    bounds = R.page_bounds(c.K)
    O, LSE, sel = binding.pulsar_sparse_attn(*(x.to(DEV) for x in (Q, Kn, Vn, c.K, c.V, bounds, c.table, c.lens)), 3, 1, 1)
    *ref, want = R.sparse_attn(Q, Kn, Vn, c, bounds, 3, 1, 1)
    assert torch.equal(sel.cpu(), want)
    close(O, LSE, ref, Hq // Hkv, rounded=True)
