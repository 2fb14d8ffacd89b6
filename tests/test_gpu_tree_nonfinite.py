"""Infinities and NaN in K and V of a drafted tree and of the cache: they reach the rows that see their token, no others."""
import numpy as np
import pytest
import torch

from oracle import sdlm_tree_oracle as to
from test_gpu_tree import Tree
from test_gpu_tree_tasks import _reference

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
# (query heads, KV heads, head size, nodes): one and two tiles of stacked rows, more than 32 nodes
CASES = [(16, 2, 128, 20), (16, 2, 128, 9), (4, 2, 64, 64), (10, 2, 64, 40), (3, 3, 128, 50), (8, 2, 128, 1)]


def _make(hq, hk, d, n):
    """Prefixes that are empty, short, cut over several thread blocks, and some more tasks a thread block than one."""
    return Tree(hq, hk, d, [0, 70, 3000, 64] + [130 + 7 * b for b in range(60)], n, seed=60 + n)


def _same_bits(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("hq,hk,d,n", CASES)
def test_values_of_hidden_nodes(hq, hk, d, n):
    t = _make(hq, hk, d, n)
    base = t.attn()
    t.check(base)
    rng = np.random.default_rng(n)
    put = torch.zeros(t.v.shape, dtype=torch.float32)      # what is put in the place of values, 0 where they stay
    for b in (0, 1, 2, 5, t.B - 1):
        for j in rng.choice(n, max(1, n // 6), replace=False):
            h = int(rng.integers(hk))
            for c in rng.choice(d, 3, replace=False):
                put[b, j, h, c] = [INF, -INF, NAN][int(rng.integers(3))]
    t.v = torch.where(put.cuda() != 0, put.cuda(), t.v.float()).to(torch.bfloat16)
    want = torch.zeros(t.q.shape)                            # infinities and NaN of the nodes each row sees, added up
    for b in range(t.B):
        for j in range(n):
            want[b, j] = put[b, to.tree_path(t.par[b], j)].sum(0).repeat_interleave(hq // hk, 0)
    want = want.cuda()
    got = t.attn()
    torch.cuda.synchronize()
    hit = want != 0
    assert torch.equal(torch.where(hit, 0.0, got.float()), torch.where(hit, 0.0, base.float()))
    assert torch.equal(torch.nan_to_num(torch.where(hit, got.float(), 0.0), 1.0, 2.0, 3.0), torch.nan_to_num(torch.where(hit, want, 0.0), 1.0, 2.0, 3.0))
    assert int(hit.sum()) >= 5 and _same_bits(got, t.attn()) and t.sd.device_status()[0] == 0


@pytest.mark.parametrize("hq,hk,d,n", CASES)
def test_keys_of_hidden_nodes(hq, hk, d, n):
    t = _make(hq, hk, d, n)
    base = t.attn()
    G, hit = hq // hk, torch.zeros((t.B, n, hk), dtype=torch.bool)
    for b in (0, 2, 5, t.B - 1):
        for node, h, x in ((n // 3, 0, NAN), (n // 2, hk - 1, INF)):
            t.k[b, node, h, 3] = x
            for j in range(n):
                hit[b, j, h] |= node in to.tree_path(t.par[b], j)
    got = t.attn()
    torch.cuda.synchronize()
    rows = hit.repeat_interleave(G, 2).cuda()
    assert _same_bits(got[~rows], base[~rows])
    for b in (0, 2, 5, t.B - 1):  # a key of minus infinity after the product has no weight; plus infinity and NaN give NaN
        ref, size = _reference(t, b)
        assert torch.equal(got[b].isfinite(), ref.isfinite())
        fine = ref.isfinite()
        # scores of products of size 1 (d * 2^-24 * 40 at the most), weights rounded to bf16 and powers of two, each in both sums
        assert bool(((got[b].double() - ref).abs()[fine] <= 2.0 ** -8 * ref.abs()[fine] + size[fine] * (2.0 ** -7 + 9e-4)).all())


@pytest.mark.parametrize("hq,hk,d,n", CASES)
def test_cached_tokens(hq, hk, d, n):
    t = _make(hq, hk, d, n)
    base = t.attn()
    for b, at in ((1, 69), (2, 1500), (7, 3), (8, 64)):
        kv, x = (t.kc, NAN) if b < 7 else (t.vc, INF)
        for i in range(4):  # neighbours: in different positions of the registers a row's scores are in
            kv[b][at - i, 0, 2] = x
        t.sd.kv_release_seq(b)
        t.sd.kv_add_seq(b, t.kc[b], t.vc[b])
    got = t.attn()
    torch.cuda.synchronize()
    G, hit = hq // hk, torch.zeros(t.q.shape, dtype=torch.bool, device="cuda")
    hit[1:3, :, :G] = True
    hit[7:9, :, :G, 2] = True
    assert _same_bits(got[~hit], base[~hit]) and not bool(got[hit].isfinite().any())
