"""Commit of accepted paths into many layers at once: ragged trees, other slots, and the same as a call a layer."""
import numpy as np
import pytest
import torch

import paper_2509_24007_b200 as pk
from test_gpu_tree import Tree, _check_commit, _draft

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hk,d,B,n,layers", [(4, 2, 64, 40, 20, 3), (16, 2, 128, 9, 64, 5), (2, 1, 64, 300, 7, 2), (2, 1, 64, 1, 1, 64)])
def test_ragged_trees_into_every_layer(hq, hk, d, B, n, layers):
    rng = np.random.default_rng(B)
    lens, slots = [int(x) for x in rng.integers(0, 200, B)], [int(x) for x in rng.permutation(B)]
    nodes = [int(x) for x in rng.integers(0, n + 1, B)]
    ts = [Tree(hq, hk, d, lens, n, nodes=nodes, slots=slots, seed=70) for _ in range(layers)]
    for i, t in enumerate(ts):
        t.k, t.v = t.k + i, t.v - i
    draft, decided = _draft(ts[0], 0.9)
    out = pk.tree_commit_layers([t.sd for t in ts], torch.from_numpy(draft).cuda(), torch.from_numpy(decided).cuda(), ts[0].parent,
                                [t.k for t in ts], [t.v for t in ts], n_nodes=ts[0].n_nodes, seq_ids=ts[0].seq_ids)
    for t in ts:
        assert _check_commit(t, draft, decided, *out)["status"][0] == 0


def test_a_layer_call_equals_a_call_a_layer():
    lens, nodes = [64, 10, 0, 127, 3], [9, 0, 4, 9, 1]
    ts = [Tree(4, 2, 64, lens, 9, nodes=nodes, seed=71) for _ in range(4)]
    draft, decided = _draft(ts[0], 0.9)
    d, x = torch.from_numpy(draft).cuda(), torch.from_numpy(decided).cuda()
    a = pk.tree_commit_layers([t.sd for t in ts[:2]], d, x, ts[0].parent, [t.k for t in ts[:2]], [t.v for t in ts[:2]], n_nodes=ts[0].n_nodes)
    for t in ts[2:]:
        b = t.sd.tree_commit(d, x, t.parent, t.k, t.v, n_nodes=t.n_nodes)
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    tables = [t.sd.kv_tables() for t in ts]
    for o in tables[1:]:
        assert all(np.array_equal(tables[0][k], o[k]) for k in ("page_table", "seq_len", "free_list", "free_head", "free_tail"))
