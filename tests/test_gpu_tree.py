"""GPU parity of the drafted-tree operators (tree attention, tree commit, batched gather) with the float64 oracle."""
import numpy as np
import pytest
import torch

import paper_2509_24007_b200 as pk
from oracle import sdlm_tree_oracle as to

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.float().cpu().numpy().astype(np.float64)


class Tree:
    """A context with cached sequences of the given lengths and a random tree on each."""

    def __init__(self, hq, hk, d, lens, n, nodes=None, seed=0, shape="random", slots=None, scale=0.0, spare=2, std=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.rng = np.random.default_rng(seed)
        B = len(lens)
        self.B, self.n, self.hq, self.hk, self.d, self.lens = B, n, hq, hk, d, list(lens)
        self.nodes = [n] * B if nodes is None else list(nodes)
        pages = sum((x + n + 63) // 64 + 1 for x in lens) + spare
        per = max((x + n + 63) // 64 for x in lens) + 1
        n_slots = max(B, max(slots) + 1 if slots else 0)
        self.sd = pk.Sdlm(pk.SdlmConfig(hq, hk, d, 64, 64, pages, n_slots, per, max_block=1, softmax_scale=scale))
        self.sd._pool.fill_(255)  # bf16 NaN everywhere: nothing outside the sequences may count
        self.sd.kv_reset(self.rng.permutation(pages).astype(np.int32))
        self.scale = scale or d ** -0.5
        normal = lambda *s: (torch.randn(s, generator=g, device="cuda") * std).to(torch.bfloat16)
        self.kc = [normal(x, hk, d) for x in lens]
        self.vc = [normal(x, hk, d) for x in lens]
        self.slots = list(range(B)) if slots is None else list(slots)
        self.seq_ids = None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda")
        for b, x in enumerate(lens):
            if x and self.slots[b] not in self.slots[:b]:
                self.sd.kv_add_seq(self.slots[b], self.kc[b], self.vc[b])
        self.q, self.k, self.v = normal(B, n, hq, d), normal(B, n, hk, d), normal(B, n, hk, d)
        if shape == "chain":
            par = np.tile(np.arange(n) - 1, (B, 1))
        elif shape == "star":
            par = np.full((B, n), -1)
        else:
            par = np.stack([[self.rng.integers(-1, j) if j else -1 for j in range(n)] for _ in range(B)])
        self.par = par.astype(np.int32)
        self.parent = torch.from_numpy(self.par).cuda()
        self.n_nodes = None if nodes is None else torch.tensor(nodes, dtype=torch.int32, device="cuda")

    def attn(self, **kw):
        out = torch.full_like(self.q, 7.0)
        self.sd.tree_attn(self.q, self.k, self.v, self.parent, n_nodes=self.n_nodes, seq_ids=self.seq_ids, out=out, **kw)
        return out

    def check(self, out):
        torch.cuda.synchronize()
        assert self.sd.device_status()[0] == 0
        got = _bits(out)
        for b in range(self.B):
            m = self.nodes[b]
            ref, size = to.tree_attention(_bits(self.q[b, :m]), _bits(self.kc[b]), _bits(self.vc[b]), _bits(self.k[b, :m]),
                                          _bits(self.v[b, :m]), self.par[b], self.scale)
            # Rounding each weight to bf16 (2^-8) moves the sum of weighted values and the sum of weights; scores are
            # fp32 sums of d products (d * 2^-24 of the products' absolute sum, below 2e-4 for the sizes here) and the
            # powers of two good to 7.5e-5, each again in both sums; then one rounding to bf16.
            bound = 2.0 ** -8 * np.abs(ref) + size * (2.0 ** -7 + 6e-4) + 1e-30
            err = np.abs(got[b, :m] - ref)
            assert np.all(np.isfinite(got[b, :m])) and np.all(err <= bound), \
                f"sequence {b}: {np.max(err / bound)} of the bound at {np.unravel_index(np.argmax(err / bound), err.shape)}"
            assert np.all(got[b, m:] == 7.0), "padding rows were written"


HEADS = [(16, 2, 128), (40, 8, 128), (4, 2, 64), (3, 3, 128), (64, 1, 64), (7, 1, 128)]


@pytest.mark.parametrize("hq,hk,d", HEADS)
@pytest.mark.parametrize("n", [1, 2, 17, 64])
def test_attention_over_short_and_odd_prefixes(hq, hk, d, n):
    t = Tree(hq, hk, d, [0, 1, 63, 64, 65, 127, 128, 129, 200], n, seed=n + hq)
    t.check(t.attn())


@pytest.mark.parametrize("n,lens", [(1, [1024]), (8, [5000]), (33, [3, 2500, 700]), (64, [4097]), (16, [900] * 40)])
@pytest.mark.parametrize("hq,hk,d", [(16, 2, 128), (10, 2, 64)])
def test_attention_over_longer_prefixes(n, lens, hq, hk, d):
    t = Tree(hq, hk, d, lens, n, seed=n + len(lens))
    t.check(t.attn())


@pytest.mark.parametrize("shape", ["chain", "star"])
def test_chains_and_stars(shape):
    t = Tree(16, 2, 128, [0, 100, 640], 64, shape=shape, seed=5)
    t.check(t.attn())


def test_ragged_trees_leave_padding_alone():
    t = Tree(16, 4, 64, [10, 300, 0, 64, 1000, 77], 40, nodes=[40, 0, 1, 33, 16, 7], seed=6)
    t.check(t.attn())


def test_padding_and_hidden_keys_may_hold_anything():
    """NaN in padding rows of the tree, and in the pool outside the sequences, is never seen."""
    t = Tree(8, 2, 64, [30, 129], 20, nodes=[11, 20], seed=7)
    t.k[0, 11:], t.v[0, 11:], t.q[0, 11:] = float("nan"), float("inf"), float("nan")
    t.parent[0, 11:] = 2 ** 30
    t.check(t.attn())


def test_parents_that_are_not_earlier_nodes_hang_from_the_history():
    t = Tree(8, 2, 64, [70], 12, seed=8)
    t.par[0] = [5, 0, 2, 1, 99, -7, 4, 7, 2 ** 31 - 1, -2 ** 31, 9, 11]
    t.parent.copy_(torch.from_numpy(t.par))
    t.check(t.attn())


def test_sequences_in_other_slots_and_the_same_slot_twice():
    t = Tree(16, 2, 128, [500, 90, 90, 3], 9, slots=[5, 2, 2, 7], seed=9)
    t.kc[2], t.vc[2] = t.kc[1], t.vc[1]
    t.check(t.attn())


def test_large_scores_and_another_scale():
    t = Tree(8, 2, 128, [300, 1500], 30, seed=10, std=3.0, scale=0.2)
    t.sd.device_status()
    got = _bits(t.attn())
    for b in range(2):
        ref, size = to.tree_attention(_bits(t.q[b]), _bits(t.kc[b]), _bits(t.vc[b]), _bits(t.k[b]), _bits(t.v[b]), t.par[b], t.scale)
        # products of size 9 and a scale of 0.2: 128 of them add up to some 200, so scores carry 128 * 2^-24 * 200 = 1.6e-3
        assert np.all(np.abs(got[b] - ref) <= 2.0 ** -8 * np.abs(ref) + size * (2.0 ** -7 + 4e-3))


def test_a_bad_slot_is_reported_and_its_rows_left_alone():
    t = Tree(4, 2, 64, [40, 50], 6, slots=[0, 1], seed=11)
    t.seq_ids.copy_(torch.tensor([0, 99], dtype=torch.int32))
    out = t.attn()
    torch.cuda.synchronize()
    st = t.sd.device_status(clear=True)
    assert st[0] == 7 and st[1] == 99 and bool((out[1] == 7.0).all())
    ref, size = to.tree_attention(_bits(t.q[0]), _bits(t.kc[0]), _bits(t.vc[0]), _bits(t.k[0]), _bits(t.v[0]), t.par[0], t.scale)
    assert np.all(np.abs(_bits(out[0]) - ref) <= 2.0 ** -8 * np.abs(ref) + size * (2.0 ** -7 + 6e-4))


def test_the_same_call_gives_the_same_bits_and_captures():
    t = Tree(16, 2, 128, [700, 2000, 64], 24, seed=12)
    a = t.attn()
    out = torch.zeros_like(t.q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        t.sd.tree_attn(t.q, t.k, t.v, t.parent, out=out)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(a, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.sd.tree_attn(t.q, t.k, t.v, t.parent, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, out)
    t.q.copy_(torch.randn_like(t.q))  # a replay reads the inputs as they are then
    graph.replay()
    t.check(out)


def test_a_block_of_one_node_equals_the_masked_block_attention():
    """Beside the operator that was there: one node is a block of one query position that sees the history and itself."""
    t = Tree(16, 2, 128, [700, 130], 1, seed=13)
    vis = torch.ones((2, 1), dtype=torch.int32, device="cuda")
    ref = t.sd.block_attn_masked(t.q, t.k, t.v, vis)
    assert float((ref.float() - t.attn().float()).abs().max()) <= 2e-2


@pytest.mark.parametrize("kw,code", [(dict(n=65), 2), (dict(batch=3), 2), (dict(batch=0), 1), (dict(n=0), 1), (dict(parent=None), 1),
                                     (dict(q=8), 1), (dict(out=None), 1), (dict(k=2), 1)])
def test_attention_refusals_enqueue_nothing(kw, code):
    t = Tree(4, 2, 64, [10, 20], 4, seed=14)
    out = torch.full_like(t.q, 7.0)
    ptr = dict(q=t.q.data_ptr(), k=t.k.data_ptr(), v=t.v.data_ptr(), parent=t.parent.data_ptr(), out=out.data_ptr())
    for a, x in kw.items():
        if a in ptr:
            ptr[a] = None if x is None else ptr[a] + x
    before = t.sd.launch_count()
    rc = t.sd.lib.sdlm_tree_attn(t.sd.ctx, kw.get("batch", 2), kw.get("n", 4), None, None, ptr["parent"], ptr["q"], ptr["k"],
                                 ptr["v"], ptr["out"], torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == code and t.sd.launch_count() == before and bool((out == 7.0).all())


def test_binding_refuses_wrong_tensors():
    t = Tree(4, 2, 64, [10, 20], 4, seed=15)
    with pytest.raises(ValueError):
        t.sd.tree_attn(t.q[:, :3].contiguous(), t.k, t.v, t.parent)
    with pytest.raises(TypeError):
        t.sd.tree_attn(t.q.float(), t.k, t.v, t.parent)
    with pytest.raises(TypeError):
        t.sd.tree_attn(t.q, t.k, t.v, t.parent.long())
    with pytest.raises(ValueError):
        t.sd.tree_attn(t.q, t.k, t.v, t.parent, n_nodes=torch.ones(3, dtype=torch.int32, device="cuda"))


# ---- commit ------------------------------------------------------------------------------------------------
def _draft(t, p=0.8):
    B, n = t.B, t.n
    draft = t.rng.integers(0, 6, size=(B, n)).astype(np.int32)
    decided = t.rng.integers(100, 106, size=(B, n)).astype(np.int32)
    for b in range(B):
        for j in range(1, n):
            if 0 <= t.par[b, j] < j and t.rng.random() < p:
                decided[b, t.par[b, j]] = draft[b, j]
    return draft, decided


def _check_commit(t, draft, decided, acc, tok, path, fails=()):
    acc, tok, path = (x.cpu().numpy() for x in (acc, tok, path))
    tables = t.sd.kv_tables()
    room = max(t.lens) + t.n
    per = t.sd.cfg.max_pages_per_seq * 64
    k = torch.zeros((t.B, min(room, per), t.hk, t.d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    ids = torch.tensor(t.slots, dtype=torch.int32, device="cuda")
    t.sd.kv_gather_batch(k, v, seq_ids=ids)
    pages = []
    for b in range(t.B):
        way = to.tree_walk(t.par[b], draft[b], decided[b], t.nodes[b])
        new = [] if b in fails else way
        assert acc[b] == (-1 if b in fails else len(way))
        assert list(tok[b]) == [decided[b, i] for i in new] + [-1] * (t.n - len(new))
        if b not in fails:
            assert list(path[b]) == way + [-1] * (t.n - len(way))
        total = t.lens[b] + len(new)
        assert tables["seq_len"][t.slots[b]] == total
        assert torch.equal(k[b, :total], torch.cat([t.kc[b], t.k[b, new]])) and bool((k[b, total:] == 0).all())
        assert torch.equal(v[b, :total], torch.cat([t.vc[b], t.v[b, new]])) and bool((v[b, total:] == 0).all())
        pages += list(tables["page_table"][t.slots[b], :(total + 63) // 64])
    assert len(set(pages)) == len(pages) and min(pages, default=0) >= 0
    return tables


@pytest.mark.parametrize("hq,hk,d", [(16, 2, 128), (4, 2, 64), (8, 8, 64)])
@pytest.mark.parametrize("n", [1, 5, 32, 33, 64])
def test_commit_appends_the_accepted_path(hq, hk, d, n):
    t = Tree(hq, hk, d, [0, 1, 63, 64, 100, 128], n, seed=20 + n)
    draft, decided = _draft(t)
    out = t.sd.tree_commit(torch.from_numpy(draft).cuda(), torch.from_numpy(decided).cuda(), t.parent, t.k, t.v)
    tables = _check_commit(t, draft, decided, *out)
    assert tables["status"][0] == 0


def test_commit_of_whole_chains_fills_pages():
    t = Tree(4, 2, 64, [0, 1, 63, 64], 64, shape="chain", seed=30)
    draft = np.tile(np.arange(64, dtype=np.int32), (4, 1))
    decided = draft + 1
    out = t.sd.tree_commit(torch.from_numpy(draft).cuda(), torch.from_numpy(decided).cuda(), t.parent, t.k, t.v)
    _check_commit(t, draft, decided, *out)
    assert out[0].tolist() == [64] * 4


def test_commit_of_ragged_trees_in_other_slots():
    t = Tree(4, 2, 64, [10, 0, 64, 7], 20, nodes=[20, 0, 1, 13], slots=[3, 1, 6, 0], seed=31)
    draft, decided = _draft(t)
    out = t.sd.tree_commit(torch.from_numpy(draft).cuda(), torch.from_numpy(decided).cuda(), t.parent, t.k, t.v,
                           n_nodes=t.n_nodes, seq_ids=t.seq_ids)
    _check_commit(t, draft, decided, *out)


def test_commit_of_many_sequences_hands_out_pages_in_order():
    t = Tree(2, 1, 64, [60 + b % 9 for b in range(300)], 8, seed=32)
    ring = t.sd.kv_tables()["free_list"]
    head = t.sd.kv_tables()["free_head"]
    draft, decided = _draft(t)
    out = t.sd.tree_commit(torch.from_numpy(draft).cuda(), torch.from_numpy(decided).cuda(), t.parent, t.k, t.v)
    tables = _check_commit(t, draft, decided, *out)
    for b in range(t.B):
        a = len(to.tree_walk(t.par[b], draft[b], decided[b], t.n))
        if (t.lens[b] + 63) // 64 < (t.lens[b] + a + 63) // 64:
            assert tables["page_table"][b, (t.lens[b] + a + 63) // 64 - 1] == ring[head % len(ring)]
            head += 1
    assert tables["free_head"] == head


def test_commit_failures_are_reported_and_commit_nothing():
    t = Tree(4, 2, 64, [64, 10, 20, 30], 4, slots=[0, 1, 2, 3], seed=33, shape="chain")
    draft = np.tile(np.arange(4, dtype=np.int32), (4, 1))
    decided = draft + 1
    ids = torch.tensor([0, 1, 1, -5], dtype=torch.int32, device="cuda")  # a slot twice, a slot that is none
    d, x = torch.from_numpy(draft).cuda(), torch.from_numpy(decided).cuda()
    acc, tok, path = t.sd.tree_commit(d, x, t.parent, t.k, t.v, seq_ids=ids)
    assert acc.tolist() == [4, -1, -1, -1] and t.sd.device_status(clear=True)[0] == 7
    t.sd.device_status()
    _check_commit(t, draft, decided, acc, tok, path, fails=(1, 2, 3))


def test_commit_without_free_pages():
    t = Tree(4, 2, 64, [64, 64, 10], 4, seed=34, shape="chain", spare=0)
    tables = t.sd.kv_tables()
    free = tables["free_tail"] - tables["free_head"]
    big = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert free >= 1 and big.numel() == 0
    # one more context whose pool has a single page left after the prefixes
    sd = pk.Sdlm(pk.SdlmConfig(4, 2, 64, 64, 64, 4, 3, 3, max_block=1))
    for b in range(3):
        sd.kv_add_seq(b, t.kc[b], t.vc[b])
    draft = np.tile(np.arange(4, dtype=np.int32), (3, 1))
    acc, tok, path = sd.tree_commit(torch.from_numpy(draft).cuda(), torch.from_numpy(draft + 1).cuda(), t.parent, t.k, t.v)
    assert acc.tolist() == [4, -1, 4] and sd.device_status(clear=True)[0] == 4
    assert sd.kv_tables()["seq_len"].tolist() == [68, 64, 14] and tok[1].tolist() == [-1] * 4


def test_commit_into_several_layers():
    ts = [Tree(4, 2, 64, [10, 62, 64], 9, seed=35) for _ in range(3)]
    for i, t in enumerate(ts):
        t.k, t.v = t.k + i, t.v - i
    draft, decided = _draft(ts[0])
    out = pk.tree_commit_layers([t.sd for t in ts], torch.from_numpy(draft).cuda(), torch.from_numpy(decided).cuda(),
                                ts[0].parent, [t.k for t in ts], [t.v for t in ts])
    for t in ts:
        _check_commit(t, draft, decided, *out)
    with pytest.raises(pk.SdlmError):
        pk.tree_commit_layers([ts[0].sd, ts[0].sd], torch.from_numpy(draft).cuda(), torch.from_numpy(decided).cuda(),
                              ts[0].parent, [ts[0].k] * 2, [ts[0].v] * 2)


def test_commit_captures_and_replays():
    t = Tree(4, 2, 64, [60], 3, seed=36, shape="chain", spare=6)
    draft = torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda")
    decided = draft + 1
    saved = t.sd.kv_save()
    acc, tok, path = (torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros_like(draft), torch.zeros_like(draft))
    t.sd.tree_commit(draft, decided, t.parent, t.k, t.v, accepted_len=acc, out_tokens=tok, path=path)
    t.sd.kv_restore(saved)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.sd.tree_commit(draft, decided, t.parent, t.k, t.v, accepted_len=acc, out_tokens=tok, path=path)
    for i in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert t.sd.kv_tables()["seq_len"][0] == 63 + 3 * i and acc.tolist() == [3]
    k, v = t.sd.kv_gather(0, 66)
    assert torch.equal(k, torch.cat([t.kc[0], t.k[0], t.k[0]])) and torch.equal(v, torch.cat([t.vc[0], t.v[0], t.v[0]]))


def test_batched_gather_equals_the_single_one_and_leaves_the_rest():
    t = Tree(4, 2, 128, [0, 1, 64, 200], 1, slots=[2, 0, 3, 1], seed=37)
    k = torch.full((4, 130, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    t.sd.kv_gather_batch(k, v, seq_ids=t.seq_ids)
    for b, x in enumerate(t.lens):
        m = min(x, 130)
        assert torch.equal(k[b, :m], t.kc[b][:m]) and torch.equal(v[b, :m], t.vc[b][:m])
        assert bool((k[b, m:] == 7.0).all()) and bool((v[b, m:] == 7.0).all())
    lib, st = t.sd.lib, torch.cuda.current_stream().cuda_stream
    assert lib.sdlm_kv_gather_batch(t.sd.ctx, 9, 5, None, k.data_ptr(), v.data_ptr(), st) == 2
    assert lib.sdlm_kv_gather_batch(t.sd.ctx, 1, 5, None, k.data_ptr() + 2, v.data_ptr(), st) == 1
    assert lib.sdlm_kv_gather_batch(t.sd.ctx, 1, 5, None, None, v.data_ptr(), st) == 1
    assert lib.sdlm_kv_gather_batch(t.sd.ctx, 1, 0, None, None, None, st) == 0


@pytest.mark.parametrize("kw,code", [(dict(n=65), 2), (dict(batch=9), 2), (dict(batch=0), 1), (dict(parent=None), 1), (dict(path=None), 1),
                                     (dict(next=None), 1), (dict(k=2), 1)])
def test_commit_refusals_enqueue_nothing(kw, code):
    t = Tree(4, 2, 64, [10, 20], 4, seed=38)
    z = torch.full((2, 4), 7, dtype=torch.int32, device="cuda")
    p = dict(parent=t.parent.data_ptr(), draft=z.data_ptr(), next=z.data_ptr(), k=t.k.data_ptr(), v=t.v.data_ptr(),
             acc=z.data_ptr(), tok=z.data_ptr(), path=z.data_ptr())
    for a, x in kw.items():
        if a in p:
            p[a] = None if x is None else p[a] + x
    before = t.sd.launch_count()
    rc = t.sd.lib.sdlm_tree_commit(t.sd.ctx, kw.get("batch", 2), kw.get("n", 4), None, None, p["parent"], p["draft"], p["next"],
                                   p["k"], p["v"], p["acc"], p["tok"], p["path"], torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == code and t.sd.launch_count() == before and bool((z == 7).all())
    assert t.sd.kv_tables()["seq_len"].tolist() == [10, 20]


# ---- the calls of a verification pass, one after the other -----------------------------------------------------
def test_a_pass_over_a_tree_rotate_attend_sample_commit():
    """Two passes: each node's query and key rotated at its depth behind the history, attention, logits, greedy tokens
    behind every node from the sampler, the accepted path committed; the second pass sees the first one's rows."""
    hq, hk, d, n, V = 8, 2, 64, 7, 96
    t = Tree(hq, hk, d, [33, 64], n, seed=40)
    rope = pk.RopeConfig(theta=10000.0)
    w = (torch.randn((V, hq * d), device="cuda") * 0.3).to(torch.bfloat16)
    f, m = to.rope_frequencies(d, 10000.0)
    kc, vc = [_bits(x) for x in t.kc], [_bits(x) for x in t.vc]
    for step in range(2):
        q, k, v = torch.randn_like(t.q), torch.randn_like(t.k), torch.randn_like(t.v)
        depth = np.array([[len(to.tree_path(t.par[b], j)) - 1 for j in range(n)] for b in range(2)], dtype=np.int32)
        qr, kr = t.sd.qk_norm_rope(q, k, rope, positions=torch.from_numpy(depth).cuda(), relative=True)
        out = t.sd.tree_attn(qr, kr, v, t.parent)
        logits = t.sd.linear(out.view(2 * n, hq * d), w)
        token, prob, entropy, kept = t.sd.sample(logits, torch.rand(2 * n, device="cuda"),
                                                 temperature=torch.zeros(2 * n, device="cuda"))
        decided = token.view(2, n).cpu().numpy()
        draft = t.rng.integers(0, V, size=(2, n)).astype(np.int32)
        for b in range(2):
            for j in range(1, n):
                if 0 <= t.par[b, j] < j and t.rng.random() < 0.7:
                    draft[b, j] = decided[b, t.par[b, j]]
        acc, tok, path = t.sd.tree_commit(torch.from_numpy(draft).cuda(), token.view(2, n), t.parent, kr, v)
        for b in range(2):
            ref_q, _ = to.norm_rope(_bits(q[b]), len(kc[b]) + depth[b], f, m, False)
            assert np.max(np.abs(_bits(qr[b]) - ref_q)) <= 2.0 ** -8 * np.max(np.abs(ref_q)) + 1e-5
            ref, size = to.tree_attention(_bits(qr[b]), kc[b], vc[b], _bits(kr[b]), _bits(v[b]), t.par[b], t.scale)
            assert np.all(np.abs(_bits(out[b]) - ref) <= 2.0 ** -8 * np.abs(ref) + size * (2.0 ** -7 + 6e-4))
            assert np.array_equal(decided[b], _bits(logits.view(2, n, V)[b]).argmax(-1))
            way = to.tree_walk(t.par[b], draft[b], decided[b], n)
            assert path[b].tolist() == way + [-1] * (n - len(way)) and acc[b].item() == len(way)
            assert tok[b].tolist() == [decided[b, i] for i in way] + [-1] * (n - len(way))
            kc[b], vc[b] = np.concatenate([kc[b], _bits(kr[b, way])]), np.concatenate([vc[b], _bits(v[b, way])])
        assert t.sd.device_status()[0] == 0
        assert t.sd.kv_tables()["seq_len"].tolist() == [len(x) for x in kc]
