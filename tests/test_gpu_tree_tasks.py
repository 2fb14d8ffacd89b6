"""Tree attention where one thread block runs tasks of different shapes one after the other: more than 128 stacked rows
(two tiles, a softmax group each), then at most 128 (one tile that both groups share), over long prefixes."""
import numpy as np
import pytest
import torch

from oracle import sdlm_tree_oracle as to
from test_gpu_tree import Tree

pytestmark = pytest.mark.gpu


def _grow(t, total):
    """Keys whose scores grow by `total` along each prefix (and vary by 1 around that), so that a row's reference moves
    again and again: element 0 of every query is large, element 0 of a key says how far along it is."""
    big = 8.0
    t.q[..., 0] = big
    for b, x in enumerate(t.lens):
        if x:
            t.kc[b][:, :, 0] = (torch.arange(x, device="cuda") * (total / (x * big * t.scale))).to(torch.bfloat16)[:, None]
            t.sd.kv_release_seq(t.slots[b])
            t.sd.kv_add_seq(t.slots[b], t.kc[b], t.vc[b])
    t.k[..., 0] = total / (big * t.scale)


def _reference(t, b):
    """Sequence b in 64 bits on the GPU: out and sum_t p_t |v_t|, [nodes, hq, d]."""
    m, x, G = t.nodes[b], t.lens[b], t.hq // t.hk
    sees = torch.zeros((m, x + m), dtype=torch.bool)
    sees[:, :x] = True
    for j in range(m):
        sees[j, [x + i for i in to.tree_path(t.par[b], j)]] = True
    out, size = (torch.zeros((m, t.hq, t.d), dtype=torch.float64, device="cuda") for _ in range(2))
    for h in range(t.hk):
        k, v = torch.cat((t.kc[b][:, h], t.k[b, :m, h])).double(), torch.cat((t.vc[b][:, h], t.v[b, :m, h])).double()
        s = torch.einsum("jgd,td->jgt", t.q[b, :m, h * G:(h + 1) * G].double(), k) * t.scale
        w = torch.softmax(s.masked_fill(~sees.cuda()[:, None], float("-inf")), -1)
        out[:, h * G:(h + 1) * G] = w @ v
        size[:, h * G:(h + 1) * G] = w @ v.abs()
    return out, size


def _check(t, out, scores):
    """Weights rounded to bf16 move the sum of weighted values and the sum of weights by 2^-8 each; scores of up to `scores`
    are fp32 sums of d products, off by at most d * 2^-24 of the sum of their sizes (`scores` + 8 covers it), which
    moves a weight by that much, in both sums; the powers of two are good to 7.5e-5, in both sums; one rounding to bf16."""
    torch.cuda.synchronize()
    assert t.sd.device_status()[0] == 0
    loose = 2.0 ** -7 + 2 * (t.d * 2.0 ** -24 * (scores + 8.0) + 7.5e-5)
    for b in range(t.B):
        m = t.nodes[b]
        ref, size = _reference(t, b)
        off = (out[b, :m].double() - ref).abs() / (2.0 ** -8 * ref.abs() + size * loose + 1e-30)
        assert bool((off <= 1.0).all()), f"sequence {b} ({t.lens[b]} tokens, {m} nodes): {off.max().item()} of the bound"
        assert bool((out[b, m:] == 7.0).all()), "padding rows were written"


# (query heads, KV heads, head size, nodes of the sequences in turn): tasks of 129..224 rows, then of 128 or fewer; with
# five heads a group and 64 nodes a sequence has a task of 256 rows and one of 64
CASES = [(16, 2, 128, (28, 16, 17, 1, 20, 15)), (8, 1, 64, (28, 16, 17, 1, 20, 15)), (16, 2, 64, (18, 2)), (40, 8, 128, (64,)),
         (20, 4, 64, (64, 60))]


@pytest.mark.parametrize("hq,hk,d,nodes", CASES)
@pytest.mark.parametrize("many,lo,hi", [(40, 2500, 5000), (240, 100, 600)])
def test_wide_tasks_followed_by_narrow_ones(hq, hk, d, nodes, many, lo, hi):
    if hq == 40:
        many //= 5
    rng = np.random.default_rng(many + hq)
    lens = [int(x) for x in rng.integers(lo, hi, many)]
    n = max(nodes)
    t = Tree(hq, hk, d, lens, n, nodes=[nodes[b % len(nodes)] for b in range(many)], seed=many)
    _grow(t, 40.0)
    first = t.attn()
    _check(t, first, 44.0)
    for _ in range(30):
        assert torch.equal(first, t.attn())


@pytest.mark.parametrize("hq,hk,d", [(4, 4, 64), (8, 2, 128)])
def test_thread_blocks_with_many_tasks_of_one_key_tile(hq, hk, d):
    """One node on an empty history (its key is the only one: the result is its value, exactly), some 30 tasks a thread
    block of which the second softmax group and its issuer have no key tile; among them a few of two and three tiles."""
    lens = [0] * 2000
    for b in range(0, 2000, 97):
        lens[b] = 40 + b % 70
    t = Tree(hq, hk, d, lens, 1, seed=3)
    want = t.v.repeat_interleave(hq // hk, 2)
    alone = torch.tensor([x == 0 for x in lens], device="cuda")
    first = t.attn()
    assert torch.equal(first[alone], want[alone])
    for b in range(0, 2000, 97):
        ref, size = _reference(t, b)
        # products of size 1: scores are good to d * 2^-24 * 8, the rest as above
        assert bool(((first[b].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + size * (2.0 ** -7 + 3e-4)).all())
    for _ in range(50):
        assert torch.equal(first, t.attn())
    assert t.sd.device_status()[0] == 0
