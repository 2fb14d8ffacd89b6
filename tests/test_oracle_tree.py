"""Pins of the float64 oracle of the drafted-tree operators (no GPU)."""
import numpy as np
import pytest

from oracle import sdlm_layer_oracle as lo
from oracle import sdlm_tree_oracle as to


def test_plain_rotation_is_the_layer_oracles_rotation():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(1, 3, 2, 64))
    f, m = to.rope_frequencies(64, 10000.0)
    got, _ = to.norm_rope(x[0], np.array([7, 8, 9]), f, m, False)
    ref = lo.rope(x, np.array([[7, 8, 9]]), 10000.0)
    assert np.allclose(got, np.asarray(ref).reshape(got.shape), atol=1e-12)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_depends_on_differences_only(interleaved):
    rng = np.random.default_rng(1)
    f, m = to.rope_frequencies(32, 10000.0, "yarn", 1.0)
    a, b = rng.normal(size=(1, 1, 48)), rng.normal(size=(1, 1, 48))
    assert m == 1.0
    dots = []
    for shift in (0, 11, 5000):
        x, _ = to.norm_rope(a, np.array([3 + shift]), f, m, interleaved)
        y, _ = to.norm_rope(b, np.array([10 + shift]), f, m, interleaved)
        assert np.isclose(np.linalg.norm(x), np.linalg.norm(a)) and np.array_equal(x[..., 32:], a[..., 32:])
        dots.append(float(np.sum(x * y)))
    assert np.allclose(dots, dots[0])


def test_yarn_keeps_fast_pairs_and_divides_slow_ones():
    f0, _ = to.rope_frequencies(128, 1e6)
    f, m = to.rope_frequencies(128, 1e6, "yarn", 4.0, 32768)
    assert np.isclose(f[0], f0[0]) and np.isclose(f[-1], f0[-1] / 4) and np.all(np.diff(f / f0) <= 1e-15) and m > 1
    g, _ = to.rope_frequencies(128, 1e6, "ntk", 4.0)
    assert np.isclose(g[0], f0[0]) and np.isclose(g[-1], f0[-1] / 4)   # the last pair is stretched by the whole factor


def test_a_chain_is_causal_attention_and_siblings_do_not_see_each_other():
    rng = np.random.default_rng(2)
    n, d = 5, 8
    q, k, v = (rng.normal(size=(n, 1, d)) for _ in range(3))
    kc, vc = rng.normal(size=(3, 1, d)), rng.normal(size=(3, 1, d))
    chain, _ = to.tree_attention(q, kc, vc, k, v, [-1, 0, 1, 2, 3], 0.3)
    allk, allv = np.concatenate([kc, k]), np.concatenate([vc, v])
    for j in range(n):
        s = allk[:4 + j, 0] @ q[j, 0] * 0.3
        p = np.exp(s) / np.exp(s).sum()
        assert np.allclose(chain[j, 0], p @ allv[:4 + j, 0])
    star, _ = to.tree_attention(q, kc, vc, k, v, [-1] * n, 0.3)
    alone, _ = to.tree_attention(q[3:4], kc, vc, k[3:4], v[3:4], [-1], 0.3)
    assert np.allclose(star[3], alone[0])
    empty, _ = to.tree_attention(q[:1], kc[:0], vc[:0], k[:1], v[:1], [-1], 0.3)
    assert np.allclose(empty, v[:1])


def test_walk_takes_the_lowest_matching_child():
    parent = [-1, 0, 0, 0, 2, 2, 4]
    draft = [9, 5, 7, 7, 1, 3, 2]
    decided = [7, 0, 3, 3, 2, 8, 8]
    assert to.tree_walk(parent, draft, decided, 7) == [0, 2, 5]     # twin 3 is not taken
    assert to.tree_walk(parent, draft, decided, 5) == [0, 2]
    assert to.tree_walk(parent, draft, [5] * 7, 7) == [0, 1]
    assert to.tree_walk(parent, draft, [5] * 7, 0) == []
    assert to.tree_path([3, 0, 2, 1], 3) == [3, 1, 0] and to.tree_path([3, 0, 2, 1], 2) == [2]


def test_sampling_draws_each_token_as_often_as_its_weight():
    l = np.array([0.0, 1.0, -np.inf, 2.0, np.nan, 1.0], dtype=np.float32)
    w = np.exp(np.array([0.0, 1.0, 2.0, 1.0]))
    counts = np.zeros(6)
    for i in range(4000):
        counts[to.sample(l, (i + 0.5) / 4000)[0]] += 1
    assert np.allclose(counts[[0, 1, 3, 5]] / 4000, w / w.sum(), atol=3e-4) and counts[2] == counts[4] == 0


@pytest.mark.parametrize("kw,kept", [(dict(top_k=1), {3}), (dict(top_k=2), {3, 1}), (dict(top_k=3), {3, 1, 5}),
                                     (dict(temperature=0.0), {3}), (dict(top_p=0.0), {3}), (dict(top_p=0.5), {3}), (dict(top_p=0.6), {3, 1}),
                                     (dict(top_k=2, top_p=0.99), {3, 1}), (dict(min_p=0.3), {3, 1, 5}), (dict(min_p=2.0), {3})])
def test_filters_keep_a_prefix_with_ties_by_index(kw, kept):
    l = np.array([0.0, 1.0, -np.inf, 2.0, np.nan, 1.0], dtype=np.float32)
    got = {to.sample(l, u, **kw)[0] for u in np.linspace(0, 0.9999, 200)}
    assert got == kept and to.sample(l, 0.5, **kw)[3] == len(kept)


def test_sampling_from_nothing():
    assert to.sample(np.full(4, -np.inf), 0.5)[:4] == (-1, 0.0, 0.0, 0)
