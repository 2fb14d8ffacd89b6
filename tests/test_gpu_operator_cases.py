"""The measured cases of the tree and sampling operators: inputs follow from case and seed alone, and on the same inputs the
library gives what the plain form gives."""
import random

import pytest
import torch

from perf import operators as ops

pytestmark = pytest.mark.gpu


def _cases():
    small = [c for c in ops.listed() if c["name"] in ("rope_token", "rope_tree", "tree_token", "tree_batch", "sample_row", "sample_batch",
                                                      "commit_one", "commit_batch")]
    tiny = [dict(op="sample", shape="tiny", rows=256, dtype=t, peak=p, filters=f, banned=b)
            for t, p, f, b in (("bf16", 4.0, "all", True), ("fp32", 8.0, "all", False), ("bf16", 6.0, "top_p", False), ("fp32", 6.0, "top_k", True))]
    rng, drawn = random.Random(7), []
    for op, n in (("rope", 3), ("tree", 3), ("sample", 4), ("commit", 3)):
        of = []
        while len(of) < n:
            c = ops._drawn(rng, op)
            if ops.work(c)["bytes"] < 1e8 and ops.work(c)["flops"] < 1e11:
                of.append(c)
        drawn += of
    return small + tiny + drawn


CASES = _cases()


def _leaves(state):
    return {k: v for k, v in state.items() if isinstance(v, torch.Tensor)}


@pytest.mark.parametrize("i", range(len(CASES)), ids=[c.get("name", f"{c['op']}{i}") for i, c in enumerate(CASES)])
def test_inputs_repeat_and_the_library_gives_what_the_plain_form_gives(i, monkeypatch):
    case = CASES[i]
    plain = _leaves(ops.prepare(case, 1000 + i))
    monkeypatch.setattr(ops, "own", True)
    state, again = ops.prepare(case, 1000 + i), ops.prepare(case, 1000 + i)
    other = ops.prepare(case, 2000 + i)
    name = {"rope": "q", "tree": "q", "sample": "logits", "commit": "kt"}[case["op"]]
    assert not torch.equal(state[name], other[name])
    del other
    for k, v in _leaves(state).items():
        if k not in ("out", "q_out", "k_out", "saved"):  # (what the calls write is not an input)
            assert torch.equal(v.view(torch.uint8) if v.is_contiguous() else v, again[k].view(torch.uint8) if v.is_contiguous() else again[k]), k
            if k in plain:
                assert torch.equal(v, plain[k]), k
    del plain
    got = ops.run(state)
    got = {"out": got} if isinstance(got, torch.Tensor) else got
    got = {k: v.clone() for k, v in got.items()}
    rerun = ops.run(again)
    rerun = {"out": rerun} if isinstance(rerun, torch.Tensor) else rerun
    assert all(torch.equal(got[k], rerun[k]) for k in got)
    monkeypatch.setattr(ops, "own", False)
    want = ops.run(state)
    want = {"out": want} if isinstance(want, torch.Tensor) else want
    largest = max(float(state[k].abs().max()) for k in ("vt", "vh") if state[k].numel()) if case["op"] == "tree" else 0.0
    for k, a in want.items():
        b = got[k]
        assert a.dtype == b.dtype and a.shape == b.shape
        if a.dtype == torch.int32 or case["op"] == "commit":
            assert torch.equal(a, b), k
        elif case["op"] == "sample":
            # weights good to 1e-11 a side, sums of them rounded to 2^-45 each (2e-9 at the most), one rounding to 32 bits a side
            assert bool(((a - b).abs() <= 2 * 2.0 ** -24 * a.abs() + 1e-7).all()), k
        elif case["op"] == "rope":
            # fp32 on both sides (norm, two products, a sum: 8 roundings of 2^-24 of numbers up to the row's largest), one
            # rounding to bf16 each
            size = a.float().abs().amax(-1, keepdim=True) * 2.0
            assert bool(((a.float() - b.float()).abs() <= 2 * 2.0 ** -8 * a.float().abs() + 16 * 2.0 ** -24 * size).all()), k
        else:
            # weights rounded to bf16 and powers of two, each in both sums (see test_gpu_tree.py; a weighted mean of |v| is at
            # most the largest), one rounding to bf16 each
            assert bool(((a.float() - b.float()).abs() <= 2 * 2.0 ** -8 * a.float().abs() + largest * (2.0 ** -7 + 6e-4)).all()), k
