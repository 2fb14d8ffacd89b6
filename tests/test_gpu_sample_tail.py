"""top-p whose border lies among a quarter of a million tokens of weight e^-20, where the bins by distance end."""
import numpy as np
import pytest
import torch

import paper_2509_24007_b200 as pk

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    return pk.Sdlm(pk.SdlmConfig(2, 1, 64, 64, 64, 4, 4, 4, max_block=8))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("low,high", [(-19.97, -19.97), (-19.99, -19.9), (-20.5, -19.5), (-19.0, -18.0), (-22.0, -19.0)])
def test_borders_in_the_thin_tail(sd, dtype, low, high):
    V, R = 1 << 18, 12
    rng = np.random.default_rng(5)
    x = rng.uniform(low, high, (R, V)).astype(np.float32)
    x[:, 777] = 0.0
    logits = torch.from_numpy(x).cuda().to(dtype)
    T = np.float32(1.25 if dtype == torch.float32 else 1.0)
    logits = logits if T == 1.0 else logits * float(T)
    x = logits.double().cpu().numpy() / float(T)
    w = np.exp(x)
    total = w.sum(1)
    p = (1.0 - (total - 1.0) / total * np.linspace(0.02, 0.98, R)).astype(np.float32)  # p reaches into the tail by different shares
    k = np.array([0, 200000, 0, 100000] * (R // 4), dtype=np.int32)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    u = rng.random(R).astype(np.float32)
    tok, prob, ent, kept = (a.cpu().numpy() for a in sd.sample(logits, dev(u), dev(np.full(R, T)), dev(k), dev(p)))
    for r in range(R):
        v = np.sort(w[r])[::-1][:k[r] or V]
        n = max(1, int(np.count_nonzero(np.concatenate(([0.0], np.cumsum(v)[:-1])) < float(p[r]) * v.sum())))
        # Sums: each weight of e^-20 or less is rounded to 2^-45, by 2^-46 / e^-22 (5e-5) of it at the most, on either side of
        # the border; p is exact in the goal.  So the border may move by that share of the kept and of the left tokens.
        assert abs(int(kept[r]) - n) <= 2 + 2 * 5.2e-5 * len(v), (r, kept[r], n)
        mass = v[:n].sum()
        assert abs(prob[r] - w[r, tok[r]] / mass) <= 1e-6 * prob[r] + 1e-12
        assert w[r, tok[r]] >= v[min(len(v), n + 30) - 1] * (1 - 1e-9)

