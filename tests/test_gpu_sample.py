"""GPU parity of sampling from logits (sdlm_sample) with the float64 oracle."""
import math

import numpy as np
import pytest
import torch

import paper_2509_24007_b200 as pk
from oracle import sdlm_tree_oracle as to

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sd():
    return pk.Sdlm(pk.SdlmConfig(2, 1, 64, 64, 64, 4, 4, 4, max_block=8))


def _check(sd, logits, u, T=None, k=None, p=None, m=None, exact=False):
    """Every row against the oracle.  A token may differ only where the oracle itself is within 1e-9 of a border (the
    kernel's weights are good to 1e-11 and rounded to 2^-45, 2e-9 of the sum over 2^18 of them at the very most); nowhere
    with exact: weights that are whole numbers, whose sums both sides form without rounding."""
    dev = lambda x, dt: None if x is None else torch.as_tensor(np.asarray(x), dtype=dt, device="cuda")
    tok, prob, ent, kept = sd.sample(logits, dev(u, torch.float32), dev(T, torch.float32), dev(k, torch.int32),
                                     dev(p, torch.float32), dev(m, torch.float32))
    tok, prob, ent, kept = (x.cpu().numpy().reshape(-1) for x in (tok, prob, ent, kept))
    x = logits.float().cpu().numpy().reshape(-1, logits.shape[-1])
    u = np.broadcast_to(np.asarray(u, dtype=np.float32).reshape(-1), (len(x),))
    close = 0
    for r in range(len(x)):
        at = lambda a, default: default if a is None else np.asarray(a).reshape(-1)[r]
        t, q, e, n, near = to.sample(x[r], u[r], at(T, 1.0), int(at(k, 0)), at(p, 1.0), at(m, 0.0))
        if near < 1e-9 and not exact:
            close += 1
            continue
        assert (tok[r], kept[r]) == (t, n), (r, tok[r], t, kept[r], n, near)
        assert abs(prob[r] - q) <= 2.0 ** -23 * q + 1e-9 and abs(ent[r] - e) <= 2.0 ** -22 * e + 1e-7
    assert close <= max(1, len(x) // 20)
    return tok


def _params(rng, R):
    return dict(T=rng.uniform(0.5, 1.5, R), k=rng.choice([0, 1, 2, 7, 50, 400, 10 ** 6, -3], R),
                p=rng.choice([0.0, 0.1, 0.5, 0.9, 0.99, 1.0, 1.5], R), m=rng.choice([0.0, 0.01, 0.2, 1.0, 3.0], R))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 100, 1023, 1024, 4099, 8192, 8193, 20011, 33000, 151936])
def test_every_filter_over_sizes(sd, dtype, V):
    rng = np.random.default_rng(V)
    R = 24 if V < 50000 else 6
    logits = torch.from_numpy((rng.normal(size=(R, V)) * 3).astype(np.float32)).cuda().to(dtype)
    u = rng.random(R)
    _check(sd, logits, u)
    _check(sd, logits, u, **_params(rng, R))
    for one in ("k", "p", "m"):
        _check(sd, logits, u, **{one: _params(rng, R)[one]})
    assert sd.device_status()[0] == 0


def test_the_largest_vocabulary(sd):
    rng = np.random.default_rng(9)
    for dtype in (torch.bfloat16, torch.float32):
        logits = torch.from_numpy(rng.normal(size=(3, 1 << 18)).astype(np.float32)).cuda().to(dtype)
        _check(sd, logits, rng.random(3), p=[0.5, 0.9, 1.0], k=[0, 100000, 0])
    with pytest.raises(pk.SdlmError) as e:
        sd.sample(torch.zeros((1, (1 << 18) + 1), dtype=torch.bfloat16, device="cuda"), torch.zeros(1, device="cuda"))
    assert e.value.code == 3


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ties_go_to_the_lowest_index(sd, dtype):
    V = 9001
    logits = torch.zeros((40, V), dtype=dtype, device="cuda")
    u = (np.arange(40) + 0.5) / 40
    tok = _check(sd, logits, u, exact=True)
    assert np.array_equal(tok, np.floor(u * V))
    tok = _check(sd, logits, u, k=np.full(40, 10), exact=True)
    assert np.array_equal(tok, np.arange(40) // 4)
    _check(sd, logits, u, p=np.full(40, 0.25), k=np.full(40, 1000), exact=True)
    assert np.array_equal(_check(sd, logits, u, T=np.zeros(40)), np.zeros(40))
    logits[:, ::2] = -1.0
    logits[:, 5] = logits[:, 7001] = 2.0
    logits[:, 100] = -0.0
    assert set(_check(sd, logits, u, k=np.full(40, 2))) == {5, 7001}
    _check(sd, logits, u, k=np.full(40, 5))     # 0 and -0 are one value
    _check(sd, logits, u, p=np.full(40, 0.3))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masked_tokens_infinities_and_nan(sd, dtype):
    rng = np.random.default_rng(11)
    V, R = 5003, 16
    x = (rng.normal(size=(R, V)) * 2).astype(np.float32)
    x[:, rng.choice(V, 4000, replace=False)] = -np.inf
    x[3, :] = -np.inf                                  # nothing left
    x[4, :] = np.nan
    x[5, :] = -np.inf
    x[5, 4999] = -30.0                                 # one left
    x[6, ::3] = np.nan
    x[7, ::2] = float(torch.finfo(dtype).min)          # masks of the type's lowest value
    x[8, :] = float(torch.finfo(dtype).min)
    x[9, [17, 400]] = np.inf
    x[10, 2500] = np.inf
    x[11, :] = 1e-30
    logits = torch.from_numpy(x).cuda().to(dtype)
    ref = logits.clone()
    ref[ref == math.inf] = torch.finfo(dtype).max      # +inf counts as the largest finite value
    u = rng.random(R)
    for kw in ({}, dict(p=np.full(R, 0.8)), dict(k=np.full(R, 900)), dict(T=np.full(R, 1e-3)), dict(T=np.zeros(R)),
               dict(k=np.full(R, 3), p=np.full(R, 0.6), m=np.full(R, 0.1))):
        a = _check(sd, ref, u, **kw)
        dev = {n: torch.as_tensor(v, dtype=torch.int32 if n == "k" else torch.float32, device="cuda") for n, v in kw.items()}
        b = sd.sample(logits, torch.as_tensor(u, dtype=torch.float32, device="cuda"), dev.get("T"), dev.get("k"), dev.get("p"))[0]
        if "m" not in kw:
            assert np.array_equal(a, b.cpu().numpy())
        assert a[3] == a[4] == -1 and a[5] == 4999


def test_temperatures_from_tiny_to_infinite(sd):
    rng = np.random.default_rng(12)
    T = [1e-45, 1e-30, 1e-6, 0.01, 100.0, 1e30, math.inf, -1.0, math.nan, 0.0]
    logits = torch.from_numpy((rng.normal(size=(len(T), 3001)) * 5).astype(np.float32)).cuda()
    u = rng.random(len(T))
    _check(sd, logits, u, T=T)
    _check(sd, logits, u, T=T, p=np.full(len(T), 0.7), k=np.full(len(T), 1500))
    _check(sd, logits.to(torch.bfloat16), u, T=T, p=np.full(len(T), 0.7))


def test_random_numbers_at_the_ends(sd):
    logits = torch.randn((5, 1000), device="cuda")
    u = np.array([0.0, 1.0 - 2.0 ** -24, 2.0 ** -149, 0.5, 0.999], dtype=np.float32)
    _check(sd, logits, u)
    tok = sd.sample(logits[:3].contiguous(), torch.tensor([-1.0, 1.0, math.nan], device="cuda"))[0]
    assert tok.tolist() == [0, 999, 0]       # outside [0, 1): held at its ends


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strided_and_unaligned_rows(sd, dtype):
    rng = np.random.default_rng(13)
    wide = torch.from_numpy((rng.normal(size=(6, 20017)) * 3).astype(np.float32)).cuda().to(dtype)
    u = rng.random(6)
    for view in (wide[:, 1:20010], wide[:, 8:16008], wide[:, :777]):
        _check(sd, view, u, p=np.full(6, 0.9), k=np.full(6, 300))
    _check(sd, wide[::2], u[:3])
    _check(sd, wide[:, :20016].reshape(2, 3, 20016)[..., :20016].contiguous(), u)


def test_confidences_feed_the_commit(sd):
    """token / prob / entropy of sampled block positions go into sdlm_accept_commit as they are."""
    D = 4
    rng = np.random.default_rng(14)
    logits = torch.from_numpy((rng.normal(size=(2, D, 64)) * 4).astype(np.float32)).cuda().to(torch.bfloat16)
    u = torch.from_numpy(rng.random((2, D)).astype(np.float32)).cuda()
    tok, prob, ent, _ = sd.sample(logits, u, top_k=torch.full((2, D), 8, dtype=torch.int32, device="cuda"))
    kv = torch.randn((2, D, 1, 64), device="cuda").to(torch.bfloat16)
    acc, out = sd.accept_commit(0.2, tok, prob, ent, kv, kv)
    c = np.cumprod(prob.cpu().numpy(), axis=1)
    for b in range(2):
        g = max([j + 1 for j in range(D) if c[b, j] >= 0.2] + [1])
        assert acc[b].item() == g and out[b, :g].tolist() == tok[b, :g].tolist()


def test_same_bits_on_every_run_and_in_a_graph(sd):
    rng = np.random.default_rng(15)
    logits = torch.from_numpy((rng.normal(size=(64, 152064))).astype(np.float32)).cuda()
    u = torch.from_numpy(rng.random(64).astype(np.float32)).cuda()
    p = torch.full((64,), 0.9, device="cuda")
    first = sd.sample(logits, u, top_p=p)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, sd.sample(logits, u, top_p=p)))
    out = [torch.zeros_like(x) for x in first]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sd.sample(logits, u, top_p=p, token=out[0], prob=out[1], entropy=out[2], n_kept=out[3])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, out))


def test_refusals(sd):
    lib, st = sd.lib, torch.cuda.current_stream().cuda_stream
    x, u = torch.zeros((2, 64), device="cuda"), torch.zeros(2, device="cuda")
    tok = torch.full((2,), 7, dtype=torch.int32, device="cuda")
    pr, en = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")

    def call(rows=2, V=64, type=1, l=x.data_ptr(), ld=64, u=u.data_ptr(), t=tok.data_ptr(), p=pr.data_ptr(), e=en.data_ptr()):
        return lib.sdlm_sample(sd.ctx, rows, V, type, l, ld, u, None, None, None, None, t, p, e, None, st)

    before = sd.launch_count()
    assert call(rows=0) == call(V=0) == call(type=2) == call(ld=63) == call(l=None) == call(u=None) == call(t=None) == 1
    assert call(p=None) == call(e=None) == call(l=x.data_ptr() + 2) == 1
    assert call(V=300000, ld=300000) == 3 and call(rows=1 << 28) == 2
    torch.cuda.synchronize()
    assert sd.launch_count() == before and tok.tolist() == [7, 7]
    for bad in (dict(u=u.double()), dict(top_k=u), dict(temperature=torch.ones(3, device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            sd.sample(x, **{"u": u, **bad})
    with pytest.raises(TypeError):
        sd.sample(x.half(), u)
    with pytest.raises(TypeError):
        sd.sample(x.t(), torch.zeros(64, device="cuda"))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_top_k_around_the_length_of_the_list(sd, dtype):
    """Few tokens kept by top-k are listed and only the list is looked at again; more are not.  Both, with every other
    filter behind them, on random rows, on rows of a few values (more ties than the list has room for), and again with the
    same bits although a list has no fixed order."""
    rng = np.random.default_rng(16)
    V = 40000
    x = (rng.normal(size=(16, V)) * 2).astype(np.float32)
    x[8:] = np.round(x[8:])
    logits = torch.from_numpy(x).cuda().to(dtype)
    u = rng.random(16)
    k = np.array([3, 50, 1000, 1024, 1025, 2048, 2049, 5000] * 2)
    for kw in (dict(), dict(p=np.full(16, 0.8)), dict(m=np.full(16, 0.05)), dict(p=np.full(16, 0.95), m=np.full(16, 0.02))):
        _check(sd, logits, u, k=k, **kw)
    dev = lambda a, dt: torch.as_tensor(a, dtype=dt, device="cuda")
    args = (logits, dev(u, torch.float32), None, dev(k, torch.int32), dev(np.full(16, 0.9), torch.float32), dev(np.full(16, 0.03), torch.float32))
    first = sd.sample(*args)
    for _ in range(4):
        assert all(torch.equal(a, b) for a, b in zip(first, sd.sample(*args)))
