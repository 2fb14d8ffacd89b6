"""GPU parity of the rotary embedding with per-head norms (sdlm_qk_norm_rope) with the float64 oracle."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2509_24007_b200 as pk
from oracle import sdlm_tree_oracle as to

pytestmark = pytest.mark.gpu
KIND = {"plain": pk.ROPE_PLAIN, "linear": pk.ROPE_LINEAR, "ntk": pk.ROPE_NTK, "yarn": pk.ROPE_YARN}


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _sd(d, max_batch=8, lens=()):
    sd = pk.Sdlm(pk.SdlmConfig(2, 1, d, 64, 64, 40, max_batch, 8, max_block=8))
    for b, x in enumerate(lens):
        if x:
            z = torch.zeros((x, 1, d), dtype=torch.bfloat16, device="cuda")
            sd.kv_add_seq(b, z, z)
    return sd


def _rand(*shape, mean=0.0, std=1.0):
    return (torch.randn(shape, device="cuda") * std + mean).to(torch.bfloat16)


def _check(x, got, pos, rope, scaling, d, weight=None, eps=1e-6):
    rot = rope.rot_dim or d
    f, m = to.rope_frequencies(rot, rope.theta, scaling, rope.factor, rope.trained_len, rope.beta_fast, rope.beta_slow)
    if rope.attn_factor:
        m = float(np.float32(rope.attn_factor))
    shape = x.shape
    ref, size = to.norm_rope(_f64(x).reshape(-1, shape[2], d), np.asarray(pos).reshape(-1), f, m, rope.interleaved,
                             None if weight is None else _f64(weight), eps)
    err = np.abs(_f64(got).reshape(ref.shape) - ref)
    # one rounding to bf16; before it some ten fp32 operations on values of the pair's size, sine and cosine (2^-22)
    bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -20 * size
    assert np.all(np.isfinite(err)) and np.all(err <= bound), float(np.max(err / (bound + 1e-300)))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [16, 32, 48, 0])
@pytest.mark.parametrize("scaling", ["plain", "linear", "ntk", "yarn"])
def test_layouts_parts_and_scalings(d, interleaved, rot, scaling):
    torch.manual_seed(rot + d)
    sd = _sd(d)
    q, k = _rand(3, 5, 7, d), _rand(3, 5, 2, d)
    wq, wk = _rand(d, mean=1.0, std=0.3), _rand(d, mean=1.0, std=0.3)
    pos = torch.randint(0, 200000, (3, 5), dtype=torch.int32, device="cuda")
    rope = pk.RopeConfig(theta=1000000.0, rot_dim=rot, interleaved=interleaved, scaling=KIND[scaling], factor=4.0)
    qo, ko = sd.qk_norm_rope(q, k, rope, positions=pos, q_weight=wq, k_weight=wk)
    _check(q, qo, pos.cpu(), rope, scaling, d, wq)
    _check(k, ko, pos.cpu(), rope, scaling, d, wk)
    qo, ko = sd.qk_norm_rope(q, k, rope, positions=pos, k_weight=wk)  # a norm of the keys alone
    _check(q, qo, pos.cpu(), rope, scaling, d)
    _check(k, ko, pos.cpu(), rope, scaling, d, wk)
    assert sd.device_status()[0] == 0


@pytest.mark.parametrize("batch,D,hq,hk", [(1, 1, 1, 1), (1, 1, 16, 2), (2, 1, 40, 8), (32, 21, 16, 2), (1, 2049, 5, 1), (8, 700, 4, 4)])
def test_sizes(batch, D, hq, hk):
    torch.manual_seed(batch * D)
    sd = _sd(128, max_batch=32)
    q, k = _rand(batch, D, hq, 128), _rand(batch, D, hk, 128)
    w = _rand(128, mean=1.0, std=0.2)
    pos = torch.randint(-50, 3000, (batch, D), dtype=torch.int32, device="cuda")
    rope = pk.RopeConfig(theta=10000.0)
    qo, ko = sd.qk_norm_rope(q, k, rope, positions=pos, q_weight=w, k_weight=w, eps=1e-5)
    _check(q, qo, pos.cpu(), rope, "plain", 128, w, 1e-5)
    _check(k, ko, pos.cpu(), rope, "plain", 128, w, 1e-5)


def test_far_positions_and_the_attention_factor():
    sd = _sd(64)
    q = _rand(1, 4, 3, 64)
    pos = torch.tensor([[2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 0]], dtype=torch.int32, device="cuda")
    rope = pk.RopeConfig(theta=500000.0, attn_factor=1.25)
    qo, none = sd.qk_norm_rope(q, None, rope, positions=pos)
    assert none is None
    # 2^31 turns of a 64-bit frequency leave 2^31 * 2^-53 * 2 pi of angle: 1.5e-6 of the pair
    f, _ = to.rope_frequencies(64, 500000.0)
    ref, size = to.norm_rope(_f64(q)[0], pos.cpu().numpy()[0], f, 1.25, False)
    assert np.all(np.abs(_f64(qo)[0] - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -20 + 4e-6) * size)


def test_positions_count_from_the_cached_lengths():
    sd = _sd(64, lens=(5, 0, 100))
    q, k = _rand(3, 4, 2, 64), _rand(3, 4, 1, 64)
    depth = torch.tensor([[0, 1, 1, 2], [0, 0, 0, 1], [3, 2, 1, 0]], dtype=torch.int32, device="cuda")
    rope = pk.RopeConfig(theta=10000.0, interleaved=True)
    for ids in ([0, 1, 2], [2, 2, 0]):
        lens = np.array([[5, 0, 100][i] for i in ids])[:, None]
        t = torch.tensor(ids, dtype=torch.int32, device="cuda")
        qo, ko = sd.qk_norm_rope(q, k, rope, positions=depth, relative=True, seq_ids=t)
        _check(q, qo, lens + depth.cpu().numpy(), rope, "plain", 64)
        qo, ko = sd.qk_norm_rope(q, k, rope, seq_ids=t)
        _check(k, ko, lens + np.arange(4), rope, "plain", 64)
    # whole heads, rotate-half, behind the history: what sdlm_rope_block computes
    rope = pk.RopeConfig(theta=10000.0)
    qo, _ = sd.qk_norm_rope(q, None, rope)
    old = sd.rope_block(q.clone(), 10000.0)
    assert float((qo.float() - old.float()).abs().max()) <= 2.0 ** -6 * 4


def test_strided_rows_and_in_place():
    torch.manual_seed(3)
    sd = _sd(128)
    qkv = _rand(2, 9, 8, 128)  # 4 query heads, 2 key heads, 2 value heads
    keep = qkv.clone()
    pos = torch.randint(0, 4000, (2, 9), dtype=torch.int32, device="cuda")
    rope = pk.RopeConfig(theta=10000.0, rot_dim=64)
    qo, ko = sd.qk_norm_rope(qkv[:, :, :4], qkv[:, :, 4:6], rope, positions=pos)
    assert torch.equal(qkv, keep)
    _check(keep[:, :, :4], qo, pos.cpu(), rope, "plain", 128)
    _check(keep[:, :, 4:6], ko, pos.cpu(), rope, "plain", 128)
    q, k = keep[:, :, :4].contiguous(), keep[:, :, 4:6].contiguous()
    sd.qk_norm_rope(q, k, rope, positions=pos, q_out=q, k_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    one, _ = sd.qk_norm_rope(keep[1:, 3:4, 2:3], None, rope, positions=pos[1:, 3:4].contiguous())
    assert torch.equal(one[0, 0, 0], qo[1, 3, 2])


def test_zero_rows_and_large_values():
    sd = _sd(64)
    q = torch.zeros((1, 3, 2, 64), dtype=torch.bfloat16, device="cuda")
    q[0, 1] = 1e18   # squares overflow bf16, not fp32
    q[0, 2] = 1e-18
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    rope = pk.RopeConfig(theta=10000.0)
    qo, _ = sd.qk_norm_rope(q, None, rope, q_weight=w)
    _check(q, qo, np.arange(3)[None], rope, "plain", 64, w)


def test_a_bad_slot_is_reported_and_its_rows_left_alone():
    sd = _sd(64, lens=(5,))
    q = _rand(2, 3, 2, 64)
    out = torch.full_like(q, 7.0)
    sd.qk_norm_rope(q, None, pk.RopeConfig(theta=10000.0), seq_ids=torch.tensor([0, 8], dtype=torch.int32, device="cuda"), q_out=out)
    st = sd.device_status(clear=True)
    assert st[0] == 7 and st[1] == 8 and bool((out[1] == 7.0).all())
    _check(q[:1], out[:1], 5 + np.arange(3)[None], pk.RopeConfig(theta=10000.0), "plain", 64)


def test_capture_and_another_stream():
    sd = _sd(128, lens=(64,))
    q, k = _rand(1, 8, 16, 128), _rand(1, 8, 2, 128)
    rope = pk.RopeConfig()
    qo, ko = sd.qk_norm_rope(q, k, rope)
    q2, k2 = torch.zeros_like(q), torch.zeros_like(k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sd.qk_norm_rope(q, k, rope, q_out=q2, k_out=k2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(q2, qo) and torch.equal(k2, ko)


@pytest.mark.parametrize("bad,code", [(dict(rot_dim=24), 3), (dict(rot_dim=80), 1), (dict(rot_dim=-16), 1), (dict(theta=1.0), 1),
                                      (dict(theta=float("nan")), 1), (dict(scaling=4), 1), (dict(scaling=1, factor=0.0), 1),
                                      (dict(scaling=3, factor=2.0, trained_len=0), 1), (dict(scaling=3, factor=2.0, beta_fast=0.0), 1),
                                      (dict(attn_factor=-1.0), 1)])
def test_refused_rotations(bad, code):
    sd = _sd(64)
    q = _rand(1, 2, 2, 64)
    before = sd.launch_count()
    with pytest.raises(pk.SdlmError) as e:
        sd.qk_norm_rope(q, None, pk.RopeConfig(**bad))
    assert e.value.code == code and sd.launch_count() == before


def test_refused_buffers():
    sd = _sd(64, max_batch=2)
    lib, st = sd.lib, torch.cuda.current_stream().cuda_stream
    q, k = _rand(2, 3, 4, 64), _rand(2, 3, 2, 64)
    out, kout = torch.empty_like(q), torch.empty_like(k)
    r = pk.RopeConfig().to_c()

    def call(batch=2, D=3, heads=4, qp=q.data_ptr(), qs=256, qo=out.data_ptr(), heads2=2, kp=k.data_ptr(), ks=128, ko=kout.data_ptr(),
             pos=None, rel=0, eps=1e-6, rope=C.byref(r)):
        return lib.sdlm_qk_norm_rope(sd.ctx, batch, D, None, pos, rel, rope, eps, heads, qp, qs, None, qo, heads2, kp, ks, None, ko, st)

    before = sd.launch_count()
    assert call(batch=0) == call(D=0) == call(heads=0) == call(heads2=-1) == 1
    assert call(qp=None) == call(qo=None) == call(kp=None) == call(ko=None) == call(rope=None) == 1
    assert call(qp=q.data_ptr() + 2) == call(qs=255) == call(qs=260) == call(ks=120) == 1
    assert call(eps=-1.0) == call(eps=float("nan")) == 1
    assert call(batch=3) == 2                                        # slots are read: no more than max_batch
    assert call(qo=q.data_ptr() + 64) == 1                           # an overlap that is not in place
    assert call(D=1, qs=512, qo=q.data_ptr()) == 1                   # in place with strided rows
    assert call(ko=out.data_ptr()) == call(ko=q.data_ptr()) == call(qo=k.data_ptr()) == 1
    assert sd.launch_count() == before
    with pytest.raises(TypeError):
        sd.qk_norm_rope(q.transpose(1, 2), None, pk.RopeConfig())
    with pytest.raises(TypeError):
        sd.qk_norm_rope(q.float(), None, pk.RopeConfig())
    with pytest.raises(ValueError):
        sd.qk_norm_rope(q, k[:1], pk.RopeConfig())
