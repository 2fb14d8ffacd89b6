"""CPU-only refusals of the tree and sampling calls: at the C boundary without a context, and of the binding's own checks."""
import ctypes as C

import pytest
import torch

import paper_2509_24007_b200 as pk
from paper_2509_24007_b200 import binding, build

INVALID_ARG = 1


@pytest.fixture(scope="module")
def lib():
    build.build()
    return pk.load_library()


def test_calls_without_a_context_are_invalid(lib):
    buf = C.create_string_buffer(4096)
    p = C.addressof(buf)
    rope = binding.RopeConfig().to_c()
    assert lib.sdlm_qk_norm_rope(None, 1, 1, None, None, 0, C.byref(rope), 1e-6, 1, p, 128, None, p, 0, None, 0, None, None, None) == INVALID_ARG
    assert lib.sdlm_tree_attn(None, 1, 1, None, None, p, p, p, p, p, None) == INVALID_ARG
    assert lib.sdlm_tree_commit(None, 1, 1, None, None, p, p, p, p, p, p, p, p, None) == INVALID_ARG
    none = (C.c_void_p * 1)(None)
    one = (C.c_void_p * 1)(p)
    assert lib.sdlm_tree_commit_layers(none, 1, 1, 1, None, None, p, p, p, one, one, p, p, p, None) == INVALID_ARG
    assert lib.sdlm_tree_commit_layers(None, 1, 1, 1, None, None, p, p, p, one, one, p, p, p, None) == INVALID_ARG
    assert lib.sdlm_kv_gather_batch(None, 1, 1, None, p, p, None) == INVALID_ARG
    assert lib.sdlm_sample(None, 1, 16, 0, p, 16, p, None, None, None, None, p, p, p, None, None) == INVALID_ARG


class _Library:
    def __getattr__(self, name):
        def call(*args):
            raise AssertionError(f"{name} was called")
        return call


class _Context:
    """The binding's methods without a device; a call that reaches the library fails the test."""
    lib, ctx = _Library(), None
    cfg = pk.SdlmConfig(n_q_heads=4, n_kv_heads=2, head_dim=64, hidden=64, vocab=64, num_pages=4, max_batch=4,
                        max_pages_per_seq=4, max_block=4)
    device, device_index = torch.device("cuda", 0), 0
    _tree_shape = binding.Sdlm._tree_shape
    _tree_commit_args = binding.Sdlm._tree_commit_args


def test_host_tensors_are_refused():
    sd, bf16, i32 = _Context(), torch.bfloat16, torch.int32
    q, kv, idx = torch.zeros(1, 3, 4, 64, dtype=bf16), torch.zeros(1, 3, 2, 64, dtype=bf16), torch.zeros(1, 3, dtype=i32)
    with pytest.raises(TypeError):
        binding.Sdlm.qk_norm_rope(sd, q, kv, binding.RopeConfig())
    with pytest.raises(TypeError):
        binding.Sdlm.tree_attn(sd, q, kv, kv, idx)
    with pytest.raises(ValueError):
        binding.Sdlm.tree_attn(sd, q, kv, kv, idx[0])
    with pytest.raises(TypeError):
        binding.Sdlm.tree_commit(sd, idx, idx, idx, kv, kv)
    with pytest.raises(TypeError):
        binding.Sdlm.kv_gather_batch(sd, kv, kv)
    with pytest.raises(ValueError):
        binding.Sdlm.kv_gather_batch(sd, q, q)
    with pytest.raises(TypeError):
        binding.Sdlm.sample(sd, torch.zeros(2, 8), torch.zeros(2))
    with pytest.raises(ValueError):
        binding.tree_commit_layers([sd, sd], idx, idx, idx, [kv], [kv])


def test_rope_structure_follows_its_fields():
    r = binding.RopeConfig(theta=10000.0, rot_dim=32, interleaved=True)
    a = r.to_c()
    assert (a.theta, a.rot_dim, a.interleaved, a.scaling) == (10000.0, 32, 1, 0)
    assert r.to_c() is a
    r.scaling, r.factor = binding.ROPE_YARN, 4.0
    b = r.to_c()
    assert (b.scaling, b.factor, b.trained_len, b.beta_fast, b.beta_slow) == (3, 4.0, 32768, 32.0, 1.0)
