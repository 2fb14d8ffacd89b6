"""How the tree and sampling calls are made: on a stream that is not the current one, on the wrong GPU, captured and
replayed with changed inputs, with the same slot in several rows."""
import pytest
import torch

import paper_2509_24007_b200 as pk

pytestmark = pytest.mark.gpu

HQ, HKV, D, N, V = 8, 2, 64, 7, 5000  # heads, head size, nodes, vocabulary


@pytest.fixture(scope="module")
def filled():
    """A context with three cached sequences; the largest magnitude of their values in `v_max`."""
    sd = pk.Sdlm(pk.SdlmConfig(HQ, HKV, D, 64, 64, 40, 4, 8, max_block=8))
    g = torch.Generator("cuda").manual_seed(3)
    sd.v_max = 0.0
    for b, m in enumerate([70, 8, 130]):
        k, v = (torch.randn((m, HKV, D), device="cuda", generator=g).bfloat16() for _ in range(2))
        sd.kv_add_seq(b, k, v)
        sd.v_max = max(sd.v_max, v.abs().max().item())
    return sd


def _tree(B, seed=5):
    g = torch.Generator("cuda").manual_seed(seed)
    r = lambda h: torch.randn((B, N, h, D), device="cuda", generator=g).bfloat16()
    parent = torch.tensor([[-1, 0, 0, 1, 1, 2, 5]] * B, dtype=torch.int32, device="cuda")
    return r(HQ), r(HKV), r(HKV), parent


def test_outputs_made_on_another_stream(filled):
    """Rows behind a sequence's nodes are cleared on the stream the kernel runs on, not on the current one."""
    q, kt, vt, parent = _tree(3)
    nodes = torch.tensor([7, 4, 1], dtype=torch.int32, device="cuda")
    ref = filled.tree_attn(q, kt, vt, parent, n_nodes=nodes)
    logits, u = torch.randn((3, V), device="cuda"), torch.rand(3, device="cuda")
    ref_s = filled.sample(logits, u)
    r = filled.qk_norm_rope(q, kt, pk.RopeConfig())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)                     # the current stream is busy for some milliseconds
    out = filled.tree_attn(q, kt, vt, parent, n_nodes=nodes, stream=side)
    got = filled.sample(logits, u, stream=side)
    rot = filled.qk_norm_rope(q, kt, pk.RopeConfig(), stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, ref)
    assert (out[1, 4:] == 0).all() and (out[2, 1:] == 0).all()
    for a, b in zip(got + rot, ref_s + r):
        assert torch.equal(a, b)


def test_tensors_of_another_gpu_are_refused(filled, monkeypatch):
    q, kt, vt, parent = _tree(3)
    monkeypatch.setattr(filled, "device_index", filled.device_index + 1)
    for call in (lambda: filled.tree_attn(q, kt, vt, parent), lambda: filled.qk_norm_rope(q, kt, pk.RopeConfig()),
                 lambda: filled.tree_attn(q=q, k_tree=kt, v_tree=vt, parent=parent),
                 lambda: filled.tree_commit(parent, parent, parent, kt, vt), lambda: filled.kv_gather_batch(kt, vt),
                 lambda: pk.tree_commit_layers([filled], parent, parent, parent, [kt], [vt]),
                 lambda: filled.sample(torch.zeros((1, 8), device="cuda"), torch.zeros(1, device="cuda"))):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_one_slot_in_every_row(filled):
    """Attention may name a slot several times: every row gives what it gives alone."""
    q, kt, vt, parent = _tree(4)
    ids = torch.tensor([2, 2, 0, 2], dtype=torch.int32, device="cuda")
    out = filled.tree_attn(q, kt, vt, parent, seq_ids=ids)
    for b in range(4):
        one = filled.tree_attn(q[b:b + 1].contiguous(), kt[b:b + 1].contiguous(), vt[b:b + 1].contiguous(), parent[b:b + 1],
                               seq_ids=ids[b:b + 1])
        # the keys are split over the thread blocks differently: each call rounds every weight to bf16 (2^-8 of it: at most
        # 2^-8 of the largest value in the result) and its result once
        assert (out[b].float() - one[0].float()).abs().max() <= 4 * 2.0 ** -8 * max(filled.v_max, vt.abs().max().item())


def test_captured_pass_follows_its_inputs(filled):
    """Attention, sampling and the walk captured once and replayed: trees, numbers and lengths are read on the device."""
    q, kt, vt, parent = _tree(3)
    logits, u = torch.randn((3, N, V), device="cuda"), torch.rand((3, N), device="cuda")
    out = torch.zeros_like(q)
    token = torch.zeros((3, N), dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        filled.tree_attn(q, kt, vt, parent, out=out)
        filled.sample(logits, u, token=token)
    for seed in (1, 2):
        q2, k2, v2, _ = _tree(3, seed)
        q.copy_(q2); kt.copy_(k2); vt.copy_(v2)
        parent.copy_(torch.tensor([[-1, 0, 1, 2, 3, 4, 5], [-1, -1, -1, 0, 0, 0, 0], [-1, 0, 0, 0, 3, 3, 3]][seed:] +
                                  [[-1] * N] * seed, dtype=torch.int32))
        logits.copy_(torch.randn((3, N, V), device="cuda")); u.copy_(torch.rand((3, N), device="cuda"))
        g.replay()
        assert torch.equal(out, filled.tree_attn(q, kt, vt, parent))
        assert torch.equal(token, filled.sample(logits, u)[0])
    g.reset()


def test_outputs_in_place_of_inputs_are_refused(filled):
    q, kt, vt, parent = _tree(3)
    tok, nxt = torch.zeros_like(parent), torch.ones_like(parent)
    before = filled.launch_count()
    wide = torch.zeros((2, *q.shape), dtype=torch.bfloat16, device="cuda").view(-1)[:q.numel() + 64]
    for call in (lambda: filled.tree_attn(q, kt, vt, parent, out=q),
                 lambda: filled.tree_attn(wide[64:].view(q.shape), kt, vt, parent, out=wide[:-64].view(q.shape)),
                 lambda: filled.tree_commit(tok, nxt, parent, kt, vt, out_tokens=nxt),
                 lambda: filled.tree_commit(tok, nxt, parent, kt, vt, path=parent),
                 lambda: filled.tree_commit(tok, nxt, parent, kt, vt, out_tokens=(t := torch.zeros_like(tok)), path=t),
                 lambda: pk.tree_commit_layers([filled], tok, nxt, parent, [kt], [vt], out_tokens=tok)):
        with pytest.raises(pk.SdlmError) as e:
            call()
        assert e.value.code == 1
    torch.cuda.synchronize()
    assert filled.launch_count() == before
