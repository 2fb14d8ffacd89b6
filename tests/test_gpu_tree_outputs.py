"""Outputs of the tree and sampling calls that lie over what is still read, and refusals of the commit one argument at a
time: each leaves the context and every buffer as they were."""
import pytest
import torch

import paper_2509_24007_b200 as pk
from test_gpu_tree import Tree

pytestmark = pytest.mark.gpu


def _refused(sd, call):
    before = sd.launch_count()
    with pytest.raises(pk.SdlmError) as e:
        call()
    assert e.value.code == 1 and sd.launch_count() == before


def _commit_tensors(t):
    i32 = dict(dtype=torch.int32, device="cuda")
    return dict(draft_token=torch.zeros((t.B, t.n), **i32), next_token=torch.ones((t.B, t.n), **i32), parent=t.parent,
                n_nodes=torch.full((t.B,), t.n, **i32), seq_ids=torch.arange(t.B, **i32),
                accepted_len=torch.full((t.B,), 7, **i32), out_tokens=torch.full((t.B, t.n), 7, **i32),
                path=torch.full((t.B, t.n), 7, **i32))


@pytest.mark.parametrize("layers", [False, True])
def test_commit_outputs_over_anything_else_are_refused(layers):
    t = Tree(4, 2, 64, [10, 20, 0], 4, seed=50)
    a = _commit_tensors(t)

    def call(**kw):
        kw = {**a, **kw}
        if layers:
            return pk.tree_commit_layers([t.sd], k_trees=[kw.pop("k", t.k)], v_trees=[kw.pop("v", t.v)], **kw)
        return t.sd.tree_commit(k_tree=kw.pop("k", t.k), v_tree=kw.pop("v", t.v), **kw)

    big = torch.full((64,), 7, dtype=torch.int32, device="cuda")   # views into it meet in one element
    rows, seqs = lambda at: big[at:at + 12].view(3, 4), lambda at: big[at:at + 3]
    at = lambda name, x: (seqs if a[name].dim() == 1 else rows)(x)
    size = lambda name: a[name].numel()
    for out in ("accepted_len", "out_tokens", "path"):
        for other in a:
            if other != out:
                _refused(t.sd, lambda: call(**{out: at(out, 20), other: at(other, 20 + size(out) - 1)}))
                _refused(t.sd, lambda: call(**{out: at(out, 20), other: at(other, 21 - size(other))}))
        for rows_of in ("k", "v"):
            kv = t.k if rows_of == "k" else t.v
            _refused(t.sd, lambda: call(**{out: kv.view(torch.int32).view(-1)[4:4 + size(out)].view(a[out].shape)}))
    torch.cuda.synchronize()
    assert bool((big == 7).all()) and t.sd.kv_tables()["seq_len"].tolist() == [10, 20, 0]
    assert all(bool((a[x] == 7).all()) for x in ("accepted_len", "out_tokens", "path"))
    call(accepted_len=seqs(0), out_tokens=rows(3), path=rows(15), seq_ids=seqs(27).copy_(a["seq_ids"]))  # side by side is fine
    assert seqs(0).tolist() == [1, 1, 1] and t.sd.kv_tables()["seq_len"].tolist() == [11, 21, 1]


@pytest.mark.parametrize("kw,code", [(dict(n=65), 2), (dict(batch=3), 2), (dict(batch=0), 1), (dict(n=0), 1)] +
                         [({x: None}, 1) for x in ("parent", "draft", "next", "k", "v", "acc", "tok", "path")] +
                         [(dict(k=2), 1), (dict(v=8), 1)])
def test_one_wrong_argument_of_a_commit_that_is_right(kw, code):
    t = Tree(4, 2, 64, [10, 20], 4, seed=51)
    a = _commit_tensors(t)
    p = dict(parent=a["parent"].data_ptr(), draft=a["draft_token"].data_ptr(), next=a["next_token"].data_ptr(), k=t.k.data_ptr(),
             v=t.v.data_ptr(), acc=a["accepted_len"].data_ptr(), tok=a["out_tokens"].data_ptr(), path=a["path"].data_ptr())

    def call(batch=2, n=4, **q):
        q = {**p, **q}
        return t.sd.lib.sdlm_tree_commit(t.sd.ctx, batch, n, None, None, q["parent"], q["draft"], q["next"], q["k"], q["v"], q["acc"],
                                         q["tok"], q["path"], torch.cuda.current_stream().cuda_stream)

    before = t.sd.launch_count()
    assert call(**{x: p[x] + y if x in p and y else y for x, y in kw.items()}) == code
    torch.cuda.synchronize()
    assert t.sd.launch_count() == before and t.sd.kv_tables()["seq_len"].tolist() == [10, 20]
    assert all(bool((a[x] == 7).all()) for x in ("accepted_len", "out_tokens", "path"))
    assert call() == 0 and a["accepted_len"].tolist() == [1, 1] and t.sd.kv_tables()["seq_len"].tolist() == [11, 21]


def test_attention_and_gather_outputs_over_index_tensors_are_refused():
    t = Tree(4, 2, 64, [10, 20, 0], 4, seed=52)
    ids, nodes = torch.arange(3, dtype=torch.int32, device="cuda"), torch.full((3,), 4, dtype=torch.int32, device="cuda")
    out = torch.full_like(t.q, 7.0)
    words = out.view(torch.int32).view(-1)
    for at in (0, words.numel() - 12):                # the first and the last words of the output
        w = words[at:at + 12]
        _refused(t.sd, lambda: t.sd.tree_attn(t.q, t.k, t.v, w.view(3, 4), out=out))
        _refused(t.sd, lambda: t.sd.tree_attn(t.q, t.k, t.v, t.parent, n_nodes=w[-3:], out=out))
        _refused(t.sd, lambda: t.sd.tree_attn(t.q, t.k, t.v, t.parent, seq_ids=w[:3], out=out))
    kv = torch.full((2, 3, 5, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    _refused(t.sd, lambda: t.sd.kv_gather_batch(kv[0], kv[0]))
    for x in (0, 1):
        _refused(t.sd, lambda: t.sd.kv_gather_batch(kv[0], kv[1], seq_ids=kv[x].view(torch.int32).view(-1)[-3:]))
    torch.cuda.synchronize()
    assert bool((out == 7.0).all()) and bool((kv == 7.0).all())
    t.sd.tree_attn(t.q, t.k, t.v, t.parent, n_nodes=nodes, seq_ids=ids, out=out)
    t.check(out)
    t.sd.kv_gather_batch(kv[0], kv[1], seq_ids=ids)   # neighbours are fine
    assert torch.equal(kv[0, 1], t.kc[1][:5]) and torch.equal(kv[1, 1], t.vc[1][:5])


def test_rotary_outputs_over_positions_and_weights_are_refused():
    t = Tree(4, 2, 64, [10, 20, 0], 4, seed=53)
    q_out, k_out = torch.full_like(t.q, 7.0), torch.full_like(t.k, 7.0)
    rope = pk.RopeConfig()
    for out in (q_out, k_out):
        flat, words = out.view(-1), out.view(torch.int32).view(-1)
        call = lambda **kw: t.sd.qk_norm_rope(t.q, t.k, rope, q_out=q_out, k_out=k_out, **kw)
        _refused(t.sd, lambda: call(positions=words[-12:].view(3, 4)))
        _refused(t.sd, lambda: call(positions=words[:12].view(3, 4), relative=True))
        _refused(t.sd, lambda: call(seq_ids=words[-3:]))
        _refused(t.sd, lambda: call(q_weight=flat[:64]))
        _refused(t.sd, lambda: call(k_weight=flat[-64:]))
    _refused(t.sd, lambda: t.sd.qk_norm_rope(t.q, t.k, rope, q_out=q_out, k_out=q_out.view(-1)[:t.k.numel()].view(t.k.shape)))
    torch.cuda.synchronize()
    assert bool((q_out == 7.0).all()) and bool((k_out == 7.0).all())
    a, b = t.sd.qk_norm_rope(t.q, t.k, rope)
    t.sd.qk_norm_rope(t.q, t.k, rope, q_out=t.q, k_out=t.k)      # in place is fine
    assert torch.equal(a, t.q) and torch.equal(b, t.k)


def test_sampling_outputs_over_logits_parameters_and_each_other():
    sd = pk.Sdlm(pk.SdlmConfig(2, 1, 64, 64, 64, 4, 4, 4, max_block=8))
    R, V = 9, 5000
    g = torch.Generator("cuda").manual_seed(54)
    logits = torch.randn((R, V), device="cuda", generator=g) * 3
    f = {x: torch.rand(R, device="cuda", generator=g) for x in ("u", "temperature", "top_p", "min_p")}
    f["min_p"] *= 0.1
    f["top_k"] = torch.arange(R, dtype=torch.int32, device="cuda") * 30
    made = lambda: dict(token=torch.full((R,), 7, dtype=torch.int32, device="cuda"), prob=torch.full((R,), 7.0, device="cuda"),
                        entropy=torch.full((R,), 7.0, device="cuda"), n_kept=torch.full((R,), 7, dtype=torch.int32, device="cuda"))
    call = lambda **kw: sd.sample(logits, **{**f, **made(), **kw})
    want = call()
    big = torch.zeros(40, device="cuda")
    as_ = lambda name, x: x.view(torch.int32) if name in ("token", "n_kept", "top_k") else x
    for out in made():
        at = lambda i: as_(out, big[i:i + R])
        _refused(sd, lambda: call(**{out: as_(out, logits.view(-1)[:R])}))
        _refused(sd, lambda: call(**{out: as_(out, logits.view(-1)[-R:])}))
        for other in (*f, *(x for x in made() if x != out)):
            _refused(sd, lambda: call(**{out: at(10), other: as_(other, big[10 + R - 1:10 + 2 * R - 1])}))
            _refused(sd, lambda: call(**{out: at(10), other: as_(other, big[11 - R:11])}))
        for other in (x for x in made() if x != out):
            _refused(sd, lambda: call(**{out: at(10), other: as_(other, big[10:10 + R])}))
    torch.cuda.synchronize()
    assert bool((big == 0).all())
    # in place of a parameter, row for row
    for out, param in (("token", "top_k"), ("prob", "u"), ("entropy", "temperature"), ("n_kept", "top_k"), ("prob", "top_p"), ("prob", "min_p")):
        same = f[param].clone()
        got = call(**{param: same, out: same})
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_missing_tensors_are_refused_by_name_of_the_call():
    t = Tree(4, 2, 64, [10], 4, seed=55)
    logits, u = torch.zeros((2, 64), device="cuda"), torch.zeros(2, device="cuda")
    for call in (lambda: t.sd.sample(logits, None), lambda: t.sd.sample(None, u), lambda: t.sd.kv_gather_batch(None, None),
                 lambda: t.sd.tree_attn(t.q, t.k, t.v, None), lambda: t.sd.tree_attn(t.q, None, t.v, t.parent),
                 lambda: t.sd.tree_commit(None, t.parent, t.parent, t.k, t.v), lambda: t.sd.qk_norm_rope(None, t.k, pk.RopeConfig())):
        with pytest.raises((TypeError, ValueError, pk.SdlmError)):
            call()
