"""Calls on drafted tokens around the kernels: what cannot be captured into a graph, tensors of another stream, options, results that
overlap inputs."""
import numpy as np
import pytest
import torch

from paper_2507_17769_amd import binding as B
from paper_2507_17769_amd import workloads as W
from paper_2507_17769_amd.runner import Engine
from test_gpu_tree import load, make_batch, make_engine, model_parts, random_tree

pytestmark = pytest.mark.gpu


def refused(status, call):
    with pytest.raises(B.PolystepError) as e:
        call()
    assert e.value.status == status, str(e.value)


def test_calls_with_work_on_the_host_are_refused_in_a_capture_and_leave_it_whole():
    """ps_verify_tokens takes ids from the host, ps_tree_plan and ps_init_qk_norm keep what they are given on it: none of them is part of a graph.  What was
    captured around them replays as ever, with steps over other ids in between, and those steps get what they get without a graph."""
    rng = np.random.default_rng(23)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        V = 320
        m, layers, head, gains = model_parts(2, V, 6)
        spec = [(40, random_tree(rng, 9)), (7, [-1, 0, -2])]
        seqs, parents, pages, n_pages = make_batch(rng, spec)
        eng = Engine(m, n_pages, 2, 2, max_position=128)
        load(eng, layers, head, gains)
        eng.kv_pool().normal_()
        tree, spare = eng.tree(seqs, parents), B.Tree(eng.ctx)
        T = len(parents)
        ids = [rng.integers(0, V, T).astype(np.int32) for _ in range(5)]
        want = [{k: v.clone() for k, v in eng.verify_tokens(tree, i, want_logits=True).items()} for i in ids]
        q = torch.randn(T, m["n_q"], m["head_dim"], device="cuda").to(torch.bfloat16)
        z = torch.randn(T, V, device="cuda")
        g = torch.ones(m["head_dim"], dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            o = eng.tree_attention(1, tree, q)
            refused(B.PS_ESTATE, lambda: eng.ctx.verify_tokens(tree, ids[0]))
            refused(B.PS_ESTATE, lambda: spare.plan(seqs, parents))
            refused(B.PS_ESTATE, lambda: eng.ctx.init_qk_norm(1, g.data_ptr(), g.data_ptr()))
            refused(B.PS_ESTATE, lambda: eng.load_qk_norm(1, g, g))
            p = eng.pick_tokens(z)
        for k in range(5):
            got = eng.verify_tokens(tree, ids[k], want_logits=True)
            o.fill_(3)
            p["next"].fill_(-7)
            graph.replay()
            again = eng.verify_tokens(tree, ids[(k + 1) % 5], want_logits=True)
            eager = eng.tree_attention(1, tree, q)
            stream.synchronize()
            assert all(torch.equal(got[n], want[k][n]) and torch.equal(again[n], want[(k + 1) % 5][n]) for n in got), k
            assert torch.equal(p["next"], z.argmax(-1).to(torch.int32))
            graph.replay()                         # the cache now holds what the last step appended
            stream.synchronize()
            assert torch.equal(o, eager), k
        refused(B.PS_ESTATE, lambda: eng.tree_attention(0, spare, q[:0]))       # its plan was refused: it is empty
        spare.plan(seqs, parents)
        assert torch.equal(eng.tree_attention(1, spare, q), eager)
        eng.close()


def test_rows_that_ask_for_a_mask_that_is_not_there():
    eng = Engine("tiny", 1, max_position=16)
    z = torch.randn(4, 5001, device="cuda")
    rules = {"mask": torch.zeros(0, 157, dtype=torch.int32, device="cuda"), "mask_row": torch.tensor([-1, 0, 3, -5], dtype=torch.int32, device="cuda")}
    got = eng.pick_tokens(z, rules, want_logits=True)
    eng.ctx.sync()
    top = z.argmax(-1).cpu().tolist()
    assert got["next"].cpu().tolist() == [top[0], -1, -1, top[3]]
    assert (got["logits"][1:3] == float("-inf")).all() and torch.equal(got["logits"][0], z[0]) and torch.equal(got["logits"][3], z[3])
    refused(B.PS_EINVAL, lambda: eng.pick_tokens(z, {"mask_row": rules["mask_row"]}))
    eng.close()


def busy(stream):
    """More than half a second of work on a stream: what is enqueued behind it has not run when the call returns."""
    with torch.cuda.stream(stream):
        x = torch.ones(1 << 28, device="cuda")
        torch.cuda.synchronize()
        for _ in range(1300):
            x.mul_(1.0)
    return x


def lies_free(address, size, dtype):
    """The allocator hands memory at `address` out to the current stream."""
    kept = [torch.empty(size, dtype=dtype, device="cuda") for _ in range(4)]
    return address in [t.data_ptr() for t in kept]


def test_tensors_dropped_after_a_call_from_another_stream_stay_until_it_has_run():
    """An engine on one stream, calls made while another is current: the memory of temporaries and of results that are dropped at once is not handed out
    before the engine's stream has come to its end."""
    rng = np.random.default_rng(3)
    stream = torch.cuda.Stream()
    spec = [(60, random_tree(rng, 30)), (5, [-1])]
    seqs, parents, pages, n_pages = make_batch(rng, spec)
    seqs = [W.SeqSpec(*s) for s in seqs]
    m, layers, head, gains = model_parts(1, 320, 2)
    with torch.cuda.stream(stream):
        eng = Engine(m, n_pages, 1, 1, max_position=256)
        load(eng, layers, head, gains)
        eng.kv_pool().normal_()
    tree = eng.tree(seqs, parents)
    T, n_q, n_kv, d, V = 31, m["n_q"], m["n_kv"], m["head_dim"], 70001
    ids = rng.integers(0, 320, T).astype(np.int32)
    eng.verify_tokens(tree, ids, want_logits=True)          # workspaces have their size: no call below waits for it
    eng.step(seqs, torch.zeros(T, m["hidden"], dtype=torch.int16, device="cuda"))
    eng.step_tokens(seqs, ids, want_hidden=True)
    torch.cuda.synchronize()

    def run(name, call, inputs):
        torch.cuda.synchronize()
        work = busy(stream)
        held = [(t.data_ptr(), t.shape, t.dtype) for t in inputs]
        out = call(*inputs)
        results = list(out.values()) if isinstance(out, dict) else [out]
        at = [(t.data_ptr(), t.shape, t.dtype) for t in results if torch.is_tensor(t)]
        del out, results
        inputs.clear()
        again = [lies_free(*x) for x in held + at]
        assert not stream.query(), f"{name}: the stream is idle, nothing was shown"
        torch.cuda.synchronize()
        del work
        return again

    odd = dict(device="cuda")
    cases = {
        "qk_norm_rope": (lambda qkv: eng.qk_norm_rope(0, tree, qkv), [torch.randn(T, (n_q + 2 * n_kv) * d, **odd)]),
        "tree_attention": (lambda q: eng.tree_attention(0, tree, q), [torch.randn(T, n_q, d, **odd).to(torch.bfloat16)]),
        "pick_tokens": (lambda z, p: eng.pick_tokens(z, {"presence": p}, want_logits=True), [torch.randn(T, V, **odd), torch.ones(T, **odd)]),
        "verify_tokens": (lambda p: eng.verify_tokens(tree, ids, {"presence": p}, want_logits=True, want_hidden=True), [torch.ones(2, **odd)]),
        "step": (lambda x: eng.step(seqs, x)[0], [torch.zeros(T, m["hidden"], dtype=torch.int16, **odd)]),
        "step_tokens": (lambda: eng.step_tokens(seqs, ids, want_hidden=True), []),
    }
    for name, (call, inputs) in cases.items():
        assert not any(run(name, call, inputs)), name
    eng.close()


def test_steps_over_trees_are_counted_like_others():
    """Option time_attention = N: every Nth step, whatever kind it is."""
    rng = np.random.default_rng(4)
    m, layers, head, gains = model_parts(2, 320, 4)
    seqs, parents, pages, n_pages = make_batch(rng, [(20, [-1, 0, 0])])
    eng = Engine(m, n_pages, 2, 2, max_position=64)
    load(eng, layers, head, gains)
    tree = eng.tree(seqs, parents)
    eng.ctx.set_option("time_attention", 3)
    for _ in range(6):
        eng.verify_tokens(tree, [1, 2, 3])
    assert len(eng.ctx.attention_times()) == 2 * 2
    eng.close()


def test_results_over_inputs_are_refused_where_they_would_be_read_again():
    """Rows of one tensor may lie between another's; a result that shares memory with its input is refused, but for fp32 logits changed in place."""
    m, layers, head, gains = model_parts(1, 320, 9)
    eng = Engine(m, 4, 1, 1, max_position=64)
    c, T, d = eng.ctx, 3, m["head_dim"]
    wq, wqkv = m["n_q"] * d, (m["n_q"] + 2 * m["n_kv"]) * d
    tree = eng.tree([(1, T, T, [2])], [-1, 0, 0])
    buf = torch.randn(T, 2 * wqkv, device="cuda").to(torch.bfloat16)
    P, row = buf.data_ptr(), 2 * wqkv
    for out, ldo in ((P, row), (P + 2 * 8, row), (P + 2 * (wq - 8), row), (P + 2 * (row - wq + 8), row), (P + 2 * wq, row + 8), (P + 2 * (2 * row + wq - 8), row)):
        refused(B.PS_EINVAL, lambda: c.tree_attention(0, tree, P, row, out, ldo))
        refused(B.PS_EINVAL, lambda: c.tree_attention(0, tree, out, ldo, P, row))
    q = buf[:, :wq].clone()
    want = eng.tree_attention(0, tree, q)
    for at in (wq, row - wq):                                       # between the rows of q
        buf[:, :wq] = q
        assert torch.equal(eng.tree_attention(0, tree, buf[:, :wq], buf[:, at:at + wq]), buf[:, at:at + wq]) and torch.equal(buf[:, at:at + wq].reshape(want.shape), want)
    for q_at in (P, P + 2 * (2 * row + wqkv - 8), P - 2 * (T * wq - 8)):
        refused(B.PS_EINVAL, lambda: c.qk_norm_rope(0, tree, P, B.PS_BF16, row, q_at))
    V = 100
    z = torch.randn(4, 2 * V, device="cuda")
    Z = z.data_ptr()
    for dtype, ld, n, out, ldo in ((B.PS_F32, 2 * V, 4, Z, V), (B.PS_F32, V, 4, Z, 2 * V), (B.PS_F32, 2 * V, 4, Z + 4, 2 * V), (B.PS_F32, 2 * V, 4, Z + 4 * (V - 1), 2 * V),
                                   (B.PS_BF16, 2 * V, 4, Z, 2 * V), (B.PS_BF16, V, 1, Z, V), (B.PS_F32, V, 1, Z + 4, V), (B.PS_F32, 2 * V, 3, Z + 4 * (V + 1), 2 * V)):
        refused(B.PS_EINVAL, lambda: c.pick_tokens(Z, dtype, ld, n, V, None, out, ldo))
    logits, half = z[:, :V].clone(), z[:, :V].to(torch.bfloat16)
    c.pick_tokens(Z, B.PS_F32, 2 * V, 4, V, None, Z + 4 * V, 2 * V)     # side by side
    assert torch.equal(z[:, V:], logits)
    c.pick_tokens(Z, B.PS_F32, 2 * V, 1, V, None, Z, 5 * V)             # one row, in place
    z.view(torch.bfloat16)[:, :V] = half                              # bf16 rows of half the bytes, their results behind them
    c.pick_tokens(Z, B.PS_BF16, 4 * V, 4, V, None, Z + 4 * V, 2 * V)
    assert torch.equal(z[:, V:], half.float())
    eng.close()


def test_gains_are_taken_after_the_work_that_makes_them():
    """load_qk_norm returns when the gains have been copied; they are copied behind the work of the caller's stream, which they come from."""
    home, other = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(home):
        eng = make_engine(4, 2, 64, 2)
        tree = eng.tree([(1, 3, 3, [1])])
        qkv = torch.randn(3, 8 * 64, device="cuda")
        eng.load_qk_norm(0, torch.full((64,), 2.0, device="cuda"), torch.full((64,), 3.0, device="cuda"))
        want = eng.qk_norm_rope(0, tree, qkv).clone()
        gains = torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
        eng.load_qk_norm(0, *gains)
    torch.cuda.synchronize()
    work = busy(other)
    with torch.cuda.stream(other):
        eng.load_qk_norm(0, gains[0].fill_(2.0), gains[1].fill_(3.0))
    with torch.cuda.stream(home):
        assert torch.equal(eng.qk_norm_rope(0, tree, qkv), want)
    torch.cuda.synchronize()
    del work
    eng.close()


def test_tensors_of_the_wrong_kind_are_refused_alike_from_every_stream():
    eng = make_engine(4, 2, 64, 2)
    tree = eng.tree([(1, 3, 3, [1])])
    z, q = torch.zeros(3, 100, device="cuda"), torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    for stream in (eng.stream, torch.cuda.Stream()):
        with torch.cuda.stream(stream):
            for error, call in ((ValueError, lambda: eng.qk_norm_rope(0, tree, torch.zeros(3, 512))), (ValueError, lambda: eng.qk_norm_rope(0, tree, torch.zeros(3, 512, device="cuda"), q.cpu())),
                                (ValueError, lambda: eng.tree_attention(0, tree, q.cpu())), (ValueError, lambda: eng.tree_attention(0, tree, q, q.cpu())),
                                (ValueError, lambda: eng.pick_tokens(z.cpu())), (TypeError, lambda: eng.pick_tokens(z, {"presence": torch.zeros(3)})),
                                (TypeError, lambda: eng.pick_tokens(z, {"presence": torch.zeros(3, dtype=torch.int32, device="cuda")})),
                                (ValueError, lambda: eng.pick_tokens(z, {"no_rule": z})), (TypeError, lambda: eng.verify_tokens(tree, [0, 0, 0], {"presence": torch.zeros(1)}))):
                with pytest.raises(error):
                    call()
    eng.close()
