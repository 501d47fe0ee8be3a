"""Host side of the operators on drafted tokens: plans of token trees (under AddressSanitizer and UndefinedBehaviorSanitizer), index
arrays, refusals that need no device, and the oracle against closed forms."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import layer as olayer
from oracle import tree as ot
from paper_2507_17769_amd import binding as B
from paper_2507_17769_amd import workloads as W

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def host_ctx(model="tiny", max_position=20000, n_layers=1):
    m = W.MODELS[model]
    return B.Context(m["hidden"], m["n_q"], m["n_kv"], m["head_dim"], m["ffn"], n_layers, max_position, 1e-5, m["rope_base"], host_only=True)


def test_plans_of_trees_say_who_sees_what(tmp_path):
    csrc = os.path.join(ROOT, "paper_2507_17769_amd", "csrc")
    exe = str(tmp_path / "tree_plan_check")
    cmd = ["g++", "-O2", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", csrc,
           os.path.join(ROOT, "tests", "tree_plan_check.cpp"), os.path.join(csrc, "planner.cpp"), os.path.join(csrc, "tree_plan.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("OK "), r.stdout + r.stderr


def test_tree_indices_are_slots_in_order_and_positions_by_depth():
    c = host_ctx()
    t = B.Tree(c)
    assert t.plan([]).indices()[0].tolist() == [0]
    parents = [-1, 0, 0, 1, -2, -1, 0, 1]
    seqs = [(7, 5, 22, [3, 9]), (8, 3, 3, [4])]
    cu, pos, slots = t.plan(seqs, parents).indices()
    assert cu.tolist() == [0, 5, 8]
    assert pos.tolist() == [17, 18, 18, 19, 17, 0, 1, 2]
    assert slots.tolist() == [9 * 16 + i for i in range(1, 6)] + [64, 65, 66]
    chain = t.plan(seqs).indices()
    assert all(np.array_equal(a, b) for a, b in zip(chain, c.step_indices(seqs)))


def test_malformed_trees_are_refused_and_leave_the_tree_empty():
    c = host_ctx(max_position=2000)
    c.kv_alloc(130, 1, 0)
    t = B.Tree(c)
    ok = [(1, 3, 20, [0, 1])]
    cases = [
        (ok, [-1, 0, 2], B.PS_EINVAL, "node 2"),           # itself
        (ok, [-1, 2, 0], B.PS_EINVAL, "node 1"),           # a later node
        (ok, [-3, 0, 0], B.PS_EINVAL, "node 0"),
        (ok, [-2, 0, 0], B.PS_EINVAL, "padding"),
        ([(1, 3, 2, [0])], None, B.PS_EINVAL, "kv_len"),
        ([(1, 3, 20, [0, 130])], None, B.PS_ERANGE, "outside"),
        ([(1, 3, 20, [0, 0])], None, B.PS_EINVAL, "twice"),
        ([(1, 1025, 1100, list(range(69)))], [-1, -1] + list(range(1, 1024)), B.PS_ERANGE, "nodes"),
    ]
    for seqs, parents, status, word in cases:
        t.plan(ok)
        with pytest.raises(B.PolystepError) as e:
            t.plan(seqs, parents)
        assert e.value.status == status and word in str(e.value), str(e.value)
        with pytest.raises(B.PolystepError) as e:
            t.indices()
        assert e.value.status == B.PS_ESTATE
    with pytest.raises(ValueError):
        t.plan(ok, [-1, 0])
    # another context's tree, also one that has taken its place in memory
    other = host_ctx()
    with pytest.raises(B.PolystepError) as e:
        other._check(B.lib.ps_tree_plan(other.handle, t.handle, None, 0, None))
    assert e.value.status == B.PS_ESTATE
    other.destroy()
    c.destroy()
    t.destroy()          # after its context


def test_host_only_contexts_refuse_what_needs_a_device():
    c = host_ctx()
    t = B.Tree(c).plan([(1, 2, 5, [0])])
    calls = [lambda: c.init_qk_norm(0, 16, 16), lambda: c.qk_norm_rope(0, t, 16, B.PS_F32, 512, 16), lambda: c.tree_attention(0, t, 16, 256, 16, 256),
             lambda: c.tree_keep(t, [[0]]), lambda: c.pick_tokens(16, B.PS_F32, 64, 1, 64), lambda: c.verify_tokens(t, [0, 0]), lambda: c.kv_pool()]
    for call in calls:
        with pytest.raises(B.PolystepError) as e:
            call()
        assert e.value.status == B.PS_ESTATE
    assert B.lib.ps_tree_create(c.handle, None) == B.PS_EINVAL
    assert B.lib.ps_tree_create(None, ctypes.byref(ctypes.c_void_p())) == B.PS_EINVAL
    B.lib.ps_tree_destroy(None)
    for f, args in ((B.lib.ps_tree_keep, (None, None, None, None)), (B.lib.ps_qk_norm_rope, (None, 0, None, None, 0, 0, None)),
                    (B.lib.ps_tree_attention, (None, 0, None, None, 0, None, 0)), (B.lib.ps_verify_tokens, (None,) * 8), (B.lib.ps_kv_pool, (None, None, None))):
        assert f(*args) == B.PS_EINVAL


# ------------------------------------------------------------------------------------------------------ the oracle
def test_oracle_a_chain_is_causal_attention():
    rng = np.random.default_rng(3)
    sh = olayer.Shape(64, 4, 2, 16, 64)
    n, prefix = 6, 21
    pool = olayer.PagedKV(3, 1, sh.n_kv, sh.head_dim)
    k, v = rng.standard_normal((2, prefix + n, sh.n_kv, sh.head_dim))
    pool.write(0, [2, 0, 1], 0, k, v)
    K, V = pool.gather(0, [2, 0, 1], prefix + n, np.float64)
    q = rng.standard_normal((n, sh.n_q, sh.head_dim))
    want = olayer.attention_paged(q, [olayer.Seq(n, prefix + n, [2, 0, 1])], pool, 0, sh.n_kv)
    got, spread = ot.attention(q, K, V, prefix, list(range(-1, n - 1)))
    assert np.allclose(got, want, rtol=1e-12, atol=1e-12) and (spread >= np.abs(got) - 1e-12).all()


def test_oracle_a_node_is_the_end_of_its_own_chain():
    """Each node attends as the last token of a sequence that holds nothing but its branch."""
    rng = np.random.default_rng(4)
    parents = [-1, 0, 0, 2, -1, 1, 5, -2, 3]
    prefix, n, d = 5, len(parents), 8
    k, v = rng.standard_normal((2, prefix + n, 1, d))
    q = rng.standard_normal((n, 2, d))
    got, _ = ot.attention(q, k, v, prefix, parents)
    for i, p in enumerate(parents):
        if p == ot.PAD:
            assert not got[i].any()
            continue
        at = list(range(prefix)) + [prefix + j for j in ot.branch(parents, i)]
        for h in range(2):
            s = k[at, 0] @ q[i, h] / np.sqrt(d)
            w = np.exp(s) / np.exp(s).sum()
            assert np.allclose(got[i, h], w @ v[at, 0], rtol=1e-12)
    assert ot.depths(parents).tolist() == [0, 1, 1, 2, 0, 2, 3, 0, 3]


def test_oracle_normalised_heads_have_unit_square_mean():
    rng = np.random.default_rng(5)
    u = rng.standard_normal((3, 4, 64)) * 7
    n = ot.norm_heads(u, np.ones(64), 0.0)
    assert np.allclose(np.mean(n * n, axis=-1), 1.0) and np.allclose(n / u, (n / u)[..., :1])


def test_oracle_rules_by_hand():
    z = np.array([2.0, -1.0, 0.5, 3.0, 1.0, 0.0])
    got = ot.apply_rules(z, [0, 1, 3, 3, 9, -1], 2, [3, 4], 2.0, 0.25, 0.5, [(5, 1.0), (2, -4.0), (2, 4.0), (77, 1.0)], np.array([1, 1, 1, 1, 1, 0], bool))
    # 0: prompt 2/2; 1: prompt -1*2; 2: bias 4; 3: output three times 3/2 - .75 - .5; 4: branch 1/2 - .25 - .5; 5: not allowed
    assert got.tolist() == [1.0, -2.0, 4.5, 0.25, -0.25, -np.inf]
    i, lp = ot.pick(got)
    w = np.exp(got)
    assert i == 2 and np.isclose(lp, np.log(w[2] / w.sum()))
    assert ot.pick(np.full(4, -np.inf)) == (-1, -np.inf)
    assert ot.pick(np.array([1.0, 7.0, 7.0]))[0] == 1
    assert ot.pick(np.array([np.nan, 1.0]))[0] == 1 and np.isnan(ot.pick(np.array([np.nan, 1.0]))[1])


def test_oracle_verification_of_a_chain_is_a_prefill():
    from oracle import head as ohead
    rng = np.random.default_rng(6)
    m = W.MODELS["tiny"]
    from oracle import run as orun
    sh = orun.shape_from(m)
    w = orun.widen_weights(W.layer_weights(m, 1, 0), np.float64)
    hw = orun.widen_weights(W.head_weights(m, 64, 2), np.float64)
    ids = rng.integers(0, 64, 9)
    seqs = [olayer.Seq(9, 9, [0])]
    a, b = orun.make_pool(m, 1), orun.make_pool(m, 1)
    lg, hid = ot.verify(sh, hw, [w], [None], seqs, [list(range(-1, 8))], ids, a, np.float64)
    want = olayer.stack_forward(ohead.embed(ids, hw["embedding"]), [w], seqs, b, sh)
    assert np.allclose(hid, want, rtol=1e-9, atol=1e-9) and np.array_equal(a.bits, b.bits)
    assert np.allclose(lg[-1:], ohead.logits(want, seqs, hw["g_final"], hw["w_out"], sh.rms_eps), rtol=1e-9, atol=1e-9)
