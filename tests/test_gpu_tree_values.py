"""Attention of token trees where the cache holds what a node sees and no finite sum can hide: infinities and NaN in the prefix, scores far from
zero, rows whose scores are all -inf.  Oracle and tolerances are those of test_gpu_tree."""
import numpy as np
import pytest
import torch

from oracle import tree as ot
from paper_2507_17769_amd import binding as B
from test_gpu_tree import EPS32, HALF, bf, chain, check_attention, f64, random_tree, run_attention

pytestmark = pytest.mark.gpu
KINDS = (float("inf"), float("-inf"), float("nan"))


def one_bad_value_a_pair(prefix, d):
    """(position, dimension, value): in every pair of pages that the prefix reaches, one place of its own dimension."""
    return [(min(32 * j + 7 * j % 32, prefix - 1), j % d, KINDS[j % 3]) for j in range((prefix + 31) // 32)]


# tokens that fill one 16-row tile or less go to single wavefronts, further ones to teams
@pytest.mark.parametrize("n_q,n_kv,d", [(8, 2, 128), (4, 4, 64), (16, 1, 128)])
@pytest.mark.parametrize("parents", [[-1], [-1, 0, -2], [-1, -1, 0], None], ids=["one", "padded", "tree", "team"])
@pytest.mark.parametrize("workers", [0, 1, 7])
def test_values_of_the_prefix_that_are_not_finite_reach_every_node(n_q, n_kv, d, parents, workers):
    """Each such value has a dimension of its own: there every live row of the first kv head's queries shows that value, wherever its pair of pages lies in
    a block of pages, and whatever loop takes the pair."""
    rng = np.random.default_rng(d + workers)
    tokens = 16 * n_kv // n_q
    par = parents if parents is None else parents[:max(1, min(tokens, len(parents)))]
    prefixes = [5, 40, 64, 95, 100, 127, 700, 1023, 1100] + ([2100] if d == 128 else [])
    spec = [(p, random_tree(rng, 2 * tokens + 3, pad=1) if par is None else par) for p in prefixes]

    def edit(k, v, p, t):
        for pos, dim, what in one_bad_value_a_pair(p, d):
            v[pos, 0, dim] = what
    eng, _, out, q, kv = run_attention(rng, n_q, n_kv, d, spec, [("attn_workers", workers)], q_scale=0.3, edit=edit)
    group, t0, mended, clean = n_q // n_kv, 0, out.clone(), []
    for (p, t), (k, v) in zip(spec, kv):
        n, bad = len(t), one_bad_value_a_pair(p, d)
        live = np.array(t) != B.PS_TREE_PAD
        rows = out[t0:t0 + n][torch.from_numpy(live)].float()
        c = v.clone()
        for pos, dim, what in bad:
            c[pos, 0, dim] = 0.0
            got = rows[:, :group, dim]
            assert (torch.isnan(got) if np.isnan(what) else got == what).all(), (p, n, pos, dim, what, got)
        want, _ = ot.attention(f64(q[t0:t0 + n]), f64(k), f64(c), p, t)
        for _, dim, _ in bad:                       # the other dimensions are compared as ever
            mended[t0:t0 + n, :group, dim] = bf(want[:, :group, dim])
        clean.append((k, c))
        t0 += n
    check_attention(mended, q, clean, spec, d)
    eng.close()


WIDE = [("attn_workers", 0), ("attn_workers", 1), ("attn_workers", 6), ("attn_workers", 40)]


@pytest.mark.parametrize("option", WIDE, ids=[str(o[1]) for o in WIDE])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("n_q,n_kv,d", [(4, 2, 64), (8, 2, 128), (16, 1, 128)])
def test_equal_scores_far_from_zero_weigh_the_same(n_q, n_kv, d, sign, option):
    """Every product of a query and a key is d 2^23, a sum of powers of two and exact: scores of some 2^27, whose fp32 steps are 8.  All weights of a row are
    the same number then, whatever it is: a mean of L values is off by their fp32 sums, a division, and the rounding of the result."""
    seed = np.random.default_rng(6)
    spec = [(200, chain(1)), (0, [-1, -1, -2]), (333, [-1, 0]), (1500, random_tree(seed, 40, pad=3)), (90, random_tree(seed, 9))]

    class Draws:                                     # run_attention draws keys, values, then queries
        def standard_normal(self, shape):
            return np.full(shape, 2.0 ** 12) if len(shape) == 2 else seed.standard_normal(shape)
        permutation = staticmethod(seed.permutation)
    eng, _, out, q, kv = run_attention(Draws(), n_q, n_kv, d, spec, [option], q_scale=1.0, edit=lambda k, v, p, t: k.fill_(sign * 2.0 ** 11))
    assert (q.float() == 2.0 ** 12).all()
    t0 = 0
    for (p, t), (k, v) in zip(spec, kv):
        see = np.concatenate([np.repeat((np.array(t) != B.PS_TREE_PAD)[:, None], p, 1), ot.sees(t)], 1)
        V = np.repeat(f64(v), n_q // n_kv, axis=1)
        for i in range(len(t)):
            got = f64(out[t0 + i])
            if not see[i].any():
                assert not got.any()
                continue
            want, mag = V[see[i]].mean(0), np.abs(V[see[i]]).mean(0)
            assert (np.abs(got - want) <= HALF * np.abs(want) + (2 * see[i].sum() + 4) * EPS32 * mag * (1 + HALF)).all(), (p, i)
        t0 += len(t)
    eng.close()


@pytest.mark.parametrize("option", WIDE, ids=[str(o[1]) for o in WIDE])
def test_rows_whose_scores_are_all_minus_infinity_are_nan(option):
    """The softmax of nothing but -inf is not a number, however the plan cuts the row's keys; only padding, which sees nothing, is zero.  The other kv
    head's rows are as ever."""
    rng = np.random.default_rng(7)
    spec = [(200, chain(1)), (0, [-1, -2]), (1500, random_tree(rng, 40, pad=3)), (640, [-1, 0]), (90, random_tree(rng, 9, pad=1))]

    def edit(k, v, p, t):
        k[:, 0] = 0.0
        k[:, 0, 0] = float("-inf")
    n_q, n_kv, d = 8, 2, 128

    class Positive:
        def standard_normal(self, shape):
            x = rng.standard_normal(shape)
            return np.abs(x) + 0.1 if len(shape) == 2 else x
        permutation = staticmethod(rng.permutation)
    eng, _, out, q, kv = run_attention(Positive(), n_q, n_kv, d, spec, [option], edit=edit)
    pad = torch.from_numpy(np.concatenate([np.array(t) == B.PS_TREE_PAD for _, t in spec]))
    assert torch.isnan(out[~pad][:, :4]).all() and not out[pad].any()
    fine = [(k.clone(), v) for k, v in kv]
    for k, _ in fine:
        k[:, 0] = 0.0
    t0 = 0
    mended = out.clone()
    for (p, t), (k, v) in zip(spec, fine):
        n = len(t)
        mended[t0:t0 + n, :4] = bf(ot.attention(f64(q[t0:t0 + n]), f64(k), f64(v), p, t)[0][:, :4])
        t0 += n
    check_attention(mended, q, fine, spec, d)
    eng.close()
