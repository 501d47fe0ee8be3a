"""The operators on drafted tokens where a fixed size inside a kernel ends: lists, branches and biases longer than a block keeps, rows that
share blocks, more rows than one launch's workspace holds, nodes too far apart for a launch's packed lists, replays beside other calls.
Tolerances and oracles are those of test_gpu_tree."""
import numpy as np
import pytest
import torch

from paper_2507_17769_amd.runner import Engine
from test_gpu_tree import chain, check_picks, make_batch, make_engine, make_rules, pool_rows, random_tree, rows_by_rules

pytestmark = pytest.mark.gpu


def masks_for(rng, rows, V):
    words = (V + 31) // 32
    mask = np.where(rng.random((rows, words)) < 0.4, rng.integers(0, 1 << 32, (rows, words)), 0).astype(np.uint32).view(np.int32)
    return {"mask": mask, "mask_row": rng.integers(-1, rows, rows).astype(np.int32)}


# 1000 tokens hold all the list's: a branch of hundreds and biases of hundreds, with repeats on both sides of what a block keeps
@pytest.mark.parametrize("rows,V,n_bias,tokens", [(150, 1200, 700, 40), (300, 5000, 257, 2), (40, 70000, 2500, 300)])
def test_branches_and_biases_longer_than_a_block_keeps(rows, V, n_bias, tokens):
    rng = np.random.default_rng(rows)
    eng = Engine("tiny", 1, max_position=16)
    tree = {"row_list": np.zeros(rows, np.int32), "row_prev": np.arange(-1, rows - 1, dtype=np.int32),
            "row_token": rng.integers(0, tokens, rows).astype(np.int32)}
    _, r = make_rules(rng, 1, V, 500, 0, tree=tree)
    r["bias_token"] = rng.integers(0, min(V, 1000), n_bias).astype(np.int32)
    r["bias_value"] = (rng.standard_normal(n_bias) * 5).astype(np.float32)
    r["bias_begin"] = np.array([0, n_bias], np.int32)
    dev = {k: torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in r.items()}
    z = torch.from_numpy((rng.standard_normal((rows, V)) * 3).astype(np.float32)).cuda()
    check_picks(eng.pick_tokens(z, dev, want_logits=True), rows_by_rules(z.cpu().numpy(), r, V, rows))
    eng.close()


# enough tokens that a block takes several rows, whose lists change inside it, with and without whole quads of logits
@pytest.mark.parametrize("rows,V,dtype,ordered", [(50, 140000, "f32", True), (203, 70001, "bf16", False), (520, 50000, "f32", True), (515, 50002, "bf16", False)])
def test_rows_of_one_block_with_lists_of_their_own(rows, V, dtype, ordered):
    rng = np.random.default_rng(V)
    eng = Engine("tiny", 1, max_position=16)
    n_lists = 1 + rows // 5
    lists = rng.integers(-1, n_lists + 1, rows).astype(np.int32)
    if ordered:
        lists = np.sort(lists)
    prev = np.array([int(rng.integers(max(-1, i - 3), i)) for i in range(rows)], np.int32)
    token = rng.integers(-1, 30, rows).astype(np.int32)
    dev, r = make_rules(rng, n_lists, V, 60, 10, tree={"row_list": lists, "row_prev": prev, "row_token": token}, masks=masks_for(rng, rows, V))
    z = torch.from_numpy((rng.standard_normal((rows, V)) * 3).astype(np.float32)).cuda()
    z = z.to(torch.bfloat16) if dtype == "bf16" else z
    check_picks(eng.pick_tokens(z, dev, want_logits=True), rows_by_rules(z.float().cpu().numpy(), r, V, rows))
    eng.close()


def test_more_rows_than_a_launch_takes():
    rng = np.random.default_rng(4)
    eng = Engine("tiny", 1, max_position=16)
    rows, V = 9000, 96                                  # two launches and a part of one
    dev, r = make_rules(rng, rows, V, 6, 4, masks=masks_for(rng, rows, V))
    z = torch.from_numpy((rng.standard_normal((rows, V)) * 3).astype(np.float32)).cuda()
    want = rows_by_rules(z.cpu().numpy(), r, V, rows)
    check_picks(eng.pick_tokens(z, dev, want_logits=True), want)
    # many segments a row: the partial results of fewer rows fit; trees whose branches cross the launches
    rows, V = 300, 1 << 20
    z = torch.empty(rows, V, dtype=torch.bfloat16, device="cuda").normal_(0, 3, generator=torch.Generator("cuda").manual_seed(1))
    prev = torch.arange(-1, rows - 1, dtype=torch.int32, device="cuda")
    best = z.argmax(-1).tolist()
    token = torch.full((rows,), -1, dtype=torch.int32)
    token[::10] = torch.tensor(best[::10], dtype=torch.int32)
    rules = {"frequency": torch.tensor([1e4], device="cuda"), "row_list": torch.zeros(rows, dtype=torch.int32, device="cuda"), "row_prev": prev, "row_token": token.cuda()}
    got = eng.pick_tokens(z, rules)
    nxt, lp = got["next"].cpu().numpy(), got["logprob"].cpu().numpy().astype(np.float64)
    out = set()
    for i in range(rows):
        if token[i] >= 0:
            out.add(int(token[i]))
        x = z[i].double()
        x[torch.tensor(sorted(out), device="cuda")] -= 1e4
        top = x.max()
        assert nxt[i] == int((x == top).nonzero()[0]), i
        w = torch.exp(x - top)
        want, mean = -float(torch.log(w.sum())), float((w * (1.5 * (x - top).abs() + 4)).sum() / w.sum())
        assert abs(lp[i] - want) <= (mean + V + 2 * abs(want)) * 2.0 ** -24, (i, lp[i], want)
    eng.close()


def test_kept_nodes_far_apart():
    n = 70000
    rng = np.random.default_rng(9)
    spec = [(21, chain(n)), (40, chain(3))]
    seqs, parents, pages, n_pages = make_batch(rng, spec)
    eng = make_engine(2, 1, 64, n_pages, max_position=n + 100)
    pool = eng.kv_pool()
    pool.copy_(torch.randint(-2 ** 15, 2 ** 15, pool.shape, dtype=torch.int16, generator=torch.Generator().manual_seed(3)).view(torch.bfloat16).to(pool.device))
    torch.cuda.synchronize()
    before = pool[0].clone()
    keep = [np.array([0, 2, 5, 30, 65530, 65539, 69990, 69999]), np.array([1, 2])]
    eng.tree_keep(eng.tree(seqs, parents), keep)
    eng.ctx.sync()
    for (p, t), pg, ks in zip(spec, pages, keep):
        moved = p + np.arange(len(ks))
        for was, now in zip(pool_rows(before, pg, p + ks), pool_rows(pool[0], pg, moved)):
            assert torch.equal(was.contiguous().view(torch.int16), now.contiguous().view(torch.int16))
        rest = np.setdiff1d(np.arange(p + len(t)), moved)
        for was, now in zip(pool_rows(before, pg, rest), pool_rows(pool[0], pg, rest)):
            assert torch.equal(was.contiguous().view(torch.int16), now.contiguous().view(torch.int16))
    eng.close()


def test_picks_of_replays_and_of_calls_between_them():
    """Counters of arrived blocks are left at zero by every launch, in whatever order a graph's launches and others come."""
    rng = np.random.default_rng(8)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        eng = Engine("tiny", 1, max_position=16)
        V = 40000
        z = torch.from_numpy((rng.standard_normal((12, V)) * 3).astype(np.float32)).cuda()
        dev, r = make_rules(rng, 12, V, 60, 10)
        other = torch.from_numpy((rng.standard_normal((5, 2 * V)) * 3).astype(np.float32)).cuda()
        eng.pick_tokens(z, dev)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            captured = eng.pick_tokens(z, dev, want_logits=True)
        for turn in range(4):
            z.copy_(torch.from_numpy((rng.standard_normal((12, V)) * 3).astype(np.float32)))
            graph.replay()
            got = eng.pick_tokens(other)
            stream.synchronize()
            check_picks(captured, rows_by_rules(z.cpu().numpy(), r, V, 12))
            check_picks(got, other.cpu().numpy(), full=False)
    eng.close()


@pytest.mark.parametrize("n_q,n_kv,d", [(4, 2, 64), (32, 8, 128), (64, 8, 128)])
@pytest.mark.parametrize("prefix,n", [(700, 3), (1500, 40), (40, 64)])
def test_a_row_depends_on_no_other_rows_query(n_q, n_kv, d, prefix, n):
    """To the bit: what the softmax of a tile does for one of its rows is not seen in another."""
    rng = np.random.default_rng(prefix + n_q)
    spec = [(prefix, random_tree(rng, n)), (prefix // 2, random_tree(rng, n))]
    seqs, parents, pages, n_pages = make_batch(rng, spec)
    eng = make_engine(n_q, n_kv, d, n_pages)
    eng.kv_pool().normal_(generator=torch.Generator("cuda").manual_seed(1))
    tree = eng.tree(seqs, parents)
    q = torch.randn(2 * n, n_q, d, device="cuda", generator=torch.Generator("cuda").manual_seed(2)).to(torch.bfloat16)
    loud = q.clone()
    loud[::2] *= 40
    nan = q.clone()
    nan[::2] = float("nan")
    out = [eng.tree_attention(0, tree, x) for x in (q, loud, nan)]
    eng.ctx.sync()
    assert torch.isfinite(out[0].float()).all()
    assert torch.equal(out[0][1::2], out[1][1::2]) and torch.equal(out[0][1::2], out[2][1::2])
    assert not torch.equal(out[0][::2], out[1][::2])
    eng.close()
