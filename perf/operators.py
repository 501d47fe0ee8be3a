"""The operators of a step that verifies drafted tokens, each on its own: their plain forms and the calls a user makes of them.

A batch holds sequences with a cached prefix each and new tokens ("nodes") that form a tree: a node attends to the prefix, to its
ancestors and to itself.  Node i of a sequence is stored at slot prefix + i and rotated for position prefix + depth.  The operators:

  norm_rope   queries and keys normalised head by head, rotated, and appended to the paged cache with the values
  attention   every node over its branch and the cached prefix
  pick        penalties for repeated tokens, biases and grammar masks on logits; the most likely token and its log-probability
  keep        the cache rows of an accepted branch become the prefix's next positions, in all layers

Head layouts are those of the repository's models ("tiny", "8b", "70b") in the listed cases and any supported one in the drawn cases;
the vocabulary is the benchmark's.  A case is a dict of plain values:

  op          one of the above
  n_q, n_kv, dim            head layout
  seqs, nodes, shape        sequences; nodes of each ("ragged": 1 to that many; "tree"/"chain": exactly that many)
  lo, hi                    cached prefix lengths, uniform in between
  pad                       share of the sequences whose last nodes are padding (a drafter's fixed tree, cut short)
  dtype, gap                type of the projection or of the logits; elements between two rows beyond their length
  rows, vocab, history, biases, masks, tree, full     pick: logit rows, list lengths, share of rows under a grammar, rows as nodes of
                            trees of this many (0: a sequence each), whether the changed logits are wanted too
  lengths     seed of the lengths and trees, so that a case always means the same work
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 16
EPS, BASE = 1e-5, 500000.0
DEV = "cuda"


def _batch(case):
    """Per sequence: (prefix, parents as int32 array)."""
    r = random.Random(case["lengths"])
    out = []
    for s in range(case["seqs"]):
        n = case["nodes"] if case["shape"] != "ragged" else r.randint(1, case["nodes"])
        prefix = r.randint(case["lo"], case["hi"])
        if case["shape"] == "chain":
            parents = list(range(-1, n - 1))
        else:   # each node hangs below one of the eight before it, or below the prefix
            parents = [r.randint(max(-1, i - 8), i - 1) for i in range(n)]
        if n > 1 and r.random() < case["pad"]:
            for i in range(n - r.randint(1, n // 2), n):
                parents[i] = -2
        out.append((prefix, np.array(parents, dtype=np.int32)))
    return out


def _depths(parents):
    d = np.zeros(len(parents), dtype=np.int64)
    for i, p in enumerate(parents):
        d[i] = d[p] + 1 if p >= 0 else 0
    return d


def _ancestors(parents):
    """[n][n] truth values: node j is node i or one of its ancestors; nothing for padding."""
    n = len(parents)
    a = np.zeros((n, n), dtype=bool)
    for i, p in enumerate(parents):
        if p >= 0:
            a[i] = a[p]
        a[i, i] = p > -2
    return a


def _tables(case, batch):
    """Page tables, drawn without repeats from a pool with some pages to spare."""
    need = [(p + len(t) + PAGE - 1) // PAGE for p, t in batch]
    n_pages = sum(need) + sum(need) // 8 + 2
    perm = np.random.RandomState(case["lengths"]).permutation(n_pages).astype(np.int32)
    at = np.concatenate([[0], np.cumsum(need)])
    return [perm[at[i]:at[i + 1]] for i in range(len(need))], n_pages


def _kept(case, batch):
    """Nodes of the longest branch of each tree, ascending: what a verifier accepts at best."""
    out = []
    for _, parents in batch:
        d = np.where(parents > -2, _depths(parents), -1)
        i, path = int(np.argmax(d)), []
        while i >= 0:
            path.append(i)
            i = int(parents[i])
        out.append(np.array(path[::-1], dtype=np.int32))
    return out


def listed():
    return [
        # one decode token of the smallest model: what a launch costs
        dict(name="norm_rope_1_token", op="norm_rope", n_q=4, n_kv=2, dim=64, seqs=1, nodes=1, shape="chain", lo=17, hi=17, pad=0.0, dtype="float32", gap=0, lengths=1),
        # an ordinary verification batch: 16 requests with five drafted tokens and the last accepted one
        dict(name="norm_rope_8b_96", op="norm_rope", n_q=32, n_kv=8, dim=128, seqs=16, nodes=6, shape="tree", lo=100, hi=900, pad=0.0, dtype="float32", gap=0, lengths=2),
        # many wide trees, a projection of bf16 rows inside wider rows, odd token counts
        dict(name="norm_rope_70b_2016", op="norm_rope", n_q=64, n_kv=8, dim=128, seqs=32, nodes=63, shape="tree", lo=0, hi=250, pad=0.5, dtype="bfloat16", gap=64, lengths=3),
        # the smallest call: one token over two pages
        dict(name="attention_1_node", op="attention", n_q=4, n_kv=2, dim=64, seqs=1, nodes=1, shape="chain", lo=17, hi=17, pad=0.0, lengths=4),
        # a draft model's chain of five at medium prefixes, few requests
        dict(name="attention_8b_chains", op="attention", n_q=32, n_kv=8, dim=128, seqs=8, nodes=6, shape="chain", lo=512, hi=4096, pad=0.0, lengths=5),
        # a busy server: 32 requests with trees of 16
        dict(name="attention_8b_trees_16", op="attention", n_q=32, n_kv=8, dim=128, seqs=32, nodes=16, shape="tree", lo=512, hi=4096, pad=0.25, lengths=6),
        # wide trees over long caches, ragged and padded
        dict(name="attention_70b_trees_64", op="attention", n_q=64, n_kv=8, dim=128, seqs=16, nodes=64, shape="ragged", lo=1000, hi=8000, pad=0.5, lengths=7),
        # one request answered alone
        dict(name="pick_1_row", op="pick", rows=1, vocab=128256, dtype="float32", gap=0, history=1500, biases=16, masks=1.0, tree=0, full=False, lengths=8),
        # a decode batch with everything on, logits of bf16, and the changed logits for a sampler
        dict(name="pick_64_rows", op="pick", rows=64, vocab=128256, dtype="bfloat16", gap=0, history=4000, biases=300, masks=0.5, tree=0, full=True, lengths=9),
        # verification of eight trees of 63 nodes
        dict(name="pick_504_nodes", op="pick", rows=504, vocab=128256, dtype="float32", gap=0, history=2000, biases=32, masks=0.25, tree=63, full=False, lengths=10),
        # one request's accepted branch in a small model
        dict(name="keep_1_seq", op="keep", n_q=4, n_kv=2, dim=64, layers=1, seqs=1, nodes=8, shape="tree", lo=30, hi=30, pad=0.0, lengths=11),
        # a busy server's branches in four layers
        dict(name="keep_64_seqs", op="keep", n_q=32, n_kv=8, dim=128, layers=4, seqs=64, nodes=64, shape="tree", lo=0, hi=400, pad=0.25, lengths=12),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    op = rng.choice(["norm_rope", "attention", "attention", "pick", "pick", "keep"])
    c = dict(op=op, lengths=rng.randrange(1 << 30))
    if op == "pick":
        tree, full = rng.choice([0, 0, _log(rng, 2, 64)]), rng.random() < 0.5
        rows = _log(rng, 1, 120 if full else 250)
        c.update(rows=max(1, rows // tree) * tree if tree else rows, vocab=_log(rng, 500, 200000), dtype=rng.choice(["float32", "bfloat16"]),
                 gap=rng.choice([0, 0, 3, 64]), history=_log(rng, 1, 6000), biases=rng.choice([0, _log(rng, 1, 300)]), masks=rng.choice([0.0, 0.5, 1.0]),
                 tree=tree, full=full)
        return c
    n_kv = rng.choice([1, 2, 4, 8])
    c.update(n_kv=n_kv, n_q=n_kv * rng.choice([1, 2, 4, 8, 16]) if n_kv < 8 else rng.choice([8, 32, 64]), dim=rng.choice([64, 128]),
             seqs=_log(rng, 1, 32), nodes=_log(rng, 1, 64), shape=rng.choice(["tree", "ragged", "chain"]), pad=rng.choice([0.0, 0.5]))
    if op == "attention":
        c["seqs"] = min(c["seqs"], max(1, 500 // c["nodes"]))
        c["lo"] = _log(rng, 1, 1000) - 1
        c["hi"] = c["lo"] + _log(rng, 1, 2500)
    else:
        c["lo"] = rng.randint(0, 200)
        c["hi"] = c["lo"] + rng.randint(0, 200)
        if op == "norm_rope":
            c.update(dtype=rng.choice(["float32", "bfloat16"]), gap=rng.choice([0, 8, 64]))
        else:
            c["layers"] = rng.randint(1, 4)
    return c


def work(case):
    if case["op"] == "pick":
        rows, V, size = case["rows"], case["vocab"], 4 if case["dtype"] == "float32" else 2
        lists, masks = _lists(case), int(round(case["masks"] * rows))
        b = rows * V * (size + (4 if case["full"] else 0)) + masks * (V / 8) + 4 * int(lists["history_begin"][-1]) + 8 * int(lists["bias_begin"][-1]) + 8 * rows
        return {"bytes": b, "flops": 6 * rows * V}
    batch = _batch(case)
    T, nq, nkv, d = sum(len(t) for _, t in batch), case["n_q"], case["n_kv"], case["dim"]
    if case["op"] == "norm_rope":
        size = 4 if case["dtype"] == "float32" else 2
        return {"bytes": T * (nq + 2 * nkv) * d * (size + 2), "flops": 10 * T * (nq + nkv) * d}
    if case["op"] == "keep":
        moved = sum(int((k != np.arange(len(k))).sum()) for k in _kept(case, batch))
        return {"bytes": max(1, moved) * case["layers"] * nkv * d * 4 * 2, "flops": 0}
    seen = sum(int(_ancestors(t).sum()) + p * int((t > -2).sum()) for p, t in batch)
    return {"bytes": sum(p + len(t) for p, t in batch) * nkv * d * 4 + T * nq * d * 4, "flops": 4 * d * nq * seen}


# ---------------------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _lists(case):
    """pick: lengths of the sequences' token and bias lists (one list for a sequence, whose rows are one token or a tree)."""
    r = random.Random(case["lengths"])
    n = case["rows"] // case["tree"] if case["tree"] else case["rows"]
    hist = [r.randint(0, case["history"]) for _ in range(n)]
    hist[0] = case["history"]
    prompt = [r.randint(0, h) for h in hist]
    bias = [r.randint(0, case["biases"]) for _ in range(n)]
    begin = np.concatenate([[0], np.cumsum(hist)]).astype(np.int32)
    return {"n": n, "history_begin": begin, "output_begin": (begin[:-1] + np.array(prompt)).astype(np.int32),
            "bias_begin": np.concatenate([[0], np.cumsum(bias)]).astype(np.int32)}


def _pick_inputs(case, seed):
    rows, V = case["rows"], case["vocab"]
    g, ls = _gen(seed), _lists(case)
    n = ls["n"]
    base = torch.randn(rows, V + case["gap"], generator=g, device=DEV) * 2.5
    base = base.to(getattr(torch, case["dtype"]))

    def dev(a):
        return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)

    def uniform(lo, hi, k):
        return torch.rand(k, generator=g, device=DEV) * (hi - lo) + lo

    # tokens repeat: half of a text comes from a small part of the vocabulary
    H, Bn = int(ls["history_begin"][-1]), int(ls["bias_begin"][-1])
    wide = torch.randint(0, V, (H,), generator=g, device=DEV, dtype=torch.int32)
    near = torch.randint(0, max(1, V // 100), (H,), generator=g, device=DEV, dtype=torch.int32)
    x = {"logits": base[:, :V], "history": torch.where(torch.rand(H, generator=g, device=DEV) < 0.5, wide, near),
         "history_begin": dev(ls["history_begin"]), "output_begin": dev(ls["output_begin"]),
         "repetition": uniform(1.0, 1.5, n), "frequency": uniform(-0.2, 0.8, n), "presence": uniform(0.0, 0.6, n),
         "bias_begin": dev(ls["bias_begin"]), "bias_token": torch.randint(0, V, (Bn,), generator=g, device=DEV, dtype=torch.int32),
         "bias_value": torch.randn(Bn, generator=g, device=DEV) * 4.0}
    n_masks = int(round(case["masks"] * rows))
    words = (V + 31) // 32
    m = torch.randint(0, 1 << 32, (n_masks, words), generator=g, device=DEV, dtype=torch.int64)
    keep = torch.rand(n_masks, words, generator=g, device=DEV) < 0.2   # a grammar allows a small part
    m = torch.where(keep, m, torch.zeros_like(m))
    if n_masks > 4:
        m[3] = 0                                                    # a grammar that has ended allows nothing
    x["mask"] = (m - ((m >> 31) << 32)).to(torch.int32)               # the same 32 bits
    order = torch.randperm(rows, generator=g, device=DEV)
    mask_row = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    mask_row[order[:n_masks]] = torch.arange(n_masks, dtype=torch.int32, device=DEV)
    x["mask_row"] = mask_row
    if case["tree"]:
        r = random.Random(case["lengths"] + 1)
        k = case["tree"]
        prev, lists = [], []
        for s in range(n):
            prev += [-1] + [s * k + r.randint(max(0, i - 8), i - 1) for i in range(1, k)]
            lists += [s] * k
        x["row_prev"], x["row_list"] = dev(np.array(prev, dtype=np.int32)), dev(np.array(lists, dtype=np.int32))
        x["row_token"] = torch.randint(0, max(1, V // 50), (rows,), generator=g, device=DEV, dtype=torch.int32)
        depth = max(1, int(_depths(np.array(prev, dtype=np.int32)).max()) + 1)
        chain = np.full((rows, depth), -1, dtype=np.int64)         # rows whose tokens a row has behind it
        for i in range(rows):
            j, e = i, 0
            while j >= 0:
                chain[i, e] = j
                j, e = prev[j], e + 1
        x["chain"] = dev(chain)
    return x


def _cache_inputs(case, seed):
    batch = _batch(case)
    tables, n_pages = _tables(case, batch)
    g, nq, nkv, d = _gen(seed), case["n_q"], case["n_kv"], case["dim"]
    T = sum(len(t) for _, t in batch)
    x = {"batch": batch, "tables": tables, "n_pages": n_pages, "T": T,
         "pool": torch.randn(case.get("layers", 1), n_pages, nkv, 2, PAGE * d, generator=g, device=DEV).to(torch.bfloat16)}
    if case["op"] == "norm_rope":
        width = (nq + 2 * nkv) * d
        x["qkv"] = (torch.randn(T, width + case["gap"], generator=g, device=DEV) * 1.5).to(getattr(torch, case["dtype"]))[:, :width]
        x["g_q"] = (1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
        x["g_k"] = (1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
    if case["op"] == "attention":
        x["q"] = (torch.randn(T, nq, d, generator=g, device=DEV) * 1.5).to(torch.bfloat16)
    if case["op"] == "keep":
        x["kept"] = _kept(case, batch)
    return x


def _slots(x, positions):
    """Device page ids and places of logical positions, one array of them for each sequence."""
    page = np.concatenate([t[p // PAGE] for t, p in zip(x["tables"], positions)])
    place = np.concatenate([p % PAGE for p in positions])
    return torch.from_numpy(page.astype(np.int64)).to(DEV), torch.from_numpy(place.astype(np.int64)).to(DEV)


def prepare(case, seed):
    s = {"case": case}
    if case["op"] == "pick":
        s.update(_pick_inputs(case, seed))
        if own:
            from paper_2507_17769_amd.runner import Engine
            s["engine"] = Engine("tiny", 1, max_position=PAGE)
            s["rules"] = {k: s[k] for k in ("history", "history_begin", "output_begin", "repetition", "frequency", "presence", "bias_token",
                                            "bias_value", "bias_begin", "mask", "mask_row", "row_list", "row_prev", "row_token") if k in s}
        return s
    x = _cache_inputs(case, seed)
    s.update(x)
    batch = x["batch"]
    if own:
        from paper_2507_17769_amd.runner import Engine
        model = dict(hidden=256, n_q=case["n_q"], n_kv=case["n_kv"], head_dim=case["dim"], ffn=256, rope_base=BASE)
        layers = case.get("layers", 1)
        eng = Engine(model, x["n_pages"], layers, layers, max_position=max(p + len(t) for p, t in batch))
        s["pool"] = eng.kv_pool().copy_(x["pool"])
        if case["op"] == "norm_rope":
            eng.load_qk_norm(0, x["g_q"], x["g_k"])
        s["engine"] = eng
        s["tree"] = eng.tree([(i, len(t), p + len(t), pages) for i, ((p, t), pages) in enumerate(zip(batch, x["tables"]))],
                             np.concatenate([t for _, t in batch]))
        return s
    if case["op"] == "norm_rope":
        s["page"], s["place"] = _slots(x, [p + np.arange(len(t)) for p, t in batch])
        s["position"] = torch.from_numpy(np.concatenate([p + _depths(t) for p, t in batch])).to(DEV)
    elif case["op"] == "keep":
        s["from"] = _slots(x, [p + k for (p, _), k in zip(batch, x["kept"])])
        s["to"] = _slots(x, [p + np.arange(len(k)) for (p, _), k in zip(batch, x["kept"])])
    else:
        n_max, L = max(len(t) for _, t in batch), max(p + len(t) for p, t in batch)
        n_pg = (L + PAGE - 1) // PAGE
        pages = np.zeros((len(batch), n_pg), dtype=np.int64)
        visible = np.zeros((len(batch), n_max, n_pg * PAGE), dtype=bool)
        row = np.full((len(batch), n_max), x["T"], dtype=np.int64)    # one past the last row: a row of zeros
        at = 0
        for b, ((p, t), table) in enumerate(zip(batch, x["tables"])):
            n = len(t)
            pages[b, :len(table)] = table
            visible[b, :n, :p] = (t > -2)[:, None]
            visible[b, :n, p:p + n] = _ancestors(t)
            row[b, :n] = at + np.arange(n)
            at += n
        s["pages"], s["visible"], s["row"] = (torch.from_numpy(a).to(DEV) for a in (pages, visible, row))
    return s


# ----------------------------------------------------------------------------------------------------------------- plain
def _keys_of(pool, d):
    """A layer's pool as keys: [page][kv head][d/32][4][place][8]."""
    return pool[:, :, 0].view(pool.shape[0], pool.shape[1], d // 32, 4, PAGE, 8)


def _values_of(pool, d):
    """A layer's pool as values: [page][kv head][d/32][place/4][d%16][d/16%2][place%4]."""
    return pool[:, :, 1].view(pool.shape[0], pool.shape[1], d // 32, 4, 16, 2, 4)


def _plain_norm_rope(s):
    c = s["case"]
    T, nq, nkv, d = s["T"], c["n_q"], c["n_kv"], c["dim"]
    x = s["qkv"].float().view(T, nq + 2 * nkv, d)
    gain = torch.cat([s["g_q"].float().expand(nq, d), s["g_k"].float().expand(nkv, d)])
    qk = x[:, :nq + nkv]
    qk = qk * torch.rsqrt((qk * qk).mean(-1, keepdim=True) + EPS) * gain
    theta = BASE ** (-2.0 * torch.arange(d // 2, device=DEV, dtype=torch.float64) / d)
    phi = s["position"].double()[:, None] * theta
    co, si = phi.cos().float()[:, None], phi.sin().float()[:, None]
    lo, hi = qk[..., :d // 2], qk[..., d // 2:]
    qk = torch.cat([lo * co - hi * si, hi * co + lo * si], -1).to(torch.bfloat16)
    pool = s["pool"][0]
    page, place = s["page"], s["place"]
    _keys_of(pool, d)[page, :, :, :, place] = qk[:, nq:].reshape(T, nkv, d // 32, 4, 8)
    v = x[:, nq + nkv:].to(torch.bfloat16).reshape(T, nkv, d // 32, 2, 16).transpose(-1, -2)
    _values_of(pool, d)[page, :, :, place // 4, :, :, place % 4] = v
    return {"q": qk[:, :nq].contiguous(), "pool": s["pool"]}


def _plain_attention(s):
    c = s["case"]
    nq, nkv, d = c["n_q"], c["n_kv"], c["dim"]
    B, n_pg = s["pages"].shape
    n, L, G = s["row"].shape[1], n_pg * PAGE, nq // nkv
    pool = s["pool"][0]
    k = _keys_of(pool, d)[s["pages"]].permute(0, 2, 1, 5, 3, 4, 6).reshape(B, nkv, L, d).float()
    v = _values_of(pool, d)[s["pages"]].permute(0, 2, 1, 4, 7, 3, 6, 5).reshape(B, nkv, L, d).float()
    q = torch.cat([s["q"], s["q"].new_zeros(1, nq, d)])[s["row"]].float()
    q = q.view(B, n, nkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, nkv, n * G, d)
    z = torch.matmul(q, k.transpose(-1, -2)).view(B, nkv, n, G, L) * (1.0 / math.sqrt(d))
    z = z.masked_fill(~s["visible"][:, None, :, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    w = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(B, nkv, n * G, L), v).view(B, nkv, n, G, d) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.permute(0, 2, 1, 3, 4).reshape(B, n, nq, d).to(torch.bfloat16)
    out = torch.empty(s["T"] + 1, nq, d, dtype=torch.bfloat16, device=DEV)
    out[s["row"]] = o
    return {"out": out[:s["T"]]}


def _lists_of(begin, total):
    """The list that each entry of a ragged array belongs to."""
    return torch.searchsorted(begin[1:].contiguous(), torch.arange(total, device=DEV, dtype=begin.dtype), right=True)


def _plain_pick(s):
    c = s["case"]
    rows, V = c["rows"], c["vocab"]
    n = s["repetition"].shape[0]
    H, Bn = s["history"].shape[0], s["bias_token"].shape[0]
    owner = _lists_of(s["history_begin"], H)
    made = torch.arange(H, device=DEV) >= s["output_begin"].long()[owner]
    flat = owner * V + s["history"].long()
    count = torch.zeros(n * V, device=DEV).index_add_(0, flat, made.float()).view(n, V)
    prompt = torch.zeros(n * V, dtype=torch.bool, device=DEV)
    prompt[flat[~made]] = True
    prompt = prompt.view(n, V)
    # of two biases of a token, the later one
    place = torch.full((n * V,), -1, dtype=torch.long, device=DEV)
    place.scatter_reduce_(0, _lists_of(s["bias_begin"], Bn) * V + s["bias_token"].long(), torch.arange(Bn, device=DEV), "amax")
    bias = torch.where(place >= 0, torch.cat([s["bias_value"], s["bias_value"].new_zeros(1)])[place], torch.zeros((), device=DEV)).view(n, V)
    if c["tree"]:
        of = s["row_list"].long()
        count, prompt, bias = count[of], prompt[of], bias[of]
        behind = s["chain"] >= 0
        token = s["row_token"].long()[s["chain"].clamp(min=0)]
        count.scatter_add_(1, token, behind.float())
    else:
        of = torch.arange(n, device=DEV)
    rep, freq, pres = (s[k][of][:, None] for k in ("repetition", "frequency", "presence"))
    z = s["logits"].float()
    z = torch.where(prompt | (count > 0), torch.where(z > 0, z / rep, z * rep), z)
    z = z - freq * count
    z = torch.where(count > 0, z - pres, z) + bias
    if s["mask"].shape[0]:
        bits = (s["mask"][:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
        allowed = bits.view(s["mask"].shape[0], -1)[:, :V].bool()
        held = s["mask_row"] >= 0
        allowed = torch.where(held[:, None], allowed[s["mask_row"].clamp(min=0).long()], torch.ones((), dtype=torch.bool, device=DEV))
        z = z.masked_fill(~allowed, -math.inf)
    top = z.amax(-1, keepdim=True)
    index = torch.arange(V, device=DEV)
    pick = torch.where((z == top) & (top > -math.inf), index, V).amin(-1)
    total = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top)).sum(-1)
    logprob = torch.where(pick < V, -torch.log(total), torch.full_like(total, -math.inf))
    out = {"next": torch.where(pick < V, pick, -torch.ones_like(pick)).to(torch.int32), "logprob": logprob}
    if c["full"]:
        out["logits"] = z
    return out


def _plain_keep(s):
    d = s["case"]["dim"]
    pool = s["pool"]
    (p0, t0), (p1, t1) = s["from"], s["to"]
    layers, pages, nkv = pool.shape[:3]
    k = pool[:, :, :, 0].view(layers, pages, nkv, d // 32, 4, PAGE, 8)
    v = pool[:, :, :, 1].view(layers, pages, nkv, d // 32, 4, 16, 2, 4)
    k[:, p1, :, :, :, t1] = k[:, p0, :, :, :, t0]
    v[:, p1, :, :, t1 // 4, :, :, t1 % 4] = v[:, p0, :, :, t0 // 4, :, :, t0 % 4]
    return {"pool": pool}


def run(state):
    op = state["case"]["op"]
    if own:
        eng = state["engine"]
        if op == "norm_rope":
            return {"q": eng.qk_norm_rope(0, state["tree"], state["qkv"]), "pool": state["pool"]}
        if op == "attention":
            return {"out": eng.tree_attention(0, state["tree"], state["q"])}
        if op == "keep":
            eng.tree_keep(state["tree"], state["kept"])
            return {"pool": state["pool"]}
        return eng.pick_tokens(state["logits"], state["rules"], want_logits=state["case"]["full"])
    return {"norm_rope": _plain_norm_rope, "attention": _plain_attention, "pick": _plain_pick, "keep": _plain_keep}[op](state)


# ----------------------------------------------------------------------------------------------------------------- exact
def _places(x, b, positions):
    """(page, place) of logical positions of sequence b, as lists."""
    return [int(x["tables"][b][p // PAGE]) for p in positions], [int(p % PAGE) for p in positions]


def exact(case, seed):
    if case["op"] == "pick":
        return _exact_pick(case, _pick_inputs(case, seed))
    x = _cache_inputs(case, seed)
    d, nkv, nq = case["dim"], case["n_kv"], case["n_q"]
    if case["op"] == "keep":
        return None   # moved bits: compared as such
    pool = x["pool"].double()
    kk = pool[0, :, :, 0].view(-1, nkv, d // 8, PAGE, 8)                 # eight values of a token after another
    vv = pool[0, :, :, 1].view(-1, nkv, d // 32, PAGE // 4, 16, 2, 4)
    if case["op"] == "norm_rope":
        q = torch.empty(x["T"], nq, d, dtype=torch.float64, device=DEV)
        theta = torch.tensor([BASE ** (-2.0 * j / d) for j in range(d // 2)], dtype=torch.float64, device=DEV)
        at = 0
        for b, (p, t) in enumerate(x["batch"]):
            n = len(t)
            rows = x["qkv"][at:at + n].double().view(n, -1, d)
            turn = torch.polar(torch.ones(n, d // 2, dtype=torch.float64, device=DEV),
                               torch.from_numpy(p + _depths(t)).to(DEV).double()[:, None] * theta)

            def turned(u, gain):
                u = u / (u.square().mean(-1, keepdim=True) + EPS).sqrt() * gain.double()
                u = torch.complex(u[..., :d // 2], u[..., d // 2:]) * turn[:, None]
                return torch.cat([u.real, u.imag], -1)

            q[at:at + n] = turned(rows[:, :nq], x["g_q"])
            page, place = _places(x, b, p + np.arange(n))
            kk[page, :, :, place] = turned(rows[:, nq:nq + nkv], x["g_k"]).view(n, nkv, d // 8, 8)
            v = rows[:, nq + nkv:]
            for i in range(n):
                vv[page[i], :, :, place[i] // 4, :, :, place[i] % 4] = v[i].view(nkv, d // 32, 2, 16).transpose(-1, -2)
            at += n
        return {"q": q, "pool": pool}
    out = torch.zeros(x["T"], nq, d, dtype=torch.float64, device=DEV)
    at = 0
    for b, (p, t) in enumerate(x["batch"]):
        n = len(t)
        table = torch.from_numpy(x["tables"][b].astype(np.int64)).to(DEV)
        k = kk[table].permute(1, 0, 3, 2, 4).reshape(nkv, -1, d)[:, :p + n]
        v = vv[table].permute(1, 0, 3, 6, 2, 5, 4).reshape(nkv, -1, d)[:, :p + n]
        sees = torch.cat([torch.ones(n, p, dtype=torch.bool), torch.from_numpy(_ancestors(t))], 1).to(DEV)
        live = torch.from_numpy(t > -2).to(DEV)
        q = x["q"][at:at + n].double().view(n, nkv, -1, d)
        for h in range(nkv):
            z = torch.matmul(q[live, h].reshape(-1, d), k[h].t().contiguous()).view(int(live.sum()), nq // nkv, -1) / math.sqrt(d)
            w = torch.softmax(z.masked_fill(~sees[live][:, None], -math.inf), -1)
            got = torch.matmul(w.view(-1, p + n), v[h]).view(-1, nq // nkv, d)
            part = torch.zeros(n, nq // nkv, d, dtype=torch.float64, device=DEV)
            part[live] = got
            out[at:at + n, h * (nq // nkv):(h + 1) * (nq // nkv)] = part
        at += n
    return {"out": out}


def _exact_pick(case, x):
    rows, V = case["rows"], case["vocab"]
    h = {k: x[k].cpu().numpy() for k in ("history", "history_begin", "output_begin", "repetition", "frequency", "presence", "bias_begin",
                                         "bias_token", "bias_value", "mask", "mask_row")}
    tree = {k: x[k].cpu().numpy() for k in ("row_list", "row_token", "chain")} if case["tree"] else None
    z = x["logits"].double()
    logprob = np.empty(rows)
    whole = torch.empty(rows, V, dtype=torch.float64, device=DEV) if case["full"] else None
    for i in range(rows):
        s = int(tree["row_list"][i]) if tree else i
        b0, b1, bo = int(h["history_begin"][s]), int(h["history_begin"][s + 1]), int(h["output_begin"][s])
        made = h["history"][bo:b1]
        if tree:
            made = np.concatenate([made, tree["row_token"][tree["chain"][i][tree["chain"][i] >= 0]]])
        row = z[i]
        seen, times = np.unique(made, return_counts=True)
        every = torch.from_numpy(np.unique(np.concatenate([h["history"][b0:bo], made])).astype(np.int64)).to(DEV)
        row = row.clone()
        r = float(h["repetition"][s])
        row[every] = torch.where(row[every] > 0, row[every] / r, row[every] * r)
        at = torch.from_numpy(seen.astype(np.int64)).to(DEV)
        row[at] -= float(h["frequency"][s]) * torch.from_numpy(times.astype(np.float64)).to(DEV) + float(h["presence"][s])
        last = dict(zip(h["bias_token"][int(h["bias_begin"][s]):int(h["bias_begin"][s + 1])].tolist(),
                        h["bias_value"][int(h["bias_begin"][s]):int(h["bias_begin"][s + 1])].astype(np.float64).tolist()))
        if last:
            row[torch.tensor(list(last), device=DEV)] += torch.tensor(list(last.values()), dtype=torch.float64, device=DEV)
        m = int(h["mask_row"][i])
        if m >= 0:
            bits = np.unpackbits(np.ascontiguousarray(h["mask"][m]).view(np.uint8), bitorder="little")[:V]
            row[torch.from_numpy(bits == 0).to(DEV)] = -math.inf
        top = float(row.max())
        logprob[i] = top - float(torch.logsumexp(row, 0)) if top > -math.inf else -math.inf
        if whole is not None:
            whole[i] = row
    out = {"next": None, "logprob": torch.from_numpy(logprob)}
    if whole is not None:
        out["logits"] = whole
    return out
