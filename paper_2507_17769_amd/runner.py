"""Convenience wrapper used by the tests, the smoke entry and the benchmark: owns a library
context plus the torch tensors (device memory only) that feed it.  All computation happens in
libpolystep; torch allocates buffers and moves bytes."""
import ctypes as C

import numpy as np
import torch

from . import binding as B
from . import workloads as W


def bits_to_dev(bits, device):
    """uint16 bf16 bit patterns (numpy) -> int16 device tensor holding the same bits."""
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(device)


def dev_to_bits(t):
    return t.detach().cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


class _PoolMemory:
    """The KV pool as torch sees foreign device memory; keeps the context that owns it alive."""

    def __init__(self, ctx):
        self.ctx = ctx
        address, n_bytes = ctx.kv_pool()
        self.__cuda_array_interface__ = {"shape": (n_bytes // 2,), "typestr": "<i2", "data": (address, False), "version": 3}


_DTYPE_CODES = {torch.float32: B.PS_F32, torch.bfloat16: B.PS_BF16}


def _dtype_code(t):
    if t.dtype not in _DTYPE_CODES:
        raise TypeError(f"expected a float32 or bfloat16 tensor, not {t.dtype}")
    return _DTYPE_CODES[t.dtype]


# The tensors of ps_logit_rules: those with an entry per list, those of offsets (one more), those with an entry per row.
_RULE_TYPES = {n: torch.float32 if n in ("repetition", "frequency", "presence", "bias_value") else torch.int32
               for n, t in B.ps_logit_rules._fields_ if t is C.c_void_p}
_RULE_LISTS = ("repetition", "frequency", "presence", "output_begin", "history_begin", "bias_begin")
_RULE_BEGINS = ("history_begin", "bias_begin")
_RULE_ROWS = ("mask_row", "row_list", "row_token", "row_prev")


class Engine:
    """Work runs on the stream that is current when the engine is made.  A caller on another stream orders the two (wait_stream); the memory of tensors
    that it hands over, and of results, is not handed out again before both streams are done with it."""

    def __init__(self, model, n_pool_pages, n_layers=1, n_kv_layers=1, max_position=None, perm_seed=0, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("Engine needs a GPU: there is no CPU fallback")
        self.model = dict(W.MODELS[model]) if isinstance(model, str) else dict(model)
        m = self.model
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.stream = torch.cuda.current_stream(self.device)
        self._stream_id = self.stream.cuda_stream, self.stream.device.index
        self.n_layers = n_layers
        if max_position is None:
            max_position = 16 * n_pool_pages
        self.ctx = B.Context(m["hidden"], m["n_q"], m["n_kv"], m["head_dim"], m["ffn"], n_layers, max_position,
                             W.RMS_EPS, m["rope_base"], stream=self.stream.cuda_stream)
        self.ctx.kv_alloc(n_pool_pages, n_kv_layers, perm_seed)
        self.n_pool_pages = n_pool_pages

    def close(self):
        self.ctx.destroy()

    def _elsewhere(self):
        """The current stream where it is not the engine's, else None."""
        handle, index = self._stream_id
        if torch._C._cuda_getCurrentRawStream(index) == handle:   # a number: a Stream object each time would cost a call as much as its checks
            return None
        return torch.cuda.current_stream(self.device)

    def _lend(self, other, *tensors):
        """Tensors of the caller's, checked, are about to be used by the engine's stream."""
        if other is not None:
            for t in tensors:
                if t is not None:
                    t.record_stream(self.stream)

    def _empty(self, other, shape, dtype):
        """A result's memory, the engine's stream's; `other`: what _elsewhere has said."""
        if other is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(self.stream):
            t = torch.empty(shape, dtype=dtype, device=self.device)
        t.record_stream(other)
        return t

    def load_layer(self, layer, weights_bits):
        dev = {k: bits_to_dev(v, self.device) for k, v in weights_bits.items()}
        self.ctx.init_layer(layer, **{k: t.data_ptr() for k, t in dev.items()})
        self.ctx.sync()

    def load_head(self, head_bits):
        """head_bits: {"embedding" [vocab][hidden], "g_final" [hidden], "w_out" [hidden][vocab]} as bf16 bit patterns."""
        dev = {k: bits_to_dev(v, self.device) for k, v in head_bits.items()}
        self.vocab = int(head_bits["embedding"].shape[0])
        self.ctx.init_head(dev["embedding"].data_ptr(), dev["g_final"].data_ptr(), dev["w_out"].data_ptr(), self.vocab)
        self.ctx.sync()

    def step_tokens(self, seqs, token_ids, want_logits=True, want_hidden=False, want_stats=False, want_parts=False):
        """Full-model step.  Returns dict with "next" (int32 tensor [n_seqs]), optionally "logits" (fp32
        [n_seqs][vocab]) and "hidden" (fp32 [T][hidden]), "stats", "parts_ms"."""
        n, T, other = len(seqs), sum(int(s.n_new) for s in seqs), self._elsewhere()
        out = {"next": self._empty(other, n, torch.int32)}
        if want_logits:
            out["logits"] = self._empty(other, (n, self.vocab), torch.float32)
        if want_hidden:
            out["hidden"] = self._empty(other, (T, self.model["hidden"]), torch.float32)
        out["stats"], out["parts_ms"] = self.ctx.step_tokens(
            seqs, token_ids, out["next"].data_ptr(), out["logits"].data_ptr() if want_logits else None,
            out["hidden"].data_ptr() if want_hidden else None, want_stats, want_parts)
        return out

    def write_kv(self, layer, pages, pos0, k_bits, v_bits):
        n = k_bits.shape[0]
        if n == 0:
            return
        k, v = bits_to_dev(k_bits, self.device), bits_to_dev(v_bits, self.device)
        self.ctx.kv_write(layer, pages, pos0, n, k.data_ptr(), v.data_ptr())
        self.ctx.sync()

    def read_kv(self, layer, pages, pos0, n):
        m = self.model
        k = torch.empty((n, m["n_kv"], m["head_dim"]), dtype=torch.int16, device=self.device)
        v = torch.empty_like(k)
        self.ctx.kv_read(layer, pages, pos0, n, k.data_ptr(), v.data_ptr())
        self.ctx.sync()
        return dev_to_bits(k), dev_to_bits(v)

    def load_prefixes(self, batch, layer=0, slot_tag=0):
        for i, s in enumerate(batch.seqs):
            if s.prefix > 0:
                k, v = batch.prefix_kv(i, slot_tag)
                self.write_kv(layer, s.pages, 0, k, v)

    def alloc_taps(self, T):
        m = self.model
        i16 = dict(dtype=torch.int16, device=self.device)
        return {
            "xn": torch.zeros((T, m["hidden"]), **i16),
            "q": torch.zeros((T, m["n_q"], m["head_dim"]), **i16),
            "attn": torch.zeros((T, m["n_q"] * m["head_dim"]), **i16),
            "x1": torch.zeros((T, m["hidden"]), dtype=torch.float32, device=self.device),
            "xn2": torch.zeros((T, m["hidden"]), **i16),
            "act": torch.zeros((T, m["ffn"]), **i16),
            "x_in": torch.zeros((T, m["hidden"]), dtype=torch.float32, device=self.device),
            "x_out": torch.zeros((T, m["hidden"]), dtype=torch.float32, device=self.device),
        }

    def step(self, seqs, x_dev, out_dev=None, want_stats=False):
        """x_dev: int16 device tensor [T][hidden] of bf16 bits.  Returns (out_dev, stats)."""
        other = self._elsewhere()
        self._lend(other, x_dev, out_dev)
        if out_dev is None:
            out_dev = self._empty(other, x_dev.shape, x_dev.dtype)
        stats = self.ctx.step(seqs, x_dev.data_ptr(), out_dev.data_ptr(), want_stats)
        return out_dev, stats

    # ---- drafted tokens -------------------------------------------------------------------------------------------
    def _rows(self, t, n_rows, width, name, dtypes=(torch.float32, torch.bfloat16)):
        """Address and row stride of a device tensor whose leading dimension is rows of `width` adjacent elements."""
        if t.device != self.device:
            raise ValueError(f"{name} is on {t.device}, the engine on {self.device}")
        if t.dtype not in dtypes:
            raise TypeError(f"{name} has type {t.dtype}")
        shape, stride = t.shape, t.stride()
        n, adjacent = 1, True
        for size, step in zip(shape[:0:-1], stride[:0:-1]):
            adjacent = adjacent and (size == 1 or step == n)
            n *= size
        if len(shape) < 2 or shape[0] != n_rows or (n_rows and n != width):
            raise ValueError(f"{name} must hold {n_rows} rows of {width}, not {tuple(shape)}")
        if n_rows and not adjacent:
            raise ValueError(f"the elements of a row of {name} must be adjacent")
        return t.data_ptr(), (stride[0] if n_rows > 1 else width)

    def kv_pool(self):
        """The KV pool as a bf16 tensor [KV slot][page][kv head][K, V][16 * head_dim] (a view: see ps_kv_pool for the order of a
        page's elements).  It keeps the context alive; ctx.kv_alloc or close() end it."""
        m = self.model
        flat = torch.as_tensor(_PoolMemory(self.ctx), device=self.device).view(torch.bfloat16)
        return flat.view(-1, self.n_pool_pages, m["n_kv"], 2, 16 * m["head_dim"])

    def tree(self, seqs, parents=None):
        """A planned batch of token trees; .plan(seqs, parents) plans it anew."""
        return B.Tree(self.ctx).plan(seqs, parents)

    def load_qk_norm(self, layer, g_q, g_k):
        """Gains [head_dim] (device bf16 tensors) of a layer that normalises its query and key heads; None, None: it does not."""
        d = self.model["head_dim"]
        if g_q is None and g_k is None:
            self.ctx.init_qk_norm(layer, None, None)
            return
        gains = [g.to(device=self.device, dtype=torch.bfloat16).contiguous() for g in (g_q, g_k)]
        if any(g.shape != (d,) for g in gains):
            raise ValueError(f"gains must hold {d} elements")
        other = self._elsewhere()
        if other is not None:
            self.stream.wait_stream(other)   # what the gains come from
        self.ctx.init_qk_norm(layer, gains[0].data_ptr(), gains[1].data_ptr())
        self.ctx.sync()

    def qk_norm_rope(self, layer, tree, qkv, q=None):
        """qkv: [T][(n_q + 2 n_kv) * head_dim] fp32 or bf16, rows anywhere on 16 bytes.  Appends keys and values; returns bf16 [T][n_q][head_dim]."""
        m = self.model
        p, ld = self._rows(qkv, tree.n_tokens, (m["n_q"] + 2 * m["n_kv"]) * m["head_dim"], "qkv")
        other = self._elsewhere()
        if q is None:
            q = self._empty(other, (tree.n_tokens, m["n_q"], m["head_dim"]), torch.bfloat16)
        elif q.shape != (tree.n_tokens, m["n_q"], m["head_dim"]) or q.dtype != torch.bfloat16 or not q.is_contiguous() or q.device != self.device:
            raise ValueError("q must be a contiguous bf16 [T][n_q][head_dim] tensor of the engine's device")
        self._lend(other, qkv, q)
        self.ctx.qk_norm_rope(layer, tree, p, _dtype_code(qkv), ld, q.data_ptr())
        return q

    def tree_attention(self, layer, tree, q, out=None):
        """q: bf16 [T][n_q][head_dim], rows anywhere on 16 bytes; returns the same shape."""
        m = self.model
        width = m["n_q"] * m["head_dim"]
        pq, ldq = self._rows(q, tree.n_tokens, width, "q", (torch.bfloat16,))
        other = self._elsewhere()
        if out is None:
            out = self._empty(other, (tree.n_tokens, m["n_q"], m["head_dim"]), torch.bfloat16)
        po, ldo = self._rows(out, tree.n_tokens, width, "out", (torch.bfloat16,))
        self._lend(other, q, out)
        self.ctx.tree_attention(layer, tree, pq, ldq, po, ldo)
        return out

    def tree_keep(self, tree, kept):
        """kept: for each sequence the nodes whose cache rows become the prefix's next positions, ascending."""
        self.ctx.tree_keep(tree, kept)

    def _rules(self, rules, n_rows, vocab=0):
        """rules: dict of device tensors with the names of ps_logit_rules ("mask" int32 [n_masks][words], whole words for `vocab` tokens)."""
        r, device, size = B.ps_logit_rules(), self.device, {}
        for name, t in rules.items():
            dtype = _RULE_TYPES.get(name)
            if dtype is None:
                raise ValueError(f"unknown rule {name}")
            if t is None:
                continue
            if t.dtype != dtype or t.device != device:
                raise TypeError(f"{name} must be a {str(dtype)[6:]} tensor of the engine's device")
            n = t.numel()
            if name != "mask":
                if t.dim() != 1 or not t.is_contiguous():
                    raise ValueError(f"{name} must be one contiguous row")
                size[name] = n
            elif t.dim() != 2 or (n and t.stride(1) != 1):
                raise ValueError("mask must hold rows of adjacent words")
            if n:
                setattr(r, name, t.data_ptr())
        lists = {k: size[k] - (k in _RULE_BEGINS) for k in _RULE_LISTS if k in size}
        if len(set(lists.values())) > 1:
            raise ValueError(f"the rules disagree about the number of lists: {lists}")
        r.n_lists = next(iter(lists.values()), 0)
        r.n_history = size.get("history", 0)
        r.n_biases = size.get("bias_token", 0)
        if r.n_history == 0:
            r.history = r.output_begin = None
        if "bias_token" in size and size.get("bias_value") != size["bias_token"]:
            raise ValueError("bias_value must hold one value per bias_token")
        for name in _RULE_ROWS:
            if size.get(name, n_rows) != n_rows:
                raise ValueError(f"{name} must hold one entry per row")
        mask = rules.get("mask")
        if mask is not None:
            r.n_masks, words = mask.shape
            if words < (vocab + 31) // 32:
                raise ValueError(f"mask holds {words} words a row, {vocab} tokens take {(vocab + 31) // 32}")
            if r.n_masks > 1 and mask.stride(0) < words:
                raise ValueError("the rows of mask overlap (mask_row gives several rows of logits one mask)")
            if r.n_masks == 0 and not r.mask_row and n_rows:
                raise ValueError("mask holds no rows, and no mask_row says which rows of logits have none")
            r.mask = r.mask or r.mask_row      # of no rows: never read, but a mask_row of 0 or above has to find that it is not there
            r.mask_stride = mask.stride(0) if r.n_masks > 1 else words
        return r

    def pick_tokens(self, logits, rules=None, want_logits=False):
        """logits: [rows][vocab] fp32 or bf16, any row stride.  Returns {"next": int32 [rows], "logprob": fp32 [rows]} and, if wanted,
        "logits": the changed ones, fp32 [rows][vocab]."""
        if logits.dim() != 2:
            raise ValueError("logits must be [rows][vocab]")
        n, vocab = logits.shape
        p, ld = self._rows(logits, n, vocab, "logits")
        r, other = None if rules is None else self._rules(rules, n, vocab), self._elsewhere()
        self._lend(other, logits, *(rules or {}).values())
        out = {"next": self._empty(other, n, torch.int32), "logprob": self._empty(other, n, torch.float32)}
        if want_logits:
            out["logits"] = self._empty(other, (n, vocab), torch.float32)
        self.ctx.pick_tokens(p, _dtype_code(logits), ld, n, vocab, r,
                             out["logits"].data_ptr() if want_logits else None, vocab, out["next"].data_ptr(), out["logprob"].data_ptr())
        return out

    def verify_tokens(self, tree, token_ids, rules=None, want_logits=False, want_hidden=False):
        """Full-model step over a batch of trees: token_ids host [T].  Returns {"next", "logprob"} for every node, optionally "logits"
        (changed by the rules) and "hidden"."""
        T, other = tree.n_tokens, self._elsewhere()
        r = None if rules is None else self._rules(rules, T, getattr(self, "vocab", 0))
        self._lend(other, *(rules or {}).values())
        out = {"next": self._empty(other, T, torch.int32), "logprob": self._empty(other, T, torch.float32)}
        if want_logits:
            out["logits"] = self._empty(other, (T, self.vocab), torch.float32)
        if want_hidden:
            out["hidden"] = self._empty(other, (T, self.model["hidden"]), torch.float32)
        self.ctx.verify_tokens(tree, token_ids, r, out["next"].data_ptr(), out["logprob"].data_ptr(),
                               out["logits"].data_ptr() if want_logits else None, out["hidden"].data_ptr() if want_hidden else None)
        return out
