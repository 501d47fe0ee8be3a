"""What Engine makes of the tensors of a call on drafted tokens, on the CPU: the pointers, counts and strides that the library gets, and what is refused
because the library would read past a tensor.  No call reaches a device here."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2507_17769_amd import binding as B
from paper_2507_17769_amd import workloads as W
from paper_2507_17769_amd.runner import Engine

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def engine():
    """An Engine as far as its checks of arguments go."""
    e = Engine.__new__(Engine)
    e.model, e.device = dict(W.MODELS["tiny"]), torch.device("cpu")
    return e


def words_read(r, n_rows, vocab, mask):
    """The last word that picks of any row may read, counted from the start of the mask's storage."""
    assert r.mask == mask.data_ptr()
    return mask.storage_offset() + (r.n_masks - 1) * r.mask_stride + (vocab + 31) // 32


@pytest.mark.parametrize("vocab", [1, 31, 32, 33, 1000])
def test_masks_are_read_within_their_tensor(vocab):
    e, words = engine(), (vocab + 31) // 32
    wide = torch.zeros(7, words + 3, dtype=torch.int32)
    for mask in (torch.zeros(5, words, dtype=torch.int32), wide, wide[:, :words], wide[1:6:2], wide[6:, 3:], wide[:1], torch.zeros(1, words, dtype=torch.int32)):
        n = mask.shape[0]
        r = e._rules({"mask": mask}, n, vocab)
        assert r.n_masks == n and words_read(r, n, vocab, mask) <= mask.untyped_storage().nbytes() // 4
        for i in range(n):
            assert r.mask + 4 * i * r.mask_stride == mask[i].data_ptr() or n == 1
    one = torch.zeros(1, words, dtype=torch.int32)
    bad = [one.expand(6, words), torch.zeros(8 * words, dtype=torch.int32).as_strided((6, words), (0, 1))]
    if words > 1:
        bad += [torch.zeros(6 + words, dtype=torch.int32).as_strided((6, words), (1, 1)), torch.zeros(6, words - 1, dtype=torch.int32),
                torch.zeros(6, words + 9, dtype=torch.int32)[:, :words - 1], torch.zeros(1, words - 1, dtype=torch.int32)]
    for mask in bad:
        with pytest.raises(ValueError):
            e._rules({"mask": mask, "mask_row": torch.zeros(6, dtype=torch.int32)}, 6, vocab)


def test_a_mask_of_no_rows_allows_nothing_where_a_row_asks_for_one():
    """mask_row at or above the number of masks: nothing is allowed, also where that number is 0; a mask_row without masks is the library's to refuse."""
    e = engine()
    none, row = torch.zeros(0, 4, dtype=torch.int32), torch.tensor([-1, 0, 2], dtype=torch.int32)
    r = e._rules({"mask": none, "mask_row": row}, 3, 100)
    assert r.mask and r.n_masks == 0 and r.mask_row == row.data_ptr() and r.mask_stride >= 4
    with pytest.raises(ValueError):
        e._rules({"mask": none}, 3, 100)
    e._rules({"mask": none}, 0, 100)
    r = e._rules({"mask_row": row}, 3, 100)
    assert r.mask_row == row.data_ptr() and not r.mask
    r = e._rules({"mask": None, "mask_row": None}, 3, 100)
    assert not r.mask and not r.mask_row and r.n_masks == 0


def test_the_stride_of_a_single_row_does_not_matter():
    e = engine()
    wide = torch.zeros(3, 67, dtype=torch.bfloat16)
    assert e._rows(wide[:, :64], 3, 64, "x") == (wide.data_ptr(), 67)
    assert e._rows(wide[1:2, :64], 1, 64, "x") == (wide[1].data_ptr(), 64)      # 67 elements are no multiple of 16 bytes, and no row follows
    assert e._rows(wide[:1, :64].view(1, 4, 16), 1, 64, "x") == (wide.data_ptr(), 64)
    assert e._rows(torch.zeros(1, 64).expand(1, 64), 1, 64, "x")[1] == 64


def test_trees_that_outlive_the_binding_end_without_a_word():
    """A script's objects that one of its functions refers to are collected after the module whose functions free them."""
    code = ("from paper_2507_17769_amd import binding as B\n"
            "c = B.Context(256, 4, 2, 64, 256, host_only=True)\n"
            "t = B.Tree(c).plan([(1, 1, 1, [0])])\n"
            "f = lambda i: (c, t)\n")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT, timeout=120)
    assert r.returncode == 0 and "Exception" not in r.stderr, r.stderr
