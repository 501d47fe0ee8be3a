"""The generated code of the operators on drafted tokens, where correctness or speed hangs on it: the attention's LDS reads are assembly whose
waits the kernel places itself, its copy queue must not be drained pair by pair, and the picks' and the moved rows' loads must be sent together."""
import os
import re
import subprocess
import tempfile

import pytest

from paper_2507_17769_amd import build as B
from test_kernel_isa import _touched_before_their_wait


def _compile(source):
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, "kernel.s")
        flags = [f for f in B.FLAGS if f != "-fPIC"]
        r = subprocess.run([B.HIPCC] + flags + ["--cuda-device-only", "-S", os.path.join(B.CSRC, source), "-o", out], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        return open(out).read()


@pytest.fixture(scope="module")
def tree_asm():
    return _compile("tree_attention.hip")


def _bodies(asm, kernel):
    for m in re.finditer(r"^(_ZN2ps\d+" + kernel + r"I\w+):\s*;.*?\n(.*?)s_endpgm", asm, re.S | re.M):
        yield m.group(1), [l.strip() for l in m.group(2).splitlines() if l.strip() and not l.strip().startswith(";")]


def _loops(lines):
    labels = {mm.group(1): i for i, l in enumerate(lines) for mm in [re.match(r"(\.LBB\d+_\d+):", l)] if mm}
    for i, l in enumerate(lines):
        mm = re.match(r"s_c?branch\w* (\.LBB\d+_\d+)$", l)
        if mm and mm.group(1) in labels and labels[mm.group(1)] < i:
            yield lines[labels[mm.group(1)]:i + 1]


def _resources(asm, kernel):
    for m in re.finditer(r"^\s*\.amdhsa_kernel (_ZN2ps\d+" + kernel + r"\S*)(.*?)\.end_amdhsa_kernel", asm, re.S | re.M):
        get = lambda key: int(re.search(key + r" (\d+)", m.group(2)).group(1))
        yield m.group(1), get(r"next_free_vgpr"), get(r"group_segment_fixed_size"), get(r"private_segment_fixed_size")


def test_tree_attention_keeps_two_blocks_per_compute_unit(tree_asm):
    """The plan deals its work to two blocks per compute unit where it is short of items: both must be resident."""
    found = list(_resources(tree_asm, "tree_kernel"))
    assert len(found) == 20                       # head dims 64 and 128 x group sizes 1 to 16 x one or more readers of a page
    for name, vgprs, lds, _ in found:
        assert vgprs <= 256 and lds <= 80 * 1024, (name, vgprs, lds)


def test_tree_attention_loops_over_a_prefix_do_not_drain_or_spill(tree_asm):
    n = 0
    for name, lines in _bodies(tree_asm, "tree_kernel"):
        team = [b for b in _loops(lines) if b.count("s_barrier") == 1 and sum(x.startswith("global_load_lds") for x in b) in (2, 4)
                and any(x.startswith("v_mfma") for x in b)]
        by_tiles = {}
        for b in team:                            # the shorter loop of a number of tiles is the one without masks
            k = sum(x.startswith("v_mfma") for x in b)
            by_tiles[k] = min(by_tiles.get(k, b), b, key=len)
        assert len(by_tiles) >= 3, (name, sorted(by_tiles))
        for k, b in by_tiles.items():
            assert not any(x.startswith("scratch_") for x in b), (name, k)
            # the only full wait is that of the rare refill of page numbers
            assert sum(x.startswith("s_waitcnt") and "vmcnt(0)" in x for x in b) <= 1, (name, k)
        n += 1
    assert n == 20


def test_tree_attention_uses_no_register_that_an_lds_read_still_writes(tree_asm):
    n = 0
    for name, lines in _bodies(tree_asm, "tree_kernel"):
        bad = _touched_before_their_wait(lines)
        assert not bad, (name, bad[:3])
        n += 1
    assert n == 20


def _longest_run_of_loads(lines, op):
    """Loads that are sent with no wait for memory between them."""
    best = run = 0
    for l in lines:
        if re.match(r"s_waitcnt.*vmcnt", l):
            run = 0
        elif l.startswith(op):
            run += 1
            best = max(best, run)
    return best


def test_picks_send_the_tokens_of_a_list_together():
    asm = _compile("pick.hip")
    found = list(_resources(asm, "pick_kernel"))
    assert len(found) == 12                       # two types x one, two or four quads a thread x whole quads or not
    for name, vgprs, _, scratch in found:
        assert scratch == 0 and vgprs <= 256, (name, vgprs, scratch)
        if name.split("pick_kernelI")[1].startswith(("Lb0ELi4ELb1E", "Lb1ELi4ELb1E")):
            assert vgprs <= 128, (name, vgprs)    # four blocks share a compute unit
    for name, lines in _bodies(asm, "pick_kernel"):
        assert _longest_run_of_loads(lines, "global_load_dword") >= 8, name


def test_kept_rows_and_heads_do_not_spill():
    for source, kernel, n in (("tree_keep.hip", "tree_keep_kernel", 2), ("qk_norm.hip", "qk_norm_rope_kernel", 4)):
        found = list(_resources(_compile(source), kernel))
        assert len(found) == n
        for name, vgprs, _, scratch in found:
            assert scratch == 0 and vgprs <= 128, (name, vgprs, scratch)
