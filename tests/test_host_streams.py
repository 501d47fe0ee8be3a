"""Where the library's device work is enqueued: on a context's stream.  Work on the default stream is not ordered before that of a stream which does not
block with it, so memory that a kernel expects to be cleared may not be cleared there."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_memory_is_cleared_on_a_contexts_stream():
    sources = sorted(glob.glob(os.path.join(ROOT, "paper_2507_17769_amd", "csrc", "*.hip")))
    assert len(sources) >= 8
    for path in sources:
        code = re.sub(r"//[^\n]*", "", open(path).read())
        assert not re.search(r"\bhipMemset(D(8|16|32))?\(", code), path       # of the default stream
        for call in re.findall(r"\bhipMemset\w*Async\(([^;]*);", code):
            assert "stream" in call, (path, call)
