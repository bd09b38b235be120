"""A block whose waits run out ends with no copy of its own in flight: it would land in shared memory that the block has put to other
use, or that belongs to the next one.  Read off the sources, since no run makes a copy hang."""
import re

import pytest

from test_kernel_sources import _closed, _code, _function


def _producer(kernel, role):
    """The code of the warp that issues the copies: the block behind `if (role)`."""
    _, body = _function(_code(), kernel)
    at = body.index("if (" + role + ")")
    start = body.index("{", at)
    return body[start:_closed(body, start, "{}")]


@pytest.mark.parametrize("kernel,role,rings", [("atf_tree_tiles", "warp == TR_WARPS", [("it", "full_bar(i % ST)", "ST")]),
                                               ("atf_tree_wide", "warp == TW_PRODUCER", [("kissued", "bar(KFULL, t % ST)", "ST"), ("vissued", "bar(VFULL, t % ST)", "ST")])])
def test_what_was_issued_is_waited_for(kernel, role, rings):
    code = _producer(kernel, role)
    last_break, last_copy = code.rindex("break;"), max(code.rindex("bulk_load_1d("), code.rindex("tma_load_3d("))
    for count, barrier, stages in rings:
        m = re.search(r"for \(int (\w) = max\(0, " + count + r" - " + stages + r"\); \1 < " + count + r"; \+\+\1\)\s*if \(!mbar_wait\(" +
                      re.escape(barrier) + r", \(\1 / " + stages + r"\) & 1\)\)", code)
        assert m, "the producer leaves copies in flight"
        assert m.start() > last_break and m.start() > last_copy


@pytest.mark.parametrize("stages", [2, 3, 4])
def test_the_last_use_of_every_stage(stages):
    """Of any number of copies issued, the waits name the last one of each stage, with its parity; a stage is issued again only when its
    copy before has arrived, so no earlier one can be in flight."""
    for issued in range(3 * stages + 2):
        waited = {i % stages: (i // stages) & 1 for i in range(max(0, issued - stages), issued)}
        last = {}
        for i in range(issued):
            last[i % stages] = (i // stages) & 1
        assert waited == last
