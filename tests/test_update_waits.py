"""A block of the update that gave up a wait does not tell the others that its part of a phase is done: what
they read would be neither right nor NaN.  They run out of time as well, and all that is not right is NaN.  On the
host, one pair of blocks."""
import os
import shutil

import pytest

from test_product_chains import MODEL, build, chains

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no C++ compiler")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    """The program of the update's tests, which then also asks how many blocks have arrived."""
    with open(os.path.join(MODEL, "orthogonalize.cpp")) as f:
        main = f.read()
    more = """
    const uint32_t arrived = *(const uint32_t*)(ws.p + ortho_plan(batch, rows, cols).arrived);
    const uint32_t whole = steps ? 2 * (3 * steps - 1) : 0;      // both blocks, at the end of every phase but the last
    if (injected ? arrived >= whole : arrived != whole) {
        printf("%u of %u arrivals\\n", arrived, whole);
        return 1;
    }
"""
    at = main.index("    const size_t n = std::min(rows, cols)")
    return build(tmp_path_factory.mktemp("waits"), main[:at] + more + main[at:], dict(kProductPairs=1), "orthogonalize")


@pytest.mark.parametrize("args", [(2, 40, 24, "bf16", "f16", "any", 2), (3, 33, 70, "f32", "bf16", "any", 0)], ids=["two", "none"])
def test_every_block_arrives_after_every_phase(program, args):
    chains(program, *args, 1)


@pytest.mark.parametrize("rank", [0, 1])
@pytest.mark.parametrize("nth", [0, 3, 7])
def test_a_block_that_gave_up_does_not_arrive(program, rank, nth):
    chains(program, 1, 200, 300, "f32", "f32", "whole", 2, 1, "drop_rank=%d" % rank, "drop_nth=%d" % nth)
