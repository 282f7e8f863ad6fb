"""The ends of what the calls for a language model's step accept: sizes of 0, the largest ones, and what the
workspaces' helpers say of them.  Nothing here needs a GPU."""
import subprocess
import sys

import paper_1905_10988_b200 as nc
from operator_util import address, status


def test_helpers_answer_for_sizes_of_zero():
    # in a process of its own: a helper that ends it (a division by zero did) shows as a failure
    text = """
import itertools
import paper_1905_10988_b200 as nc
for s in itertools.product((0, 1, 700), repeat=3):
    for f in (nc.nc_embedding_backward_workspace_bytes, nc.nc_linear_cross_entropy_forward_workspace_bytes,
              nc.nc_linear_cross_entropy_backward_workspace_bytes, nc.nc_orthogonalize_workspace_bytes):
        assert f(*s) > 0, (f.__name__, s)
"""
    got = subprocess.run([sys.executable, "-c", text], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0, (got.returncode, got.stderr[-2000:])


def test_the_embeddings_helper_refuses_what_the_call_refuses():
    keep, A = address()

    def call(rows, vocabulary, cols):
        return status(lambda: nc.nc_embedding_backward(A, 8, rows, A, nc.DTYPE_F32, cols, cols, 1.0, vocabulary, A,
                                                       nc.DTYPE_F32, cols, False, A, 0, stream=0))

    most = 256 * 65535                    # blocks of 256 columns that a grid has in its second dimension
    for rows, vocabulary, cols in ((4, 9, most), (4, 9, 1 << 24), (4, 9, (1 << 31) - 1), (1 << 31, 9, 8), (4, 1 << 31, 8)):
        assert nc.nc_embedding_backward_workspace_bytes(rows, vocabulary, cols) == 0, (rows, vocabulary, cols)
        assert call(rows, vocabulary, cols) == "NC_ERR_TOO_LARGE", (rows, vocabulary, cols)
    for rows, vocabulary, cols in ((4, 9, most - 1), ((1 << 31) - 1, 9, 8), (4, (1 << 31) - 1, 8)):
        assert nc.nc_embedding_backward_workspace_bytes(rows, vocabulary, cols) > 0, (rows, vocabulary, cols)
        assert call(rows, vocabulary, cols) == "NC_ERR_WORKSPACE", (rows, vocabulary, cols)
