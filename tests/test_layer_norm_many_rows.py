"""Layer norm with at least three rows for every owner of rows, in each of its kernels: the row ahead,
the two sets of slots in turn and the warps' scratch memory are used again from row to row.  Which kernel
a shape takes and how many rows an owner gets is worked out below and asserted without a GPU."""
import pytest

from test_layer_norm import layout, test_gpu_backward, test_gpu_forward

SMS, THREADS = 148, 256
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def deal(cols):
    """blocks of a row, threads of a group, groups of a block"""
    cluster = 1
    while cols > 16 * THREADS * cluster:
        cluster *= 2
    G = -(-(-(-cols // cluster)) // 512) * 32
    return cluster, G, THREADS // G if cluster == 1 else 1


def mode(kind, where, cols):
    ld, off = layout(where, cols, SIZE[kind])
    together = (ld * SIZE[kind]) | (off * SIZE[kind])
    cluster, G, _ = deal(cols)
    if together % 16:
        return "spread"
    whole = together % 32 == 0 and cluster <= 2 and cols == 16 * G * cluster
    return "regular" if whole else "vector"


def rows_of_an_owner(kind, where, rows, cols, backward):
    """(kernel, rows that the owners have on average)"""
    cluster, G, groups = deal(cols)
    m = mode(kind, where, cols)
    threads = 512
    if not backward:
        if m == "regular" and cols % 1024 == 0 and rows >= 512:
            G = cols // 32
            block = THREADS if kind == "f32" else 128
            cluster, groups, m = 1, max(1, block // G), "regular of 32 values"
        else:
            threads = THREADS * (3 if kind == "f32" and m != "regular" else 4)
    blocks = SMS * max(1, threads // (G * groups)) // cluster
    if backward:
        blocks = min(blocks, 592)
    owners = -(-rows // groups)
    return (m, cluster), owners / min(blocks, owners)


CASES = [("bf16", "whole", 9000, 768), ("f32", "whole", 9000, 768), ("bf16", "gap16", 4000, 2000),
         ("f16", "any", 8000, 1001), ("f32", "any", 6000, 1001), ("bf16", "whole", 2000, 5000),
         ("f32", "gap16", 1500, 5000), ("bf16", "any", 2000, 5001), ("bf16", "whole", 15000, 512),
         ("f32", "whole", 15000, 512), ("bf16", "whole", 511, 8192), ("f16", "gap16", 600, 12000),
         ("bf16", "any", 600, 12001), ("bf16", "gap16", 400, 20000), ("f32", "any", 400, 20001),
         ("bf16", "whole", 2500, 4096), ("f32", "whole", 1200, 8192)]


def test_cases_give_their_kernels_several_rows_an_owner():
    seen = {False: {}, True: {}}
    for kind, where, rows, cols in CASES:
        for backward in (False, True):
            kernel, many = rows_of_an_owner(kind, where, rows, cols, backward)
            seen[backward][kernel] = max(many, seen[backward].get(kernel, 0))
            # (rows of two blocks that fill every thread come here with fewer than 512 rows only)
            least = 1.7 if kernel == ("regular", 2) and not backward else 3
            assert many >= least, (kind, where, rows, cols, backward, many)
    every = {(m, c) for m in ("vector", "spread") for c in (1, 2, 4, 8)} | {("regular", 1), ("regular", 2)}
    assert set(seen[False]) == every | {("regular of 32 values", 1)}
    assert set(seen[True]) == every


@pytest.mark.gpu
@pytest.mark.parametrize("kind,where,rows,cols", CASES)
def test_gpu_forward_several_rows_an_owner(kind, where, rows, cols):
    test_gpu_forward(kind, kind, where, rows, cols)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,where,rows,cols", CASES)
@pytest.mark.parametrize("saved8", [False, True])
def test_gpu_backward_several_rows_an_owner(kind, where, rows, cols, saved8):
    test_gpu_backward(kind, kind, where, rows, cols, saved8)
