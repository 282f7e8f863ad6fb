"""The kernels of the 8-bit checkpoints, the layer norm and the weight gradient thread by thread on the
host (tests/device_model): their schedules on a small chip, the bounds of every access, and waits that
run out of time.  The values are
compared with a product in 64 bits; the address sanitizer checks global and shared memory; copies and
matrix instructions take effect late and in changing order; a wait that nothing ends, a barrier that
gets too many arrivals or a copy in flight at a block's end is an error."""
import concurrent.futures
import os
import random
import re
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
MODEL = os.path.join(HERE, "device_model")
sys.path.insert(0, MODEL)

import translate  # noqa: E402

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no C++ compiler")


def build(folder, name, constants=None, change=None, define=""):
    source, program = str(folder / (name + ".cpp")), str(folder / name)
    with open(os.path.join(MODEL, name + ".cpp")) as f:
        main = f.read()
    with open(source, "w") as f:
        f.write(translate.translate([name + "_kernels.cu"], constants, change) + define + main)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.run(["g++", "-std=c++20", "-O1", "-g1", "-w", "-ffp-contract=off", "-fsanitize=address",
                    "-I" + MODEL, "-I" + os.path.join(translate.ROOT, "include"),
                    "-I" + os.path.join(cuda, "include"), "-o", program, source], check=True)
    return program


def run(program, *args):
    got = subprocess.run([program] + [str(a) for a in args], capture_output=True, text=True,
                         timeout=300)
    assert got.returncode == 0 and got.stdout.startswith("ok"), got.stdout + got.stderr[-2000:]
    return got.stdout


@pytest.fixture(scope="module")
def weight_grad(tmp_path_factory):
    return build(tmp_path_factory.mktemp("model"), "weight_grad", dict(kWgPairs=2))


@pytest.fixture(scope="module")
def short_chains(tmp_path_factory):
    return build(tmp_path_factory.mktemp("chains"), "weight_grad",
                 dict(kWgPairs=2, kWgChainF32=2, kWgChainBf16=3))


# rows, n, k, layout of dY, type of dW, affine, accumulate: less than a step and a ragged one; single
# tiles, split ones, double ones, double then single, an odd number of tiles along n; rows of dY on
# 16-byte boundaries, beside them, and through the aligned copy; no tokens
CASES = [(1, 1, 1, "whole", "f32", 0, 0), (70, 40, 33, "whole", "f32", 1, 0),
         (300, 260, 300, "gap", "bf16", 1, 1), (130, 512, 520, "whole", "f32", 1, 0),
         (130, 601, 520, "any", "f32", 1, 1), (65, 600, 300, "any", "bf16", 0, 0),
         (700, 256, 256, "whole", "bf16", 1, 0), (200, 1300, 520, "any", "f32", 1, 0),
         (520, 1032, 300, "gap", "f32", 0, 1), (0, 5, 40, "whole", "f32", 1, 1),
         (700, 300, 1030, "whole", "f32", 1, 0)]


@pytest.mark.parametrize("case", CASES, ids=["-".join(map(str, c)) for c in CASES])
def test_values_and_bounds(weight_grad, case):
    run(weight_grad, *case, 1)


# a tile's steps in several chains: single and double tiles, split ones with several chains a part, a
# ragged last step, more tiles than one a pair, dY by plain loads and through the copy
CHAINS = [(500, 256, 1024, "whole", "f32", 1, 1), (450, 1024, 500, "whole", "bf16", 1, 0),
          (700, 1280, 300, "whole", "f32", 0, 0), (700, 1280, 300, "gap", "bf16", 0, 1),
          (1500, 256, 256, "whole", "f32", 1, 0), (330, 600, 530, "any", "f32", 1, 0),
          (330, 601, 530, "any", "bf16", 1, 1), (190, 256, 768, "whole", "f32", 0, 0)]


@pytest.mark.parametrize("case", CHAINS, ids=["-".join(map(str, c)) for c in CHAINS])
def test_sums_of_several_chains(short_chains, case):
    run(short_chains, *case, 1)


@pytest.mark.parametrize("rank", [0, 1])
@pytest.mark.parametrize("nth", [0, 3, 7, 12])
def test_a_wait_that_runs_out_in_any_chain_leaves_nan(short_chains, rank, nth):
    run(short_chains, 500, 256, 1024, "whole", "f32", 1, 0, 1, "drop_rank=%d" % rank,
        "drop_nth=%d" % nth)


@pytest.mark.parametrize("seed", [1, 2])
@pytest.mark.parametrize("hold", [None, 0, 1])
@pytest.mark.parametrize("rank", [0, 1])
def test_a_wait_that_runs_out_leaves_nan_and_no_partial_sums(weight_grad, rank, hold, seed):
    # a copy of one block's second tile never arrives.  Whichever block's wait ends first, and also
    # where the other block's writers begin to wait late: a value is complete or NaN, and the kernel ends
    args = ["drop_rank=%d" % rank, "drop_nth=4"]
    if hold is not None:
        args += ["hold_rank=%d" % hold, "hold_after=100", "hold_until=3500000000"]
    run(weight_grad, 192, 256, 1024, "whole", "f32", 1, 0, seed, *args)


@pytest.mark.parametrize("rank", [0, 1])
@pytest.mark.parametrize("case", [(700, 256, 1536, "whole", "bf16", 1, 0),
                                  (192, 1024, 1024, "whole", "f32", 0, 1)], ids=["single", "double"])
def test_a_block_that_stands_still_loses_no_tile_to_the_next(weight_grad, case, rank):
    # one block's writers read TMEM for longer than the other waits: what the other gives up must not
    # count as read, or the next tile is computed over the one that is still being read
    run(weight_grad, *case, 1, "hold_rank=%d" % rank, "hold_after=50", "hold_until=5000000000")


@pytest.mark.parametrize("seed", range(1, 5))
@pytest.mark.parametrize("case", [(700, 256, 1024, "whole", "f32", 1, 0),
                                  (700, 1024, 300, "whole", "f32", 1, 0),
                                  (700, 256, 520, "any", "f32", 1, 0)],
                         ids=["single", "double", "loads"])
def test_copies_that_arrive_late_are_waited_for(weight_grad, case, seed):
    # one copy in sixteen arrives only when nothing else can happen, long after those behind it
    run(weight_grad, *case, seed, "late=16")


@pytest.mark.parametrize("old,new", [
    ("step < kWgSlots || wg_wait_step(empty, step - kWgSlots, gave_up)", "true"),
    ("if (before) ok = wg_wait_step(empty, before - 1, gave_up);", "")])
def test_the_model_sees_a_wait_that_is_missing(tmp_path, old, new):
    def without(name, text):
        assert name != "weight_grad_kernels.cu" or text.count(old) == 1
        return text.replace(old, new)
    program = build(tmp_path, "weight_grad", dict(kWgPairs=2), without)
    with pytest.raises(AssertionError):
        run(program, 700, 300, 300, "whole", "f32", 1, 0, 1)


# ---- layer norm ------------------------------------------------------------------------------

TYPES = {"f32": "float", "bf16": "__nv_bfloat16"}


@pytest.fixture(scope="module")
def layer_norm(tmp_path_factory):
    """{type: program}; a program has the kernels of one type, so that two compilers share the work"""
    folders = {kind: tmp_path_factory.mktemp("norm" + kind) for kind in TYPES}

    def one(kind):
        def only(name, text):
            if name == "layer_norm_kernels.cu":
                for other in {"float", "__nv_bfloat16", "__half"} - {TYPES[kind]}:
                    text, n = re.subn(r"return ln_(forward|backward)_launch<%s>\([^;]*;" % other,
                                      "return NC_ERR_UNSUPPORTED;", text)
                    assert n == 2
            return text
        return build(folders[kind], "layer_norm", None, only,
                     "typedef %s T;\n" % TYPES[kind])
    with concurrent.futures.ThreadPoolExecutor(2) as pool:
        return dict(zip(TYPES, pool.map(one, TYPES)))


# a warp, several groups a block, a whole block, clusters of 2, 4 and 8 with and without a block that
# has no columns; one row, and many an owner
ROWS = [(1, 1), (3, 5), (40, 512), (20, 513), (30, 1024), (6, 1001), (7, 2000), (5, 4099), (9, 8192),
        (2, 16385), (3, 17000), (2, 32768)]


@pytest.mark.parametrize("layout,kind", [("whole", "f32"), ("whole", "bf16"), ("gap", "bf16"),
                                         ("any", "f32"), ("any", "bf16")])
@pytest.mark.parametrize("rows,cols", ROWS)
def test_norm_values_and_bounds(layer_norm, rows, cols, layout, kind):
    sms = 8 if cols > 8192 else 2
    p = layer_norm[kind]
    run(p, "forward", rows, cols, layout, "none", 0, 0, 0, sms, 1)
    run(p, "forward", rows, cols, layout, "random" if kind == "f32" else "nearest", 1, 0, 0, sms, 1)
    run(p, "backward", rows, cols, layout, "none", 1, 1, 0, sms, 1, "late=5")
    run(p, "backward", rows, cols, layout, "nearest", 0, 0, 1, sms, 2, "late=9")


@pytest.mark.parametrize("kind", TYPES)
def test_norm_of_regular_rows_in_a_kernel_of_their_own(layer_norm, kind):
    for cols in (1024, 2048):
        run(layer_norm[kind], "forward", 512, cols, "whole", "nearest", 1, 0, 0, 2, 1)


# the ring of bulk copies (a group of a warp, of a block, a cluster of two) and the exchange of a cluster
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("nth", [0, 5, 9, 22])
@pytest.mark.parametrize("case", [("backward", 200, 512, "whole", "nearest", 1, 1, 0, 2),
                                  ("backward", 60, 2048, "whole", "none", 1, 0, 0, 2),
                                  ("backward", 40, 8192, "whole", "nearest", 1, 1, 0, 4),
                                  ("backward", 30, 5000, "any", "nearest", 1, 1, 0, 4),
                                  ("forward", 60, 5000, "gap", "random", 1, 0, 0, 4)],
                         ids=lambda c: "-".join(map(str, c)))
def test_norm_wait_that_runs_out_leaves_nan_and_ends(layer_norm, case, nth, kind):
    # everything that the missing values reach is NaN, nothing else is wrong, and the waits behind the
    # first that ran out of time do not each take as long again
    for rank in range(2 if case[2] > 4096 else 1):
        said = run(layer_norm[kind], *case, 1, "drop_rank=%d" % rank, "drop_nth=%d" % nth)
        limits = int(re.search(r"at most (\d+) limits", said).group(1))
        assert limits <= 3, said


# ---- checkpoints -----------------------------------------------------------------------------

@pytest.fixture(scope="module")
def act8(tmp_path_factory):
    folder = {kind: tmp_path_factory.mktemp("act8" + kind) for kind in TYPES}
    return {kind: build(folder[kind], "act8", define="typedef %s T;\n" % TYPES[kind]) for kind in TYPES}


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("layout", ["whole", "gap", "any"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 5), (2, 32), (7, 96), (5, 513), (4, 1001), (3, 2048)])
def test_checkpoint_codes_and_bounds(act8, rows, cols, layout, kind):
    for random in (0, 1):
        run(act8[kind], rows, cols, layout, random, 1)


# ---- sizes, layouts and late or missing copies at random ---------------------------------------

def side(r, most, step):
    return r.choice([r.randint(1, most), step * r.randint(1, most // step), r.randint(1, 200)])


@pytest.mark.parametrize("seed", range(16))
def test_weight_grad_at_random(weight_grad, short_chains, seed):
    r = random.Random(seed)
    program = [weight_grad, short_chains][seed % 2]
    n, k, t = side(r, 900, 256), side(r, 700, 256), side(r, 700, 64)
    run(program, t, n, k, r.choice(["whole", "gap", "any"]), r.choice(["f32", "bf16"]),
        r.randint(0, 1), r.randint(0, 1), seed, "late=%d" % r.choice([3, 8, 20]))


@pytest.mark.parametrize("seed", range(16))
def test_weight_grad_that_waits_in_vain_at_random(weight_grad, short_chains, seed):
    # (four steps of the first tile at least have copies of scales in both blocks)
    r = random.Random(100 + seed)
    program = [weight_grad, short_chains][seed % 2]
    n, k, t = side(r, 900, 256), side(r, 700, 256), r.randint(256, 700)
    args = ["drop_rank=%d" % r.randint(0, 1), "drop_nth=0"]
    if r.random() < 0.6:
        args += ["hold_rank=%d" % r.randint(0, 1), "hold_after=%d" % r.choice([0, 50, 5000]),
                 "hold_until=%d" % r.choice([1000000000, 3900000000, 5000000000])]
    run(program, t, n, k, r.choice(["whole", "gap"]), r.choice(["f32", "bf16"]), r.randint(0, 1), 0,
        seed, *args)


@pytest.mark.parametrize("seed", range(24))
def test_norm_at_random(layer_norm, seed):
    r = random.Random(200 + seed)
    cols = r.choice([r.randint(1, 600), r.randint(1, 5000), 512 * r.randint(1, 16),
                     r.randint(4097, 20000)])
    rows = r.randint(1, max(1, min(80, 200000 // cols)))
    op = r.choice(["forward", "backward"])
    kept = r.choice(["none", "nearest"] + (["random"] if op == "forward" else []))
    run(layer_norm[r.choice(list(TYPES))], op, rows, cols, r.choice(["whole", "gap", "any"]), kept,
        r.randint(0, 1), r.randint(0, 1), r.randint(0, 1), 8 if cols > 4096 else r.randint(1, 3), seed,
        "late=%d" % r.choice([2, 5, 20]))
