"""The kernels of the cross entropy, the orthogonalised update and the embedding thread by thread on
the host (tests/device_model): values against sums in 64 bits, the bounds of every access, copies that
arrive late, and waits that run out of time."""
import os
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


def build(folder, name, constants=None, replace=()):
    """replace: (text, other text) of the kernels' source, for constants that are not plain numbers"""
    with open(os.path.join(MODEL, "product.hpp")) as f:
        model = f.read()

    def change(file, text):
        if file == "product.cuh":
            text = translate._without(text, ["make_box_map", "mma_shape_of", "launch_together", "grid_wait"])
            cut = [(b, e) for b, e, n, body in translate._functions(text)
                   if re.search(r"\basm\b", body) and n not in ("product_pair_barrier", "product_writers_barrier")]
            for b, e in reversed(cut):
                text = text[:b] + text[e:]
            text = model + text.replace("mma_pair(", "product_mma(")
        if file == "embedding_kernels.cu":
            text = translate._without(text, ["shared_store_pair_at"])
        for old, new in replace:
            if file == name + "_kernels.cu":
                assert text.count(old) == 1, old
                text = text.replace(old, new)
        return text

    source, program = str(folder / (name + ".cpp")), str(folder / name)
    with open(os.path.join(MODEL, name + ".cpp")) as f:
        main = f.read()
    with open(source, "w") as f:
        f.write(translate.translate(["product.cuh", name + "_kernels.cu"], constants, change) + main)
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


# ---- cross entropy: rows, width, vocabulary, type, layout, which rows have no target, type of dtable,
# accumulate, dlse.  One pair; the vocabulary in pieces of 256 or 512 for the second program.

@pytest.fixture(scope="module")
def cross_entropy(tmp_path_factory):
    return build(tmp_path_factory.mktemp("ce"), "cross_entropy", dict(kProductPairs=2))


@pytest.fixture(scope="module")
def small_pieces(tmp_path_factory):
    return build(tmp_path_factory.mktemp("ce_pieces"), "cross_entropy",
                 dict(kProductPairs=4, kCeLeastPiece=256, kCeGatherBlocks=3, kCeChain=2),
                 [("1ull << 27", "1ull << 8"), ("1ull << 25", "1ull << 8")])


CROSS_ENTROPY = [(1, 1, 1, "bf16", "whole", 0, "same", 0, 0), (5, 40, 33, "f16", "any", 0, "f32", 1, 1),
                 (70, 72, 300, "bf16", "any", 3, "same", 1, 1),
                 (300, 136, 257, "f16", "whole", 2, "same", 0, 0),
                 (130, 300, 520, "bf16", "whole", 5, "f32", 0, 1),
                 (40, 24, 1400, "bf16", "whole", 0, "same", 0, 0),
                 (3, 16, 40, "bf16", "whole", 1, "same", 0, 1)]


@pytest.mark.parametrize("case", CROSS_ENTROPY, ids=["-".join(map(str, c)) for c in CROSS_ENTROPY])
def test_cross_entropy(cross_entropy, case):
    run(cross_entropy, *case, 1)


@pytest.mark.parametrize("case", CROSS_ENTROPY[2:], ids=["-".join(map(str, c)) for c in CROSS_ENTROPY[2:]])
def test_cross_entropy_in_pieces(small_pieces, case):
    run(small_pieces, *case, 1)


@pytest.mark.parametrize("seed", [1, 2])
def test_cross_entropy_with_late_copies(cross_entropy, seed):
    run(cross_entropy, 300, 500, 600, "bf16", "whole", 7, "same", 0, 0, seed, "late=8")


@pytest.mark.parametrize("rank", [0, 1])
@pytest.mark.parametrize("nth", [0, 9])
def test_cross_entropy_wait_that_runs_out_leaves_nan(cross_entropy, rank, nth):
    run(cross_entropy, 20, 300, 260, "bf16", "whole", 0, "same", 0, 0, 1, "drop_rank=%d" % rank,
        "drop_nth=%d" % nth)


# ---- orthogonalised update: batch, rows, cols, types, layout, steps

@pytest.fixture(scope="module")
def orthogonalize(tmp_path_factory):
    return build(tmp_path_factory.mktemp("ortho"), "orthogonalize", dict(kProductPairs=1))


ORTHOGONALIZE = [(1, 1, 1, "f32", "f32", "whole", 2), (2, 40, 24, "bf16", "f16", "any", 2),
                 (1, 24, 300, "f32", "bf16", "whole", 1), (2, 300, 270, "f16", "f32", "whole", 1),
                 (1, 270, 530, "f32", "bf16", "any", 1), (3, 33, 70, "f32", "bf16", "any", 0)]


@pytest.mark.parametrize("case", ORTHOGONALIZE, ids=["-".join(map(str, c)) for c in ORTHOGONALIZE])
def test_orthogonalize(orthogonalize, case):
    run(orthogonalize, *case, 1)


@pytest.fixture(scope="module")
def split_sums(tmp_path_factory):
    # sums of A of more than eight steps in two or more parts, although there is one pair only
    return build(tmp_path_factory.mktemp("ortho_split"), "orthogonalize", dict(kProductPairs=1, kOrthoLong=8),
                 [("most = kProductPairs / units", "most = 3"), ("squares < kProductPairs && ", "")])


@pytest.mark.parametrize("case", [(1, 40, 700, "f32", "f32", "whole", 2), (1, 600, 33, "f32", "bf16", "any", 2)],
                         ids=["wide", "tall"])
def test_orthogonalize_with_split_sums(split_sums, case):
    run(split_sums, *case, 1)


def test_orthogonalize_with_late_copies(orthogonalize):
    run(orthogonalize, 1, 260, 300, "f32", "f32", "whole", 1, 2, "late=8")


@pytest.mark.parametrize("rank", [0, 1])
def test_orthogonalize_wait_that_runs_out_leaves_nan(orthogonalize, rank):
    run(orthogonalize, 1, 200, 300, "f32", "f32", "whole", 1, 1, "drop_rank=%d" % rank, "drop_nth=3")


# ---- embedding: rows, vocabulary, cols, types, layout, how the tokens fall, bytes of one, accumulate

@pytest.fixture(scope="module")
def embedding(tmp_path_factory):
    return build(tmp_path_factory.mktemp("embed"), "embedding")


EMBEDDING = [(1, 1, 1, "f32", "f32", "whole", "one", 8, 0), (0, 7, 9, "bf16", "f32", "whole", "none", 8, 0),
             (40, 300, 24, "bf16", "bf16", "whole", "many", 4, 0),
             (40, 300, 37, "bf16", "f32", "any", "many", 8, 1),
             (700, 50, 20, "f16", "f16", "whole", "few", 8, 0),
             (900, 1200, 9, "f32", "bf16", "any", "one", 4, 0),
             (300, 40, 1100, "bf16", "f32", "whole", "few", 8, 1),
             (33, 20, 12, "f16", "f32", "whole", "none", 8, 0),
             (9000, 3000, 3, "f32", "f32", "whole", "many", 8, 0)]


@pytest.mark.parametrize("case", EMBEDDING, ids=["-".join(map(str, c)) for c in EMBEDDING])
def test_embedding(embedding, case):
    run(embedding, *case, 1)


@pytest.fixture(scope="module")
def sorted_embedding(tmp_path_factory):
    # clears some of the rows beside the sort and some later, and
    # takes runs of more than three segments for long ones
    return build(tmp_path_factory.mktemp("embed_sorted"), "embedding",
                 dict(kJoinShort=3),
                 [("kClearBeside = 64 << 20", "kClearBeside = 8 << 10")])


SORTED = [(600, 50, 20, "f16", "f16", "whole", "few", 8, 0), (900, 1200, 9, "f32", "bf16", "any", "one", 4, 0),
          (700, 3000, 12, "bf16", "f32", "whole", "many", 8, 0), (520, 40, 1100, "bf16", "f32", "any", "few", 8, 1),
          (513, 20, 12, "f16", "f32", "whole", "none", 8, 0), (4500, 300, 3, "f32", "f32", "any", "many", 8, 1),
          (9000, 70000, 2, "f32", "f32", "whole", "many", 8, 0)]


@pytest.fixture(scope="module")
def chunked_embedding(tmp_path_factory):
    # sorts in chunks through memory what would fit the chip
    return build(tmp_path_factory.mktemp("embed_chunks"), "embedding", dict(kSortMaxBlocks=2),
                 [("<= (uint64_t)kSortChunk;", "<= 0;"), ("min((int)((each + kSortThreads - 1) / kSortThreads), kSortEach)", "2")])


@pytest.mark.parametrize("case", [(700, 50, 20, "f16", "f16", "whole", "few", 8, 0),
                                  (9001, 3000, 3, "f32", "f32", "whole", "many", 4, 1)], ids=["one", "two"])
def test_embedding_sorted_in_chunks(chunked_embedding, case):
    run(chunked_embedding, *case, 1)


@pytest.mark.parametrize("case", SORTED, ids=["-".join(map(str, c)) for c in SORTED])
def test_embedding_sorted(sorted_embedding, case):
    run(sorted_embedding, *case, 1)
