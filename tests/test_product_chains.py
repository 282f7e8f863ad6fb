"""How the sums of a product are cut into chains: on the host, the jobs' own text."""
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

MAIN = r"""
using namespace natcomp;

// the chains of a unit follow each other from the first step to the last, none is empty or longer than
// most, and every one begins where its columns of k do
template <typename Job> static int check(const Job& job, uint32_t steps, uint32_t chains, uint32_t most) {
    int64_t at = 0;
    for (uint32_t c = 0; c < chains; ++c) {
        const ProductUnit w = job.unit_of(0, c);
        if (w.steps <= 0 || w.steps > (int)most || w.k != at * kProductStep || w.part != c) {
            printf("chain %u of %u: k %d, steps %d, part %u; should begin at step %lld\n", c, chains, w.k,
                   w.steps, w.part, (long long)at);
            return 1;
        }
        at += w.steps;
    }
    if (at != steps) { printf("%lld of %u steps\n", (long long)at, steps); return 1; }
    return 0;
}

int main(int argc, char** argv) {
    const std::string name = argv[1];
    const uint32_t steps = (uint32_t)atoll(argv[2]);
    int bad = 2;
    if (name == "logits") {
        CeLogits<true> a = {};
        a.steps = steps; a.parts_of = (steps + kCeChain - 1) / kCeChain;
        a.tiles_n = 1; a.split = 1; a.count = 1;
        bad = check(a, steps, a.chains(), kCeChain);
    }
    if (name == "dz") {
        CeDzJob<__half, true> a = {};
        a.steps = steps; a.parts_of = (steps + kCeDzChain - 1) / kCeDzChain;
        a.tiles_n = 1; a.count = 1; a.split = {1, 1};
        bad = check(a, steps, a.chains(), kCeDzChain);
    }
    if (name == "dtable") {
        CeDtableJob<true> a = {};
        a.count = 64 * steps - 5; a.chain_steps = kCeLongChainF16;
        a.parts_of = (steps + kCeLongChainF16 - 1) / kCeLongChainF16;
        a.tiles_m = a.tiles_n = 1; a.split = {1, 1};
        bad = check(a, steps, a.chains(), kCeLongChainF16);
    }
    if (!bad) printf("ok\n");
    return bad;
}
"""


def build(folder, main, constants=None, name="cross_entropy"):
    with open(os.path.join(MODEL, "product.hpp")) as f:
        model = f.read()

    def change(file, text):
        if file != "product.cuh":
            return text
        text = translate._without(text, ["make_box_map", "mma_shape_of", "launch_together", "grid_wait"])
        cut = [(b, e) for b, e, n, body in translate._functions(text)
               if re.search(r"\basm\b", body) and n not in ("product_pair_barrier", "product_writers_barrier")]
        for b, e in reversed(cut):
            text = text[:b] + text[e:]
        return model + text.replace("mma_pair(", "product_mma(")

    source, out = str(folder / "chains.cpp"), str(folder / "chains")
    with open(source, "w") as f:
        f.write(translate.translate(["product.cuh", name + "_kernels.cu"], constants, change) + main)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.run(["g++", "-std=c++20", "-O1", "-w", "-ffp-contract=off", "-fsanitize=address", "-I" + MODEL,
                    "-I" + os.path.join(translate.ROOT, "include"), "-I" + os.path.join(cuda, "include"),
                    "-o", out, source], check=True)
    return out


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    return build(tmp_path_factory.mktemp("chains"), MAIN)


@pytest.fixture(scope="module")
def short_chains(tmp_path_factory):
    """The program of the cross entropy's tests with chains of two steps in the backward pass, one pair."""
    with open(os.path.join(MODEL, "cross_entropy.cpp")) as f:
        main = f.read()
    kernels = ["CeDzJob<__nv_bfloat16, true>", "CeDzJob<__half, true>", "CeDtableJob<true>"]
    more = "".join("    model::cluster_of[(const void*)product_kernel<%s>] = 2;\n" % k for k in kernels)
    at = main.index("    const int dtype = ")
    return build(tmp_path_factory.mktemp("short_chains"), main[:at] + more + main[at:],
                 dict(kProductPairs=2, kCeChain=2, kCeDzChain=2, kCeLongChain=2, kCeLongChainF16=1))


def chains(program, *args):
    got = subprocess.run([program] + [str(a) for a in args], capture_output=True, text=True, timeout=120)
    assert got.returncode == 0 and got.stdout.startswith("ok"), got.stdout + got.stderr[-2000:]


# 2^18 steps are a width of 2^24; the widest layer has 2^25 - 4
@pytest.mark.parametrize("steps", [17, 33, 1000, (1 << 18) - 1, 1 << 18, (1 << 18) + 1, 1 << 19, (1 << 25) - 4])
def test_the_logits_chains_cover_every_step_once(program, steps):
    chains(program, "logits", steps)


@pytest.mark.parametrize("steps", [17, 64, 65, (1 << 18) + 1, 1 << 19, (1 << 25) - 4])
def test_the_chains_of_the_recomputed_logits_cover_every_step_once(program, steps):
    chains(program, "dz", steps)


@pytest.mark.parametrize("steps", [33, 128, 1000, (1 << 20) + 1, (1 << 25) - 4])
def test_the_table_gradients_chains_cover_every_step_once(program, steps):
    chains(program, "dtable", steps)


@pytest.mark.parametrize("args", [(300, 136, 257, "f16", "whole", 2, "same", 0, 0), (130, 300, 520, "bf16", "any", 5, "f32", 1, 1),
                                  (20, 700, 40, "f16", "whole", 0, "f32", 0, 0), (5, 128, 300, "bf16", "whole", 0, "same", 0, 1),
                                  (400, 40, 300, "f16", "any", 0, "f32", 1, 0), (500, 24, 260, "bf16", "whole", 1, "same", 0, 0)],
                         ids=str)
def test_gradients_of_sums_in_chains(short_chains, args):
    chains(short_chains, *args, 1)


@pytest.mark.parametrize("rank", [0, 1])
@pytest.mark.parametrize("nth", [3, 9, 17])
def test_a_wait_that_runs_out_in_a_chain_leaves_nan(short_chains, rank, nth):
    chains(short_chains, 300, 300, 260, "f16", "whole", 0, "f32", 0, 0, 1, "drop_rank=%d" % rank, "drop_nth=%d" % nth)
