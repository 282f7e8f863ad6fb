"""The launch of kernels whose blocks wait for each other takes no more blocks than run at the same time: its text, on
the host, against stand-ins for the two calls that it makes."""
import os
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(HERE, "device_model"))

import translate  # noqa: E402

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no C++ compiler")

MAIN = r"""
#include <cstdio>
#include <cstdlib>
#include <cuda_runtime_api.h>

static int fits, launched = -1;
static bool cooperative;
static cudaError_t answer;
static cudaError_t ask(int* n, const cudaLaunchConfig_t* c) {
    if (c->blockDim.x != 320 || c->dynamicSmemBytes != 1000) exit(3);
    *n = fits;
    return answer;
}
static cudaError_t go(const cudaLaunchConfig_t* c) {
    launched = (int)c->gridDim.x;
    for (unsigned i = 0; i < c->numAttrs; ++i)
        cooperative |= c->attrs[i].id == cudaLaunchAttributeCooperative && c->attrs[i].val.cooperative;
    return cudaSuccess;
}
#define cudaOccupancyMaxActiveClusters(n, kernel, c) ask(n, c)
#define cudaLaunchKernelEx(c, kernel, ...) go(c)
template <typename... A> static void unused(const A&...) {}
%s
int main(int argc, char** argv) {
    fits = atoi(argv[2]);
    answer = (cudaError_t)atoi(argv[3]);
    const cudaError_t e = launch_together(0, dim3(atoi(argv[1])), dim3(320), 1000, nullptr, 1, 2);
    printf("%%d %%d %%d\n", launched, (int)e, (int)cooperative);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    with open(os.path.join(translate.CSRC, "product.cuh")) as f:
        text = f.read()
    found = [body for _, _, name, body in translate._functions(text) if name == "launch_together"]
    assert len(found) == 1
    folder = tmp_path_factory.mktemp("launch")
    source, out = str(folder / "launch.cpp"), str(folder / "launch")
    with open(source, "w") as f:
        f.write(MAIN % found[0])
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.run(["g++", "-std=c++17", "-w", "-I" + os.path.join(cuda, "include"), "-o", out, source], check=True)
    return out


@pytest.mark.parametrize("blocks,pairs,launched", [(148, 74, 148), (148, 73, 146), (148, 1, 2), (2, 74, 2), (30, 15, 30),
                                                   (30, 14, 28)])
def test_no_more_blocks_than_fit_at_a_time(program, blocks, pairs, launched):
    got = subprocess.run([program, str(blocks), str(pairs), "0"], capture_output=True, text=True, check=True)
    assert got.stdout.split() == [str(launched), "0", "1"]


@pytest.mark.parametrize("pairs,error", [(0, 0), (0, 46), (74, 46)])
def test_nothing_is_launched_where_none_fits_or_the_device_does_not_say(program, pairs, error):
    got = subprocess.run([program, "148", str(pairs), str(error)], capture_output=True, text=True, check=True)
    launched, status, _ = got.stdout.split()
    assert launched == "-1" and status != "0"
