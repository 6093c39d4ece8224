"""The host side of the calls on draft trees, on a CUDA runtime that is not there: a program of its own defines the runtime
calls that the library makes before and around a launch, fails the ones that it is told to, and prints what is launched."""
import os
import subprocess

import pytest

from conftest import ROOT
from paper_2603_11243_b200 import build as ssd_build

PROGRAM = r"""
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include "ssd.h"

static const char *failing = "";          // the runtime call that fails
static int registers = 168;
static cudaError_t last = cudaSuccess;    // what cudaGetLastError has to tell, once
static cudaError_t result(const char *name, cudaError_t error) {
    if (strcmp(failing, name)) return cudaSuccess;
    return last = error;
}

static CUresult encode(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                       const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
    return CUDA_SUCCESS;
}

extern "C" {
cudaError_t cudaGetDevice(int *d) { *d = 0; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int *v, cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t cudaFuncGetAttributes(cudaFuncAttributes *a, const void *) {
    memset(a, 0, sizeof *a);
    a->numRegs = registers;
    return result("cudaFuncGetAttributes", cudaErrorLaunchFailure);
}
cudaError_t cudaFuncSetAttribute(const void *, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaGetLastError(void) { const cudaError_t e = last; last = cudaSuccess; return e; }
cudaError_t cudaGetDriverEntryPointByVersion(const char *, void **f, unsigned, unsigned long long, cudaDriverEntryPointQueryResult *r) {
    const bool bad = result("cudaGetDriverEntryPointByVersion", cudaErrorInitializationError) != cudaSuccess;
    *f = bad ? nullptr : (void *)encode;
    if (r) *r = bad ? cudaDriverEntryPointSymbolNotFound : cudaDriverEntryPointSuccess;
    return bad ? cudaErrorInitializationError : cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *, void **) {
    printf("launch %u %u\n", c->gridDim.x, c->blockDim.x);
    return cudaSuccess;
}
}

// attention page_size max_pages M B: one layer of M nodes of B utterances, 4 query and 2 kv heads
static int attention(int page, int max_pages, int64_t M, int B) {
    char *const at = (char *)4096;                     // never looked at
    ssd_heads q{at, 256, 64, 4}, kv{at, 128, 64, 2};
    ssd_kv_cache c{at, at, (int64_t)page * 128, 128, 64, 1024, page, 2, 64, SSD_BF16, max_pages, (int32_t *)at, max_pages, (int32_t *)at};
    return ssd_tree_attention(&q, &kv, &kv, &c, (int64_t *)at, nullptr, B, M, (int)M, 0.125f, 0.f, &q, nullptr, (uint32_t *)at, at,
                              (size_t)1 << 40, nullptr);
}

int main(int argc, char **argv) {
    for (int i = 1; i < argc; ++i) {
        if (!strncmp(argv[i], "fail=", 5)) failing = argv[i] + 5;
        else if (!strncmp(argv[i], "registers=", 10)) registers = atoi(argv[i] + 10);
        else {
            int page, pages, M, B;
            sscanf(argv[i], "%d,%d,%d,%d", &page, &pages, &M, &B);
            const int rc = attention(page, pages, M, B);
            printf("answer %d %d\n", rc, rc == SSD_ERR_CUDA ? ssd_last_cuda_error() : 0);
        }
    }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    lib = os.path.dirname(ssd_build.build())
    d = tmp_path_factory.mktemp("host")
    (d / "host.cpp").write_text(PROGRAM)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    # the program's own definitions come before the runtime's
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-rdynamic", "-isystem", os.path.join(cuda, "include"),
                    "-I", os.path.join(ROOT, "include"), str(d / "host.cpp"), "-o", str(d / "host"), "-L" + lib, "-l:libssd.so",
                    "-Wl,-rpath," + lib, "-L" + os.path.join(cuda, "lib64"), "-lcudart", "-Wl,-rpath," + os.path.join(cuda, "lib64")],
                   check=True)
    return lambda *args: subprocess.run([str(d / "host"), *args], check=True, capture_output=True, text=True).stdout.split("\n")[:-1]


ONE = "16,100,1,1"


def test_a_call_launches_its_two_kernels(program):
    out = program(ONE)
    assert len(out) == 3 and out[2] == "answer 0 0" and out[0].endswith(" 384")


@pytest.mark.parametrize("call", ["cudaFuncGetAttributes", "cudaGetDriverEntryPointByVersion"])
def test_an_error_of_the_runtime_is_not_remembered(program, call):
    out = program("fail=" + call, ONE, "fail=", ONE)
    assert out[0].startswith("answer 5 ") and out[0] != "answer 5 0"
    assert out[1].startswith("launch ") and out[-1] == "answer 0 0"


def test_a_kernel_of_too_few_registers_is_never_launched(program):
    assert program("registers=160", ONE, ONE) == ["answer 5 98"] * 2


@pytest.mark.parametrize("page", [1, 2, 3, 7])
def test_small_pages_get_as_many_ctas_as_they_have_tiles(program, page):
    """A page of fewer than 8 slots is a tile of its own: two heads of a node and of 20 pages are 42 tiles."""
    out = program("%d,20,1,1" % page)
    assert out[0] == "launch 42 384" and out[-1] == "answer 0 0"


def test_small_calls_of_larger_pages_launch_what_they_did(program):
    for case, grid in (("8,20,1,1", 42), ("16,20,1,1", 82), ("16,100,1,1", 148), ("64,1,3,2", 36), ("100,1,1,1", 28)):
        assert program(case)[0] == "launch %d 384" % grid, case
