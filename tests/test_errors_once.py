"""A call that failed is reported by that call and by no later one: the runtime's last error, which the check behind every launch
reads, is empty again.  Without a GPU: compiled for the host over a runtime that remembers its last error."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2305_03152_amd", "csrc")
SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include "spp_common.h"
static hipError_t last = hipSuccess;
static int fail = 0;                     // how many of the next calls fail, with
static hipError_t with = hipErrorOutOfMemory;
static hipError_t answer() {
    if (fail <= 0) return hipSuccess;
    --fail;
    return last = with;
}
hipError_t hipMalloc(void** p, size_t) { const hipError_t e = answer(); *p = e == hipSuccess ? malloc(1) : nullptr; return e; }
hipError_t hipFree(void* p) { free(p); return hipSuccess; }
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipGetLastError() { const hipError_t e = last; last = hipSuccess; return e; }
hipError_t hipDeviceSynchronize() { return answer(); }
const char* hipGetErrorString(hipError_t) { return "error"; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipThreadExchangeStreamCaptureMode(hipStreamCaptureMode*) { return hipSuccess; }
namespace spp { void set_error(const char*, ...) {} }
using namespace spp;
static int waits() { SPP_HIP(hipDeviceSynchronize()); return SPP_OK; }
static int launches() { SPP_HIP(hipGetLastError()); return SPP_OK; }     // what stands behind a launch that went well
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main(int, char** argv) {
    if (!strcmp(argv[1], "workspace")) {
        DevBuf a;
        RecordedBuf b;
        fail = 4;
        CHECK(a.reserve(1000) == SPP_E_OOM && launches() == SPP_OK);
        CHECK(b.reserve(1000, nullptr) == SPP_E_OOM && launches() == SPP_OK);
        CHECK(a.reserve(1000) == SPP_OK && b.reserve(1000, nullptr) == SPP_OK);
    } else if (!strcmp(argv[1], "allocation")) {
        void* p;
        for (hipError_t e : {hipErrorOutOfMemory, hipErrorStreamCaptureUnsupported}) {
            with = e;
            fail = 2;
            CHECK(device_malloc(&p, 10) == e && launches() == SPP_OK);
            fail = 2;
            CHECK(pool_take(0, &p, 10) == e && launches() == SPP_OK);
            fail = 0;
        }
        with = hipErrorOutOfMemory;
        fail = 1;
        CHECK(device_malloc(&p, 10) == hipSuccess);                      // the second attempt
    } else if (!strcmp(argv[1], "any call")) {
        with = hipErrorLaunchFailure;
        fail = 1;
        CHECK(waits() == SPP_E_HIP && launches() == SPP_OK);
    } else {
        return 3;
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("errors")
    (d / "errors.cpp").write_text(SOURCE)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__=1", "-I", os.path.join(rocm, "include"), "-I", CSRC,
                           "-o", str(d / "errors"), str(d / "errors.cpp"), "-x", "c++", os.path.join(CSRC, "spp_pool.hip"), "-pthread"])
    return str(d / "errors")


@pytest.mark.parametrize("case", ["workspace", "allocation", "any call"])
def test_a_failure_is_reported_once(program, case):
    r = subprocess.run([program, case], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
