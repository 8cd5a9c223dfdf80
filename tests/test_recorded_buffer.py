"""A buffer whose address recorded work may hold, without a GPU: compiled for the host over an allocator that knows which blocks
live and refuses what a recording of the strictest mode refuses."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2305_03152_amd", "csrc")
SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <set>
#include "spp_common.h"
static std::set<void*> live;
static hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
static hipStreamCaptureMode mode = hipStreamCaptureModeGlobal;           // the thread's
static int room = 1 << 30;
static bool refused() { return status != hipStreamCaptureStatusNone && mode != hipStreamCaptureModeRelaxed; }
hipError_t hipMalloc(void** p, size_t) {
    *p = nullptr;
    if (refused()) return hipErrorStreamCaptureUnsupported;
    if (room-- <= 0) return hipErrorOutOfMemory;
    live.insert(*p = malloc(1));             // never freed: no address comes twice
    return hipSuccess;
}
hipError_t hipFree(void* p) {
    if (status != hipStreamCaptureStatusNone) { puts("freed while the stream records"); exit(2); }
    if (!live.erase(p)) { puts("freed twice"); exit(2); }
    return hipSuccess;
}
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "error"; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* s) { *s = status; return hipSuccess; }
hipError_t hipThreadExchangeStreamCaptureMode(hipStreamCaptureMode* m) { std::swap(mode, *m); return hipSuccess; }
namespace spp { void set_error(const char*, ...) {} }
using namespace spp;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
static void record(bool on) { status = on ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone; }
int main(int, char** argv) {
    RecordedBuf b;
    if (!strcmp(argv[1], "outgrown after a recording")) {
        CHECK(b.reserve(1000, nullptr) == SPP_OK);
        record(true);
        CHECK(b.reserve(1000, nullptr) == SPP_OK);
        void* const held = b.ptr;
        record(false);
        CHECK(b.reserve(100000, nullptr) == SPP_OK && b.ptr != held && live.count(held));
        void* const eager = b.ptr;                       // no recording has used this one
        CHECK(b.reserve(10000000, nullptr) == SPP_OK && live.count(held) && !live.count(eager) && live.size() == 2);
    } else if (!strcmp(argv[1], "begun and grown while recording")) {
        record(true);
        CHECK(b.reserve(1000, nullptr) == SPP_OK && mode == hipStreamCaptureModeGlobal);
        void* const first = b.ptr;
        CHECK(b.reserve(100000, nullptr) == SPP_OK && live.count(first) && live.size() == 2);
        record(false);
        CHECK(b.reserve(10000000, nullptr) == SPP_OK && live.size() == 3);
    } else if (!strcmp(argv[1], "an eager block outgrown while recording")) {
        CHECK(b.reserve(1000, nullptr) == SPP_OK);
        record(true);
        CHECK(b.reserve(100000, nullptr) == SPP_OK && live.size() == 2);
        record(false);
    } else if (!strcmp(argv[1], "no memory")) {
        record(true);
        CHECK(b.reserve(1000, nullptr) == SPP_OK);
        void* const held = b.ptr;
        room = 0;
        CHECK(b.reserve(100000, nullptr) == SPP_E_OOM && mode == hipStreamCaptureModeGlobal && live.count(held));
        room = 1;
        CHECK(b.reserve(100000, nullptr) == SPP_OK && live.size() == 2);
        record(false);
    } else if (!strcmp(argv[1], "never recorded")) {
        for (size_t n = 1; n < (size_t)1 << 40; n *= 3) CHECK(b.reserve(n, nullptr) == SPP_OK && live.size() == 1);
    } else {
        return 3;
    }
    b.release();
    CHECK(live.empty() && b.outgrown.empty());
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("recorded_buffer")
    (d / "buffer.cpp").write_text(SOURCE)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__=1", "-I", os.path.join(rocm, "include"), "-I", CSRC,
                           "-o", str(d / "buffer"), str(d / "buffer.cpp"), "-x", "c++", os.path.join(CSRC, "spp_pool.hip"), "-pthread"])
    return str(d / "buffer")


@pytest.mark.parametrize("case", ["outgrown after a recording", "begun and grown while recording", "an eager block outgrown while recording",
                                  "no memory", "never recorded"])
def test_blocks_that_a_recording_may_hold(program, case):
    r = subprocess.run([program, case], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_what_recorded_calls_write_to_is_such_a_buffer(tmp_path):
    """The workspaces of the calls that may be recorded: propagations and the weight gradient."""
    src = tmp_path / "members.cpp"
    src.write_text('#include "spp_common.h"\n#include <type_traits>\n' + "".join(
        "static_assert(std::is_same<decltype(spp_ctx::%s), spp::RecordedBuf>::value, \"%s\");\n" % (m, m)
        for m in ("y0", "y1", "tot", "acc", "frontier", "xvals", "bins", "gradws")))
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    r = subprocess.run(["g++", "-std=c++17", "-fsyntax-only", "-D__HIP_PLATFORM_AMD__=1", "-I", os.path.join(rocm, "include"), "-I", CSRC, str(src)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
