"""The order that calls on one gated block keep on the device, seen from the host: the library's calls of the HIP runtime go to one that writes them down and runs
nothing, so what a wait would have prevented cannot happen here."""
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(os.path.dirname(HERE), "paper_2312_08728_amd", "libbmgd.so")

# Matrices are addresses that nothing reads.  run(stream): a forward call, and what it asked of the runtime.
PROGRAM = """
import ctypes as C, sys
hip = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
lib = C.CDLL(sys.argv[2])
hip.trace_text.restype = C.c_char_p
config = (C.c_int64 * 8)(64, 64, 64, 16, 1, 0, 0, 0)           # dtype and activation share a word
block = C.c_void_p()
assert lib.bmgd_gated_create(C.byref(config), C.byref(block)) == 0
tensors = (C.c_int64 * 24)(*[v for i in range(12) for v in ((i + 1 << 32) if i < 5 else 0, 64)])
lib.bmgd_gated_last_error.restype = C.c_char_p
def run(stream, want=0):
    hip.trace_clear()
    rc = lib.bmgd_gated_forward(block, C.c_int64(16), C.byref(tensors), C.c_void_p(stream))
    assert rc == want, (rc, lib.bmgd_gated_last_error(block))
    return hip.trace_text().decode().split("\\n")[:-1]
def launched(stream, device=0):
    return ["launch %d on %d" % (stream, device)] * 2
def ordered(before, now):
    return ["record %d" % before, "wait %d" % now] + launched(now)
"""


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    out = tmp_path_factory.mktemp("hip") / "libhip_trace.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", os.path.join(HERE, "hip_trace.cpp"), "-o", str(out)], check=True)
    return str(out)


def _run(runtime, body):
    res = subprocess.run([sys.executable, "-c", PROGRAM + body, runtime, LIB], capture_output=True, text=True, timeout=100)
    assert res.returncode == 0, res.stdout + res.stderr


def test_calls_on_one_stream_need_no_marker_and_others_wait(runtime):
    _run(runtime, """
assert run(1) == launched(1) and run(1) == launched(1)
assert run(2) == ordered(1, 2)
assert run(0) == ordered(2, 0) and run(0) == launched(0)
assert run(1) == ordered(0, 1)
""")


@pytest.mark.parametrize("after", [2, 3])
def test_a_captured_call_does_not_come_between_the_calls_around_it(runtime, after):
    """A call on stream 1, one captured on stream 2, then a call on stream 3 or on 2 itself: that one waits for the first."""
    _run(runtime, f"""
assert run(1) == launched(1)
hip.trace_capture(2, 1)
assert run(2) == launched(2) and run(2) == launched(2)
hip.trace_capture(2, 0)
assert run({after}) == ordered(1, {after})
""")


def test_a_captured_call_that_is_the_first_is_nothing_to_wait_for(runtime):
    """Nothing has run on its stream; destroying the block waits for what its graph may have launched all the same."""
    _run(runtime, """
hip.trace_capture(2, 1)
assert run(2) == launched(2)
hip.trace_capture(2, 0)
assert run(3) == launched(3)
lib.bmgd_gated_destroy(block)
assert hip.trace_text().decode().split("\\n")[-2] == "synchronize"
""")
    _run(runtime, """
hip.trace_capture(2, 1)
assert run(2) == launched(2)
hip.trace_clear()
lib.bmgd_gated_destroy(block)
assert hip.trace_text() == b"synchronize\\n"
""")


def test_calls_captured_on_the_stream_of_the_call_before(runtime):
    """The stream itself orders them, and the calls behind the capture."""
    _run(runtime, """
assert run(1) == launched(1)
hip.trace_capture(1, 1)
assert run(1) == launched(1)
hip.trace_capture(1, 0)
assert run(1) == launched(1) and run(2) == ordered(1, 2)
""")


def test_a_call_that_cannot_be_ordered_is_refused(runtime):
    """Its wait for the call before would become a part of the graph that is being captured there."""
    _run(runtime, """
assert run(1) == launched(1)
hip.trace_capture(1, 1)
assert run(2, want=2) == [] and b"captured" in lib.bmgd_gated_last_error(block)
hip.trace_capture(1, 0)
assert run(2) == ordered(1, 2)
""")


def test_a_call_leaves_the_device_that_was_current(runtime):
    """The block was made on device 0; a call from a thread whose device is 1 runs on 0 and comes back with 1, also when it fails."""
    _run(runtime, """
now = C.c_int()
def current():
    hip.hipGetDevice(C.byref(now))
    return now.value
hip.hipSetDevice(1)
assert run(1) == launched(1, device=0) and current() == 1
backward = lambda: lib.bmgd_gated_backward(block, C.c_int64(16), C.byref(tensors), C.c_void_p(1))
for i in range(5, 12):
    tensors[2 * i] = i + 1 << 32
assert backward() == 0 and current() == 1
hip.trace_capture(1, 1)
assert run(2, want=2) == [] and current() == 1
lib.bmgd_gated_destroy(block)
assert current() == 1
""")
