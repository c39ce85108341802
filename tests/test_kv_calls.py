"""What the calls of the cache in four bits ask of the runtime, and in which order, and what a failure leaves behind: the host side
linked with a runtime that writes its calls down (tests/sanitize/kv_driver.cpp), under AddressSanitizer and UndefinedBehaviorSanitizer."""
import os
import subprocess

import pytest

from paper_2602_24044_amd import binding as B
from test_sanitizers import SAN, run_clean


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("kv_calls") / "kv_driver")
    subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", os.path.join(SAN, "kv_driver.cpp"), "-o", exe], check=True)

    def run(*script):
        """One line per call: (status, the runtime calls it made)."""
        lines = run_clean([exe], stdin="\n".join(script) + "\n").splitlines()
        return [(int(line.split()[1]), line.split()[2:]) for line in lines]
    return run


def test_calls_of_a_step(driver):
    assert driver("create", "extend 1 5", "store 1 0", "attend 1 0", "read 1", "poll 1", "release 1", "store 1 0")[1:] == [
        (0, ["plan1"]), (0, ["heads1"]), (0, ["attend1"]), (0, ["read1"]), (0, ["copy", "fill", "stream_wait1"]), (0, ["release1"]),
        (B.LORA_ERR_INVALID_ARG, [])]


def test_another_stream_waits(driver):
    assert driver("create", "extend 1 5", "store 2 0", "attend 2 0", "poll 0")[1:] == [
        (0, ["plan1"]), (0, ["record1", "wait2", "heads2"]), (0, ["attend2"]), (0, ["record2", "wait0", "copy", "fill", "stream_wait0"])]


def test_a_captured_call_records_and_waits_for_nothing(driver):
    assert driver("create", "extend 1 5", "capture 2 1", "extend 2 5", "store 2 0", "capture 2 0", "attend 1 0")[1:] == [
        (0, ["plan1"]), (0, ["plan2"]), (0, ["heads2"]), (0, ["attend1"])]


def test_create_waits_for_the_device_around_its_fills(driver):
    """The memory may still have a write of its last owner in a queue, on a stream that the fills' does not wait for."""
    assert driver("create") == [(0, ["device_wait", "fill", "fill", "device_wait"])]


def test_no_event_goes_into_a_capture(driver):
    """A call on another stream while the previous call's is being captured: there is no way to wait for that one's work, so the call is
    refused and nothing is enqueued.  Calls on the captured stream go on, and the other's once the capture has ended."""
    out = driver("create", "extend 1 5", "capture 1 1", "store 1 0", "store 2 0", "poll 2", "attend 1 0", "capture 1 0", "attend 2 0")
    assert out[1:] == [(0, ["plan1"]), (0, ["heads1"]), (B.LORA_ERR_INVALID_ARG, []), (B.LORA_ERR_INVALID_ARG, []), (0, ["attend1"]),
                       (0, ["record1", "wait2", "attend2"])]
    # the same with a release and a read, and a new step, which leaves the one before it in force
    out = driver("create", "extend 1 5", "capture 1 1", "extend 2 5", "release 2", "read 2", "capture 1 0", "attend 1 0")
    assert out[1:] == [(0, ["plan1"]), (B.LORA_ERR_INVALID_ARG, []), (B.LORA_ERR_INVALID_ARG, []), (B.LORA_ERR_INVALID_ARG, []),
                       (0, ["attend1"])]


@pytest.mark.parametrize("call,launch", [("extend 1 5", "plan1!"), ("release 1", "release1!")])
def test_a_step_ends_with_a_call_that_failed_on_the_way(driver, call, launch):
    """A launch that fails may have others behind it that ran: the step before is no longer what the tables say."""
    out = driver("create", "extend 1 7", "store 1 0", "fail " + launch[:-2], call, "store 1 0", "attend 1 0", "extend 1 5", "store 1 1",
                 "store 1 0")
    refused = (B.LORA_ERR_INVALID_ARG, [])
    assert out[1:] == [(0, ["plan1"]), (0, ["heads1"]), (B.LORA_ERR_HIP, [launch]), refused, refused, (0, ["plan1"]), refused, (0, ["heads1"])]


def test_a_step_outlives_a_call_that_was_refused(driver):
    out = driver("create", "extend 1 7", "extend 1 101", "extend 1 -1", "store 1 0")
    assert [r[0] for r in out[1:]] == [0, B.LORA_ERR_INVALID_ARG, B.LORA_ERR_INVALID_ARG, 0]


def test_a_stream_that_is_gone_holds_up_one_call_at_most(driver):
    """The header wants the latest call's stream alive.  Where the runtime says that it is not, its work is waited for with the device, and
    the calls go on."""
    out = driver("create", "extend 1 5", "end 1", "store 2 0", "attend 2 0", "poll 3")
    assert out[1:] == [(0, ["plan1"]), (0, ["device_wait", "heads2"]), (0, ["attend2"]),
                       (0, ["record2", "wait3", "copy", "fill", "stream_wait3"])]
    # an event that cannot be recorded, or not be waited for
    for name, calls in (("record", ["record1!", "device_wait", "heads2"]), ("wait", ["record1", "wait2!", "device_wait", "heads2"])):
        out = driver("create", "extend 1 5", f"fail {name}", "store 2 0", "attend 1 0")
        assert out[2:] == [(0, calls), (0, ["record2", "wait1", "attend1"])]
    # a wait that fails too, and a new stream that is not one, are errors; nothing is forgotten
    out = driver("create", "extend 1 5", "end 1", "fail device_wait", "store 2 0", "store 2 0", "end 4", "store 4 0", "store 2 0")
    assert out[1:] == [(0, ["plan1"]), (B.LORA_ERR_HIP, ["device_wait!"]), (0, ["device_wait", "heads2"]), (B.LORA_ERR_HIP, []), (0, ["heads2"])]
