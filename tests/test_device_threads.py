"""What the planners keep of a device between calls may be asked for by several threads at once: under the thread sanitizer, without a GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.dirname(os.path.abspath(__file__))


def test_threads_that_plan_at_the_same_time(tmp_path):
    exe = tmp_path / "device_driver"
    subprocess.check_call(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=thread", "-D__HIP_PLATFORM_AMD__", "-I" + os.path.join(ROOT, "paper_2604_04215_amd", "csrc"),
                           "-I" + os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"), os.path.join(HERE, "device_driver.cpp"), "-o", str(exe), "-pthread"])
    run = subprocess.run([str(exe)], capture_output=True, text=True)
    assert run.returncode == 0 and "wrong 0" in run.stdout, run.stdout + run.stderr


def test_no_other_table_of_devices():
    csrc = os.path.join(ROOT, "paper_2604_04215_amd", "csrc")
    for name in os.listdir(csrc):
        if name != "device.hpp":
            with open(os.path.join(csrc, name)) as f:
                assert "MultiprocessorCount" not in f.read(), name
