"""The norm, clipping and embedding entry points over a stand-in for the runtime's launch (no GPU needed): a launch that fails ends its call,
and what is empty is no reason to refuse one."""
import os
import subprocess

import pytest

from paper_1804_08066_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
ROCM = os.path.dirname(os.path.dirname(os.path.abspath(build.HIPCC)))


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if build.needs_build():
        build.build()
    exe = str(tmp_path_factory.mktemp("driver") / "launch_failure_driver")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-isystem", os.path.join(ROCM, "include"),
                    os.path.join(HERE, "launch_failure_driver.cpp"), build.LIB, "-Wl,-rpath," + os.path.dirname(build.LIB),
                    "-Wl,-rpath," + os.path.join(ROCM, "lib"), "-L", os.path.join(ROCM, "lib"), "-lamdhip64", "-o", exe], check=True)
    return exe


def passes(driver, checks):
    run = subprocess.run([driver, checks], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and run.stdout.strip() == "ok", run.stdout + run.stderr


def test_no_launch_follows_one_that_failed(driver):
    passes(driver, "failures")


def test_what_is_empty_lies_over_nothing(driver):
    passes(driver, "empty")
