"""A launch that fails ends its call (no GPU needed): the norm, clipping and embedding entry points over a stand-in for the runtime's launch."""
import os
import subprocess

from paper_1804_08066_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
ROCM = os.path.dirname(os.path.dirname(os.path.abspath(build.HIPCC)))


def test_no_launch_follows_one_that_failed(tmp_path):
    if build.needs_build():
        build.build()
    exe = str(tmp_path / "launch_failure_driver")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-isystem", os.path.join(ROCM, "include"),
                    os.path.join(HERE, "launch_failure_driver.cpp"), build.LIB, "-Wl,-rpath," + os.path.dirname(build.LIB), "-Wl,-rpath," + os.path.join(ROCM, "lib"),
                    "-L", os.path.join(ROCM, "lib"), "-lamdhip64", "-o", exe], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and run.stdout.strip() == "ok", run.stdout + run.stderr
