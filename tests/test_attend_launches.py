"""Every call that is accepted makes launches that the runtime takes, whatever its sizes: recorded without a GPU."""
import os
import subprocess

from paper_2505_24133_amd import build as B


def test_launches_hold_what_a_launch_can(repo_root, tmp_path):
    if not os.path.exists(B.LIB):
        B.build()
    exe = str(tmp_path / "attend_launches")
    inc = B.rocm_include()
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", inc, "-I", os.path.join(repo_root, "include"),
                    os.path.join(repo_root, "tests", "attend_launches.cpp"), "-o", exe, "-rdynamic", B.LIB,
                    "-L" + os.path.join(os.path.dirname(inc), "lib"), "-lamdhip64", "-Wl,-rpath," + os.path.dirname(B.LIB)], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300).stdout
    last = out.splitlines()[-1].split()
    assert last[2:4] == ["bad", "0"], out[-3000:]
    assert int(last[1]) > 1000
