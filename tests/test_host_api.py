"""The C-ABI layer as host code, with launches that do nothing (tests/host_api): what it refuses before anything runs."""
import os
import shutil
import subprocess

import pytest


@pytest.mark.parametrize("name", ["overlaps", "undefined"])
def test_on_the_host(name, tmp_path, repo_root):
    exe = str(tmp_path / name)
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(shutil.which("hipcc") or "/opt/rocm/bin/hipcc"))), "include")
    subprocess.run([shutil.which("g++") or shutil.which("c++"), "-std=c++17", "-O1", "-g", "-w", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-D__HIP_PLATFORM_AMD__=1", "-isystem", include, os.path.join(repo_root, "tests", "host_api", name + "_main.cpp"), "-o", exe], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0 and run.stdout == "ok\n", run.stdout + run.stderr
