"""Token statistics launched by several host threads at once, without a GPU: what a launch keeps for the next (shared-memory
limits that are set, clusters that a device holds) is reached by threads of a program in any order."""
import os
import subprocess

import pytest

from paper_2309_00754_gb300 import build as B


def test_launches_of_several_threads_share_nothing_without_order(tmp_path):
    here = os.path.dirname(os.path.abspath(__file__))
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(B._nvcc()))), "include")
    probe = tmp_path / "probe.cpp"
    probe.write_text("int main() { return 0; }\n")
    for cmd in (["g++", "-fsanitize=thread", str(probe), "-o", str(tmp_path / "probe")], [str(tmp_path / "probe")]):
        if subprocess.run(cmd, capture_output=True).returncode != 0:
            pytest.skip("no ThreadSanitizer here")
    obj, exe = str(tmp_path / "stats.o"), str(tmp_path / "threads")
    subprocess.run([B._nvcc(), *B.ARCH, "-O0", "-Xcicc", "-O0", "-Xptxas", "-O0", "-std=c++17", "-Xcompiler",
                    "-fPIC,-fsanitize=thread,-g", "--expt-relaxed-constexpr", "-I", os.path.join(B.ROOT, "include"), "-c",
                    os.path.join(B.CSRC, "logprobs_entropy.cu"), "-o", obj], check=True)
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=thread", "-I", cuda, "-I", os.path.join(B.ROOT, "include"),
                    os.path.join(here, "update_threads.cpp"), obj, "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and "data race" not in r.stderr, r.stderr[:3000]
