"""The choice of kernels of vq_attention_shared at its arguments' largest sizes, on the host, with checks of signed arithmetic."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("plan") / "shared_plan")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__=1", "-isystem", "/opt/rocm/include",
                           "-I", os.path.join(HERE, "..", "paper_2409_17066_amd", "csrc"), os.path.join(HERE, "shared_plan.cpp"), "-o", path])
    return path


@pytest.mark.parametrize("seqs,prefixes,heads,new,prefix,own", [
    (65535, 65535, 65535, 1, 1 << 20, 64), (65535, 1, 65535, 1, 4096, 64), (2, 65535, 65535, 1, 4096, 64), (65535, 65535, 65535, 1 << 14, 1 << 30, 1 << 30),
    (1 << 15, 65535, 32769, 1 << 15, 1 << 20, 1 << 20), (2, 65535, 65535, 1 << 29, 1 << 30, 64),
])
def test_no_number_of_workgroups_passes_its_type(program, seqs, prefixes, heads, new, prefix, own):
    """Sequences or prefixes times key heads pass 2^31: no such call is taken by one launch for both halves, nor does its number of workgroups look like a smaller one."""
    done = subprocess.run([program] + [str(n) for n in (seqs, prefixes, heads, new, prefix, own)], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
    assert done.returncode == 0, done.stderr
    status, launched = done.stdout.split()
    assert int(status) == 0 and launched in ("whole", "half")


def test_what_it_launches_of_ordinary_sizes(program):
    assert subprocess.check_output([program, "64", "1", "8", "1", "8192", "1021"], text=True).split() == ["0", "halves"]
