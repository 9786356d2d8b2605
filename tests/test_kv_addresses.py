"""Which bytes of a page the decode kernel of vq_attention loads, from its own address function, on the host."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_no_key_is_read_past_its_end(tmp_path):
    """Heads of fewer than 64 bytes have fewer words than lane groups: the last key of a pool's last page has nothing behind it."""
    program = str(tmp_path / "kv_addresses")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__=1", "-isystem", "/opt/rocm/include",
                           "-I", os.path.join(HERE, "..", "paper_2409_17066_amd", "csrc"), os.path.join(HERE, "kv_addresses.cpp"), "-o", program])
    past, other = map(int, subprocess.check_output([program], text=True).split())
    assert past <= 0, "%d bytes past a key's end" % past
    assert other == 0
