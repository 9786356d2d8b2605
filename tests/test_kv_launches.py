"""What vq_kv_append, vq_attention and vq_residual_norm launch, on a machine without a GPU (launch_log.cpp in place of the HIP runtime): all of a call or, where it
is refused, nothing, and grids of sizes that a launch can have."""
import json
import os
import random
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CHILD = """
import ctypes, json, os, sys
shim = sys.argv[1]
log = ctypes.CDLL(shim, mode=ctypes.RTLD_GLOBAL)
log.launch_log.restype = ctypes.c_char_p
sys.modules["torch"] = None
sys.path.insert(0, sys.argv[2])
import paper_2409_17066_amd as vq
vq.load()
libc = ctypes.CDLL(None)
out = []
for call in json.load(sys.stdin):
    libc.setenv(b"VQ_SWITCHES", call.get("switches", "").encode(), 1)
    d, q_heads = call["cache"], call["q_heads"]
    at = 1 << 41
    d = dict(dict(struct_size=ctypes.sizeof(vq.vq_kv_desc), k_pages=at, v_pages=at, k_scales=at, v_scales=at, page_table=at, lengths=at, reserved=0,
                  table_stride=d["table_pages"], k_page_stride=d["kv_heads"] * d["page_tokens"] * d["head_dim"],
                  v_page_stride=d["kv_heads"] * d["page_tokens"] * d["head_dim"]), **d)
    cache = vq.vq_kv_desc(**{k: v for k, v in d.items() if k != "starts"}, starts=at if d.get("starts") else None)
    width = q_heads * d["head_dim"]
    log.launch_log_clear()
    asked = None
    if call["entry"] == "append":
        rc = vq.vq_kv_append(cache, at, d["kv_heads"] * d["head_dim"], at, d["kv_heads"] * d["head_dim"], at, width, q_heads, at, width)
    else:
        asked = vq.vq_attention_workspace_bytes(cache, q_heads, call.get("window", 0), 0)
        rc = vq.vq_attention(cache, at, width, q_heads, 0.1, call.get("window", 0), 0, at, width, None, at, asked)
    launches = [line.split("|") for line in log.launch_log().decode().splitlines()]
    out.append(dict(status=rc, asked=asked, launches=[dict(name=l[0], grid=[int(g) for g in l[1].split()], threads=int(l[2]), lds=int(l[3])) for l in launches]))
json.dump(out, sys.stdout)
"""


def run(calls, folder):
    shim = os.path.join(str(folder), "launch_log.so")
    if not os.path.exists(shim):
        subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "launch_log.cpp"), "-o", shim])
    done = subprocess.run([sys.executable, "-c", CHILD, shim, os.path.dirname(HERE)], input=json.dumps(calls), stdout=subprocess.PIPE, text=True, check=True)
    return json.loads(done.stdout)


def cache(seqs=1, each=1, heads=1, dim=64, page=16, length=64, type=1, **kw):
    return dict(dict(type=type, kv_heads=heads, head_dim=dim, page_tokens=page, n_pages=4, n_seqs=seqs, n_tokens=seqs * each, max_new=each, max_length=length,
                     table_pages=-(-length // page)), **kw)


@pytest.mark.parametrize("switches", ["", "parts=3", "attention=d,parts=2", "attention=p,parts=6"])
def test_more_sequences_than_the_second_launch_takes(tmp_path, switches):
    """Parts need a launch that joins them, of up to 65535 sequences: more are taken in one part."""
    calls = [dict(entry="attention", switches=switches, q_heads=1, cache=cache(seqs=seqs, length=32768)) for seqs in (65535, 65536, 65537, 200000)]
    for call, answer in zip(calls, run(calls, tmp_path)):
        many = call["cache"]["n_seqs"] > 65535
        assert answer["status"] == 0, (call, answer)
        assert (answer["asked"] == 0) or not many, (call, answer)
        assert len(answer["launches"]) == (2 if answer["asked"] else 1)


def test_calls_are_launched_whole_or_not_at_all(tmp_path):
    rng = random.Random(1)

    def size(high):
        return int(2 ** rng.uniform(0, high))
    calls = []
    for _ in range(3000):
        entry = rng.choice(["append", "attention", "attention"])
        heads, group, seqs, each = size(6), size(8), size(rng.choice([4, 10, 22])), size(rng.choice([1, 4, 12, 24]))
        seqs = min(seqs, (1 << 30) // each)
        calls.append(dict(entry=entry, switches=rng.choice(["", "", "parts=%d" % rng.randint(0, 6), "attention=d", "attention=p", "attention=p,parts=4"]),
                          q_heads=heads * group, window=rng.choice([0, 0, size(12)]),
                          cache=cache(seqs, each, heads, 16 * rng.randint(1, 16), 1 << rng.randint(4, 8), size(rng.choice([6, 12, 20])), rng.randint(0, 1))))
    refused = 0
    for call, answer in zip(calls, run(calls, tmp_path)):
        if answer["status"] != 0:
            refused += 1
            assert not answer["launches"], (call, answer)
            continue
        assert answer["launches"], call
        for launch in answer["launches"]:
            x, y, z = launch["grid"]
            assert 1 <= x and x * launch["threads"] < 2 ** 32 and 1 <= y <= 65535 and 1 <= z <= 65535 and launch["lds"] <= 160 * 1024, (call, launch)
            assert launch["threads"] <= 1024
    assert 0 < refused < len(calls) // 2


def test_more_tokens_than_places(tmp_path):
    """Numbers of new tokens whose pages cannot be counted in 32 bits, and places before a sequence's first that cannot."""
    calls = [dict(entry=entry, q_heads=1, cache=cache(1, each, 1, 16, 256, 64, starts=starts)) for entry in ("append", "attention") for starts in (False, True)
             for each in (2 ** 30 + 1, 2 ** 31 - 300, 2 ** 31 - 1)]
    for call, answer in zip(calls, run(calls, tmp_path)):
        assert answer["status"] == -2 and not answer["launches"] and not answer["asked"], (call, answer)
