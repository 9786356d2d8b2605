"""What vq_attention_shared, vq_embed and vq_sample launch, on a machine without a GPU (launch_log.cpp in place of the HIP runtime): all of a call or, where it is
refused, nothing, and grids of sizes that a launch can have."""
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
at = 1 << 41
for call in json.load(sys.stdin):
    libc.setenv(b"VQ_SWITCHES", call.get("switches", "").encode(), 1)
    log.launch_log_clear()
    asked = None
    if call["entry"] == "embed":
        rc = vq.vq_embed(at, call["rows"], at, call["width"], call["vocabulary"], call["width"], 1.0, call["stream32"], at, call["width"])
    elif call["entry"] == "sample":
        rc = vq.vq_sample(at, call["vocabulary"], call["rows"], call["vocabulary"], at, vq.vq_sampling(struct_size=ctypes.sizeof(vq.vq_sampling), temperature=1.0, top_p=0.9), at)
    else:
        d, q_heads = call["cache"], call["q_heads"]
        page = d["kv_heads"] * d["page_tokens"] * d["head_dim"]
        cache = vq.vq_kv_desc(**d, struct_size=ctypes.sizeof(vq.vq_kv_desc), k_pages=at, v_pages=at, k_scales=at, v_scales=at, page_table=at, lengths=at, reserved=0,
                              table_stride=d["table_pages"], k_page_stride=page, v_page_stride=page)
        x = vq.vq_prefix_desc(**call["prefix"], struct_size=ctypes.sizeof(vq.vq_prefix_desc), page_table=at, lengths=at, members=at, table_stride=call["prefix"]["table_pages"])
        width = q_heads * d["head_dim"]
        asked = vq.vq_attention_shared_workspace_bytes(cache, x, q_heads)
        rc = vq.vq_attention_shared(cache, x, at, width, q_heads, 0.1, at, width, None, at, asked if call.get("room", True) else 0)
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


def shared(seqs=1, each=1, heads=1, group=1, dim=64, page=16, length=4096, prefixes=1, members=None, prefix_length=2048, own=64, type=1, **kw):
    entries = -(-length // page)
    return dict(entry="shared", q_heads=heads * group,
                cache=dict(type=type, kv_heads=heads, head_dim=dim, page_tokens=page, n_pages=4, n_seqs=seqs, n_tokens=seqs * each, max_new=each, max_length=length, table_pages=entries),
                prefix=dict(n_prefixes=prefixes, max_members=members or seqs, max_length=prefix_length, max_own=own, table_pages=-(-prefix_length // page)), **kw)


def check_grids(call, answer):
    assert answer["launches"], call
    for launch in answer["launches"]:
        x, y, z = launch["grid"]
        assert 1 <= x and x * launch["threads"] < 2 ** 32 and 1 <= y <= 65535 and 1 <= z <= 65535 and launch["lds"] <= 160 * 1024, (call, launch)
        assert launch["threads"] <= 1024


@pytest.mark.parametrize("switches,launches", [("", 2), ("shared=1", 2), ("shared=2", 3), ("shared=1,prefix=p,prefix_parts=5,parts=2", 2), ("shared=2,attention=p,parts=6", 3)])
def test_a_prefix_is_computed_by_itself(tmp_path, switches, launches):
    call = shared(seqs=64, heads=8, group=8, dim=128, length=9216, prefix_length=8192, own=1024, switches=switches)
    answer, = run([call], tmp_path)
    assert answer["status"] == 0 and answer["asked"] > 0 and len(answer["launches"]) == launches, answer
    check_grids(call, answer)


@pytest.mark.parametrize("call", [
    shared(seqs=65536, switches="shared=1"), shared(seqs=64, prefix_length=0, switches="shared=1"), shared(seqs=64, heads=8, group=8, dim=128, room=False),
    shared(seqs=1024, each=256, group=64, switches="shared=1"), shared(seqs=2, each=1 << 25, length=1 << 25, dim=256, switches="shared=1"), shared(seqs=64, switches="shared=0"),
    shared(seqs=1, each=1 << 24, heads=64, dim=256, length=1 << 24, prefixes=65535, prefix_length=1 << 20, switches="shared=1"),
], ids=lambda c: "%d by %d" % (c["cache"]["n_seqs"], c["cache"]["max_new"]))
def test_what_is_not_shared_is_plain_attention(tmp_path, call):
    """More sequences than the launch that joins takes, no prefix, no workspace, more rows than a grid has threads for, partial results of more bytes than 64 bits count."""
    answer, = run([call], tmp_path)
    assert answer["status"] == 0
    assert not any("halves" in launch["name"] for launch in answer["launches"]), answer
    check_grids(call, answer)


def test_calls_are_launched_whole_or_not_at_all(tmp_path):
    rng = random.Random(2)

    def size(high):
        return int(2 ** rng.uniform(0, high))
    calls = []
    for _ in range(3000):
        heads, group, seqs, each = size(6), size(8), size(rng.choice([4, 10, 17])), size(rng.choice([1, 4, 12, 24]))
        seqs = min(seqs, (1 << 30) // each)
        length = size(rng.choice([6, 12, 20]))
        calls.append(shared(seqs, each, heads, group, 16 * rng.randint(1, 16), 1 << rng.randint(4, 8), length, size(rng.choice([2, 2, 15])), size(rng.choice([3, 10, 31])), rng.randint(0, length),
                            rng.randint(0, length), rng.randint(0, 1),
                            switches=rng.choice(["", "", "shared=1", "shared=2", "shared=1,prefix=d,prefix_parts=%d" % rng.randint(0, 5), "shared=1,prefix=p,parts=%d" % rng.randint(0, 6),
                                                 "shared=2,attention=d,parts=%d" % rng.randint(0, 6), "shared=2,attention=p"])))
    refused = halves = 0
    for call, answer in zip(calls, run(calls, tmp_path)):
        if answer["status"] != 0:
            refused += 1
            assert not answer["launches"], (call, answer)
            continue
        check_grids(call, answer)
        halves += any("halves" in launch["name"] for launch in answer["launches"])
    assert 0 < refused < len(calls) // 2 and halves > len(calls) // 10, (refused, halves)


@pytest.mark.parametrize("vocabulary", [1, 32768, 32769, 131072, 131073, 1 << 24])
def test_rows_of_logits(tmp_path, vocabulary):
    calls = [dict(entry="sample", rows=rows, vocabulary=vocabulary) for rows in (1, 65536, (1 << 21) + 1, (1 << 31) - 1)]
    for call, answer in zip(calls, run(calls, tmp_path)):
        assert answer["status"] == 0
        check_grids(call, answer)
        assert sum(launch["grid"][0] for launch in answer["launches"]) == call["rows"]
        assert len(answer["launches"]) == -(-call["rows"] // (1 << 21))


@pytest.mark.parametrize("width", [1, 7, 8, 768, 1 << 24])
def test_rows_of_a_table(tmp_path, width):
    calls = [dict(entry="embed", rows=rows, vocabulary=32000, width=width, stream32=stream32) for rows in (1, 65536, (1 << 31) - 1) for stream32 in (0, 1)]
    for call, answer in zip(calls, run(calls, tmp_path)):
        assert answer["status"] == 0
        check_grids(call, answer)


def test_as_many_sequences_prefixes_and_key_heads_as_there_may_be(tmp_path):
    calls = [shared(seqs=seqs, heads=65535, prefixes=prefixes, switches=switches) for seqs, prefixes in ((65535, 65535), (65535, 1), (2, 65535)) for switches in ("", "shared=1", "shared=1,prefix=p")]
    for call, answer in zip(calls, run(calls, tmp_path)):
        assert answer["status"] == 0 and not any("halves_kernel<true, 64" in launch["name"] for launch in answer["launches"]), answer
        check_grids(call, answer)


@pytest.mark.parametrize("prefixes,members,length,own", [(2, 30, 8192, 300), (3, 8, 2048, 50), (10, 12, 4096, 104), (32, 8, 2048, 100)])
def test_sequences_of_a_prefix_without_a_bound(tmp_path, prefixes, members, length, own):
    """Each prefix may have all of the call's sequences: they are computed once all the same, and their partial results take no more room than the call's rows."""
    layout = dict(seqs=prefixes * members, heads=8, group=8, dim=128, length=length + own, prefixes=prefixes, prefix_length=length, own=own)
    free, bound, free_in_parts, bound_in_parts = run([shared(**layout, members=m, switches=s) for s in ("", "shared=1,prefix=d,prefix_parts=2,parts=0") for m in (None, members)], tmp_path)
    assert all(len(a["launches"]) == 2 and "halves" in a["launches"][0]["name"] for a in (free, bound)), (free, bound)
    assert free_in_parts["asked"] == bound_in_parts["asked"] > 0
