"""The launches of the paged cache's calls, looked at on the CPU: a process that records them instead of
making them (launch_record.cpp).  Every call that its argument checks accept, and that has something to
do, has to launch blocks, and fewer threads than a grid holds."""
import json
import os
import shutil
import subprocess
import sys

import pytest

from conftest import ROOT

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")

CHILD = """
import ctypes, json, sys
record = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)  # its symbols come before the runtime's
record.recorded_launch.restype = ctypes.c_char_p
from paper_2607_09686_amd import moecache as mc
L, P = mc.lib(), 1 << 12  # pointers: never followed
for line in sys.stdin:
    case = json.loads(line)
    held, norm, q, prefix = (case.pop(n, 0) for n in ("held", "norm", "q", "prefix"))
    base = dict(dtype=mc.MOE_BF16, n_heads=8, n_kv_heads=2, head_dim=128, page_tokens=16, n_pages=4, max_pages=2, n_seqs=1,
                n_tokens=1, pad=0, keys=P, values=P, pages=P, starts=P, lengths=P, status=None, hip_stream=None)
    b = mc.KvBatch(**dict(base, **case))
    s = mc.KvScales(P, P) if held else None
    n = mc.KvNorm(P if norm and q else None, P if norm else None, mc.MOE_F32, 1e-6) if norm else None
    f = mc.KvPrefix(P, P, prefix, 0) if prefix else None
    rows, kv_rows, size = b.n_heads * b.head_dim, b.n_kv_heads * b.head_dim, ctypes.c_uint64()
    out = {}
    qs = (P, rows, P, rows) if q else (None, 0, None, 0)
    def call(name, fn, *args):
        record.forget()
        rc = fn(*args)
        assert rc == 0, (name, rc, L.moe_last_error())
        found = []
        for i in range(record.recorded()):
            e = (ctypes.c_uint32 * 6)()
            found.append([record.recorded_launch(i, e).decode(), list(e)])
        out[name] = found
    call("append", L.moe_kv_append_ext, b, s, None, n, b.dtype, P, kv_rows, P, kv_rows, *qs)
    call("read", L.moe_kv_read, b, s, P, kv_rows, P, kv_rows)
    assert L.moe_kv_attend_ext_workspace(b, s, f, size) == 0
    call("attend", L.moe_kv_attend_ext, b, s, f, 0, 0.1, P, rows, P, rows, P, size.value)
    print(json.dumps(out), flush=True)
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """Of a list of cases, each call's launches: [name, [grid x, y, z, block x, y, z]]."""
    from paper_2607_09686_amd import build, moecache
    if not os.path.exists(moecache.LIB_PATH):
        build.build()
    so = tmp_path_factory.mktemp("record") / "librecord.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", os.path.join(ROOT, "tests", "launch_record.cpp"), "-o", str(so)],
                   check=True)

    def run(cases):
        r = subprocess.run([sys.executable, "-c", CHILD, str(so)], input="\n".join(map(json.dumps, cases)), capture_output=True,
                           text=True, cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT), timeout=120)
        assert r.returncode == 0, r.stderr
        found = [json.loads(line) for line in r.stdout.splitlines()]
        assert len(found) == len(cases)
        return found
    return run


KINDS = {"append": "append", "read": "read_kernel", "attend": "_kernel"}


def test_every_call_launches_blocks(launches):
    cases = [dict(head_dim=dim, n_kv_heads=kv, n_heads=kv * group, n_seqs=seqs, n_tokens=new, held=held, norm=norm, q=q,
                  prefix=prefix)
             for dim in (64, 128, 256) for kv, group in ((1, 1), (1, 16), (2, 1), (3, 4), (7, 1), (64, 16))
             for seqs, new in ((1, 1), (1, 4000), (5, 9), (70, 70), (300, 20000))
             for held, norm, q, prefix in ((0, 0, 0, 0), (0, 1, 0, 0), (0, 1, 1, 3), (1, 0, 0, 0), (1, 1, 0, 3), (1, 1, 1, 0))]
    for case, calls in zip(cases, launches(cases)):
        for call, found in calls.items():
            assert found and any(KINDS[call] in name for name, _ in found), (case, call)
            for name, extents in found:
                assert min(extents) >= 1, (case, call, name, extents)


LARGEST = [dict(n_tokens=1 << 24, n_heads=8, n_kv_heads=8, n_seqs=65536), dict(n_tokens=1 << 17, n_heads=1024, n_kv_heads=1),
           dict(n_tokens=1 << 17, n_heads=1024, n_kv_heads=64, n_seqs=65536),
           dict(n_tokens=1 << 16, n_heads=1024, n_kv_heads=64, n_seqs=65536), dict(n_tokens=1 << 12, n_heads=1024, n_kv_heads=1024),
           dict(n_tokens=1 << 12, n_heads=1024, n_kv_heads=1024, n_seqs=4096),
           dict(n_tokens=1 << 16, n_heads=64, n_kv_heads=64, n_seqs=65536), dict(n_tokens=1 << 24, n_heads=1, n_kv_heads=1)]


def test_a_grid_holds_fewer_than_2_to_the_32_threads(launches):
    """Of the largest batches that the argument checks accept, over short and long tables and prefixes."""
    cases = [dict(head_dim=dim, max_pages=pages, held=held, prefix=prefix, norm=1, q=1, **kw)
             for kw in LARGEST for dim in (64, 256) for pages in (2, 1 << 26) for held in (0, 1) for prefix in (0, 2, 1 << 26)]
    for case, calls in zip(cases, launches(cases)):
        for found in calls.values():
            for name, (x, y, z, *block) in found:
                assert x * y * z * block[0] * block[1] * block[2] < 1 << 32, (case, name, (x, y, z))
