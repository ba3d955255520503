"""What the entry points tell the runtime, without a GPU: a child process loads a stand-in for the runtime's launch functions,
which notes the calls, before the library."""
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = pytest.importorskip("paper_2606_12876_amd", reason="libaqmb.so not built")

STAND_IN = r"""
#include <stddef.h>
#include <stdint.h>
typedef struct { uint32_t x, y, z; } dim3;
typedef struct { uint64_t kernel, kind, a, b; } note;      /* kind 0: LDS limit a; 1: launch of a threads with b bytes of LDS */
note notes[4096];
int n_notes;
static dim3 grid, block;
static size_t lds;
static void* stream;
static void put(const void* k, int kind, uint64_t a, uint64_t b) {
  if (n_notes < 4096) notes[n_notes++] = (note){(uint64_t)k, kind, a, b};
}
int hipFuncSetAttribute(const void* f, int attribute, int value) { put(f, 0, value, attribute); return 0; }
int __hipPushCallConfiguration(dim3 g, dim3 b, size_t s, void* st) { grid = g; block = b; lds = s; stream = st; return 0; }
int __hipPopCallConfiguration(dim3* g, dim3* b, size_t* s, void** st) { *g = grid; *b = block; *s = lds; *st = stream; return 0; }
int hipLaunchKernel(const void* f, dim3 g, dim3 b, void** args, size_t s, void* st) {
  put(f, 1, (uint64_t)g.x * b.x * g.y * b.y * g.z * b.z, s);
  return 0;
}
int hipGetLastError(void) { return 0; }
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipDeviceGetAttribute(int* v, int attribute, int device) { *v = 256; return 0; }
"""

CHILD = r"""
import ctypes, json, sys
stand_in = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
import paper_2606_12876_amd as A
got = []
for call in json.loads(sys.argv[2]):
    n = ctypes.c_int.in_dll(stand_in, "n_notes")
    first = n.value
    if call["op"] == "adapters":
        d = A.AdaptersDesc(16, 16, None, None, call["dt"], 4, call["rank"], 64, call["d_out"])
        status = A.lib.aqmb_adapters_add(ctypes.byref(d), 16, 64, 16, call["rows"], 16, call["d_out"], 1 << 30, call["d_out"], call["y"], 16,
                                         1 << 40, None)
    else:
        c = A.KVCacheDesc(16, 16, None, None, call["page"] * call["dim"], call["dt"], 0, 4096, call["page"], 1, call["dim"])
        status = A.lib.aqmb_paged_attention(ctypes.byref(c), 16, call["dt"], call["heads"] * call["dim"], call["heads"], 16, 1 << 20, 16, call["seqs"],
                                            call["length"], 1.0, 0, 16, call["heads"] * call["dim"], None, 16, 1 << 40, None)
    notes = (ctypes.c_uint64 * (4 * 4096)).in_dll(stand_in, "notes")
    got.append([status, [list(notes[4 * i:4 * i + 4]) for i in range(first, n.value)]])
print(json.dumps(got))
"""


@pytest.fixture(scope="module")
def notes_of(tmp_path_factory):
    """calls -> for each (status, notes)."""
    d = tmp_path_factory.mktemp("stand_in")
    (d / "s.c").write_text(STAND_IN)
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-w", "-o", str(d / "s.so"), str(d / "s.c")], check=True)

    def run(calls):
        r = subprocess.run([sys.executable, "-W", "ignore", "-c", CHILD, str(d / "s.so"), json.dumps(calls)], cwd=ROOT, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        got = json.loads(r.stdout)
        assert len(got) == len(calls) and all(status == 0 and notes for status, notes in got), got
        return got

    return run


def check_limits(got):
    """A kernel's limit on LDS is one for all threads of a program, and the last one set may be another call's: so no call
    may set less than the largest launch of the same kernel needs."""
    limits, most = {}, {}
    for _, notes in got:
        for kernel, kind, a, b in notes:
            if kind == 0:
                limits.setdefault(kernel, []).append(a)
            else:
                most[kernel] = max(most.get(kernel, 0), b)
                assert b <= 65536 - 256 or kernel in limits, "a launch above 64 KiB without a limit"
    above = {k: most[k] for k in limits}
    assert above and all(min(v) >= above[k] for k, v in limits.items()), (limits, above)
    assert max(max(v) for v in limits.values()) < 163840
    return above


def test_adapters_of_every_rank_set_one_limit(notes_of):
    calls = [dict(op="adapters", dt=dt, y=y, rank=rank, rows=300, d_out=d_out)
             for dt in (0, 1) for y in (0, 1, 2) for d_out in (64, 63) for rank in (160, 256, 8, 192, 224, 161)]
    assert set(check_limits(notes_of(calls)).values()) == {82944, 115712}


def test_attention_of_every_size_sets_one_limit(notes_of):
    calls = [dict(op="attention", dt=dt, dim=dim, heads=heads, page=page, seqs=seqs, length=length)
             for dt in (0, 1) for dim in (256, 248, 232) for heads in (16, 15) for page, seqs, length in
             ((8, 2, 256), (1, 2048, 36000), (1, 4000, 20000), (1, 1, 256))]
    check_limits(notes_of(calls))
