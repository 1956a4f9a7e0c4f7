"""Which launches rk_prefix_attn makes (no GPU needed): its grid holds every (sequence, KV head) that the chosen form has to go over.

A small library with the runtime's launch function is loaded ahead of the library under test, which then calls it instead: it notes the kernel's name, the
grid and the two counts that prefix_kernel is given.  Nothing runs and no pointer is followed.
"""
import json
import os
import re
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

NOTED = r"""
#include <cstdint>
#include <cstdio>
#include <map>
#include <string>
struct Dim { uint32_t x, y, z; };
static std::map<const void*, std::string>& names() { static std::map<const void*, std::string> m; return m; }
static std::string said;
static struct { Dim g, b; size_t shared; void* stream; } set;
extern "C" {
int __hipPushCallConfiguration(Dim g, Dim b, size_t shared, void* stream) { set = {g, b, shared, stream}; return 0; }
int __hipPopCallConfiguration(Dim* g, Dim* b, size_t* shared, void** stream) { *g = set.g; *b = set.b; *shared = set.shared; *stream = set.stream; return 0; }
void __hipRegisterFunction(void**, const void* f, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names()[f] = name; }
int hipLaunchKernel(const void* f, Dim g, Dim b, void** args, size_t, void*) {
    const std::string& n = names()[f];
    const bool prefix = n.find("prefix_kernel") != std::string::npos;
    char s[1024];
    snprintf(s, sizeof s, "%s %u %u %u %u %d %d\n", n.c_str(), g.x, g.y, g.z, b.x * b.y * b.z, prefix ? *(int32_t*)args[2] : 0, prefix ? *(int32_t*)args[3] : 0);
    said += s;
    return 0;
}
int hipGetLastError() { return 0; }
const char* launches() { static std::string out; out.swap(said); said.clear(); return out.c_str(); }
}
"""

CALLS = r"""
import ctypes as C, json, sys
noted = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
noted.launches.restype = C.c_char_p
lib = C.CDLL(sys.argv[2])
class Geom(C.Structure):
    _fields_ = [("batch", C.c_int32), ("hq", C.c_int32), ("hkv", C.c_int32), ("dim", C.c_int32), ("scale", C.c_float)]
class Pages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_min", C.c_void_p), ("k_max", C.c_void_p), ("stride_p", C.c_int64), ("stride_h", C.c_int64),
                ("n_pages", C.c_int32), ("page", C.c_int32)]
P, I32, I64, SZ = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
lib.rk_prefix_workspace_bytes.argtypes, lib.rk_prefix_workspace_bytes.restype = [P, I32, I32, I32], SZ
lib.rk_prefix_attn.argtypes = [P, P, I64, I64, I32, P, P, I32, P, I32, P, I32, P, P, I32, P, P, P, P, I32, P, SZ, P]
F = 0x10000
out = []
for B, Hq, H, T, prefix, own in json.load(sys.stdin):
    g, pages = Geom(B, Hq, H, 128, 0.1), Pages(F, F, None, None, H * 16 * 128, 16 * 128, 1000, 16)
    rows = lambda n: (n + 15) // 16
    rc = lib.rk_prefix_attn(C.byref(g), F, T * Hq * 128, Hq * 128, T, C.byref(pages), F, rows(prefix), F, prefix, F, rows(prefix + own), F, None, own, None, F, None, None, 0,
                            0x100000, lib.rk_prefix_workspace_bytes(C.byref(g), T, prefix, own), None)
    out.append([rc, [l.split() for l in noted.launches().decode().splitlines()]])
print(json.dumps(out))
"""

# batch, query heads, KV heads, new tokens, rows of the prefix, rows behind it
CASES = [(b, hq, h, t, p, o)
         for b, hq, h in [(1, 1, 1), (1, 32, 8), (2, 8, 2), (4, 28, 4), (5, 64, 64), (9, 29, 29), (16, 32, 32), (16, 16, 16), (8, 64, 32), (2, 512, 512), (3, 300, 100), (16, 64, 64),
                          (17, 32, 32), (64, 32, 8), (80, 16, 8), (129, 2, 2), (300, 3, 1), (257, 1, 1), (1, 257, 257)]
         for t in (1, 2, 3, 5, 17, 100) for p, o in ((1, 1), (600, 300), (8192, 500), (300, 9000))]


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    import paper_2411_05787_amd as rk
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("noted")
    (d / "noted.cpp").write_text(NOTED)
    r = subprocess.run([cxx, "-O1", "-shared", "-fPIC", str(d / "noted.cpp"), "-o", str(d / "noted.so")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([sys.executable, "-c", CALLS, str(d / "noted.so"), rk.LIB_PATH], input=json.dumps(CASES), capture_output=True, text=True, timeout=120, cwd=ROOT)
    assert r.returncode == 0, r.stderr[-2000:]
    return dict(zip(CASES, json.loads(r.stdout)))


@pytest.mark.parametrize("form", ["columns", "one_pair", "two_pairs", "tiles"])
def test_every_pair_has_a_workgroup(launches, form):
    """prefix_kernel<cap, slope, ALL_COLS, OWN>: behind the shared workgroups, each takes 4 / OWN pairs and parts (OWN = 0: one)."""
    seen = 0
    for case, (rc, said) in launches.items():
        B, Hq, H, T, _, _ = case
        assert rc == 0 and len(said) == 2 and "paged_merge_kernel" in said[1][0], (case, rc, said)
        name, x, y, z, threads, shared, parts = said[0][0], *map(int, said[0][1:])
        m = re.search(r"prefix_kernelILi\d+ELb[01]ELb([01])ELi(\d)EE", name)
        assert m and (y, z, threads) == (1, 1, 256), (case, said[0])
        all_cols, own = m.group(1) == "1", int(m.group(2))
        per = 1 if own == 0 else 4 // own
        if form != ("columns" if all_cols else {0: "tiles", 4: "one_pair", 2: "two_pairs"}[own]):
            continue
        seen += 1
        assert all_cols == (B * T * (Hq // H) <= 16), case
        assert shared >= H and parts >= B * H and parts % (B * H) == 0, (case, shared, parts)
        assert per * (x - shared) >= parts and per * (x - shared - 1) < parts, (case, name, x, shared, parts)
    assert seen
