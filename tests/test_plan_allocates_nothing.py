"""Planning a contraction allocates nothing: a C++ exception must not leave a C entry point, and where memory has run out an allocation would throw
one.  A child process replaces `operator new` by one that throws while the plans are made."""
import os
import subprocess
import sys

from paper_1810_00952_b200 import binding as B

SOURCE = r'''
#include <cstdlib>
#include <new>
static bool failing = false;
extern "C" void fail_allocations(int on) { failing = on; }
void *operator new(std::size_t n) { if (failing) throw std::bad_alloc(); void *p = std::malloc(n ? n : 1); if (!p) throw std::bad_alloc(); return p; }
void *operator new(std::size_t n, const std::nothrow_t &) noexcept { return failing ? nullptr : std::malloc(n ? n : 1); }
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, std::size_t) noexcept { std::free(p); }
'''
CHILD = r'''
import ctypes, sys
own, lib = ctypes.CDLL(sys.argv[1]), ctypes.CDLL(sys.argv[2])
plan = lib.relay_debug_plan_units
plan.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int32, ctypes.c_void_p, ctypes.c_int32]
units = (ctypes.c_uint32 * 4096)()
for M, N, K in ((4096, 4096, 4096), (8192, 4096, 1024), (300, 40000, 64), (256, 128, 64), (65536, 65536, 64)):
    own.fail_allocations(1)
    n = plan(M, N, K, 148, units, 4096)
    own.fail_allocations(0)
    assert n > 0 or (n == -1 and M == 65536), (M, N, K, n)
print("planned")
'''


def test_plans_are_made_without_memory(tmp_path):
    src, so = tmp_path / "fail.cc", tmp_path / "libfail.so"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-shared", "-fPIC", "-o", str(so), str(src)], check=True)
    r = subprocess.run([sys.executable, "-c", CHILD, str(so), B.LIB_PATH], env=dict(os.environ, LD_PRELOAD=str(so)), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "planned" in r.stdout, r.stdout + r.stderr
