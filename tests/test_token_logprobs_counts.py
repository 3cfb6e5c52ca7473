"""The counts of finished parts that essa_token_logprobs keeps in its context: where clearing them fails, the call fails, and the next one starts again.  On the CPU: a library
in front of HIP's gives host memory and says when its calls fail; nothing is launched."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2507_04453_amd", "libessa.so")

HIP = r"""
#include <stdlib.h>
#include <string.h>
int fail_memset, memsets, mallocs, frees, launches;
int hipSetDevice(int d) { return 0; }
int hipStreamSynchronize(void* s) { return 0; }
int hipGetLastError(void) { return 0; }
int hipMalloc(void** p, size_t n) { ++mallocs; *p = malloc(n); memset(*p, 0x5a, n); return 0; }
int hipFree(void* p) { ++frees; free(p); return 0; }
int hipMemsetAsync(void* p, int v, size_t n, void* s) { ++memsets; if (fail_memset) return 719; memset(p, v, n); return 0; }
int hipLaunchKernel(const void* f, unsigned long long g0, unsigned g1, unsigned long long b0, unsigned b1, void** a, size_t l, void* s) { ++launches; return 0; }
int __hipPushCallConfiguration(unsigned long long g0, unsigned g1, unsigned long long b0, unsigned b1, size_t l, void* s) { return 0; }
int __hipPopCallConfiguration(void* g, void* b, size_t* l, void** s) { *l = 0; *s = 0; return 0; }
"""

PROGRAM = r"""
import ctypes as C, sys
hip = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)                  # in front of the HIP library: its names are found first
lib = C.CDLL(sys.argv[2])
n = lambda name: C.c_int.in_dll(hip, name)
ctx = C.create_string_buffer(4096)                             # a context of zeros: device 0, no scratch, no counts
arg = lambda: (C.cast(ctx, C.c_void_p), C.c_void_p(256), C.c_int64(100000), 1, 3, 100000, C.c_float(1.0), C.c_void_p(256), 1, C.c_void_p(256), None, 0, None, None)
n("fail_memset").value = 1
codes = [lib.essa_token_logprobs(*arg()), lib.essa_token_logprobs(*arg())]
failed = (n("memsets").value, n("launches").value, n("mallocs").value - n("frees").value)
n("fail_memset").value = 0
codes += [lib.essa_token_logprobs(*arg()), lib.essa_token_logprobs(*arg())]
print(*codes, *failed, n("memsets").value, n("launches").value)
"""


def test_counts_that_could_not_be_cleared_are_not_kept(tmp_path):
    (tmp_path / "hip.c").write_text(HIP)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(tmp_path / "hip.so"), str(tmp_path / "hip.c")], check=True)
    r = subprocess.run([sys.executable, "-c", PROGRAM, str(tmp_path / "hip.so"), LIB], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr
    first, second, third, fourth, memsets, launches, kept, memsets_after, launches_after = map(int, r.stdout.split())
    assert first != 0 and second != 0 and third == 0 and fourth == 0
    assert (memsets, launches, kept) == (2, 0, 0)              # both tried, nothing was launched, nothing is left
    assert (memsets_after, launches_after) == (3, 2)           # cleared once, then kept
