"""raise_dynamic_lds (csrc/error.hip) on the CPU: its source compiled for the host only, against stand-ins for the two runtime calls that it makes.  A kernel may be
allowed more later, on every device by itself, and what has been allowed is not asked for again."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "%s/paper_2111_01264_amd/csrc/error.hip"
#include <stdlib.h>
static int device = 0, calls = 0, asked = 0, fails = 0;
extern "C" hipError_t hipGetDevice(int* d) { *d = device; return hipSuccess; }
extern "C" hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int bytes) { ++calls; asked = bytes; return fails ? hipErrorInvalidValue : hipSuccess; }
static char kernel[100];
static void expect(int line, int k, int bytes, int want_calls, hipError_t want = hipSuccess)
{
    calls = 0;
    const hipError_t e = dqn::raise_dynamic_lds(&kernel[k], bytes);
    if (e != want || calls != want_calls || (calls && asked != bytes)) { printf("line %%d: error %%d, %%d calls, %%d bytes\n", line, (int)e, calls, asked); exit(1); }
}
#define EXPECT(...) expect(__LINE__, __VA_ARGS__)
int main()
{
    EXPECT(0, 70000, 1);
    EXPECT(0, 70000, 0);
    EXPECT(0, 65536, 0);    // less than has been allowed
    EXPECT(0, 131072, 1);   // more
    EXPECT(0, 131072, 0);
    EXPECT(0, 70000, 0);
    device = 1;
    EXPECT(0, 70000, 1);
    EXPECT(0, 131072, 1);
    device = 64;            // no device shares another one's entry
    EXPECT(0, 70000, 1);
    device = 0;
    EXPECT(0, 131072, 0);
    fails = 1;
    EXPECT(1, 70000, 1, hipErrorInvalidValue);
    fails = 0;
    EXPECT(1, 70000, 1);    // a refusal is not remembered
    EXPECT(1, 70000, 0);
    for (int k = 2; k < 100; ++k) EXPECT(k, 70000, 1);   // more kernels than are remembered
    EXPECT(99, 131072, 1);
    return 0;
}
"""


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="no compiler")
def test_larger_amounts_other_devices_and_refusals(tmp_path):
    src, exe = tmp_path / "main.hip", tmp_path / "main"
    src.write_text(PROGRAM % ROOT)
    subprocess.run(["hipcc", "--offload-host-only", "-std=c++17", "-O1", str(src), "-o", str(exe)], check=True, capture_output=True, timeout=100)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
