"""A call of matrices of several kinds when the process has no host memory left for the library: the entry points are C, so nothing is
thrown through them, and the step is taken without what there was no memory for."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

NEW = """#include <cstdlib>
#include <cstring>
#include <dlfcn.h>
#include <new>
// operator new that fails for the library alone (the runtime below it has failures of its own)
static int fail = 0, failed = 0;
extern "C" void set_fail(int on) { fail = on; }
extern "C" int failures() { return failed; }
static void *take(std::size_t n, void *from)
{
    Dl_info info;
    if (fail && dladdr(from, &info) && info.dli_fname && std::strstr(info.dli_fname, "libxconv")) {
        ++failed;
        return nullptr;
    }
    return std::malloc(n ? n : 1);
}
void *operator new(std::size_t n) { void *p = take(n, __builtin_return_address(0)); if (!p) throw std::bad_alloc(); return p; }
void *operator new(std::size_t n, const std::nothrow_t &) noexcept { return take(n, __builtin_return_address(0)); }
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, std::size_t) noexcept { std::free(p); }
void operator delete(void *p, const std::nothrow_t &) noexcept { std::free(p); }
"""
CODE = """
import ctypes, sys
new = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
import torch
from paper_2106_06998_amd import binding as xb
gen = torch.Generator().manual_seed(1)
gs = [torch.randn(*s, generator=gen).cuda() for s in ((64, 100), (130, 200), (300, 900))]      # one workgroup, single steps, groups
args = xb.make_orth_args()
outs = [[torch.zeros_like(g) for g in gs] for _ in range(3)]
lists = [xb.make_orth_items([(*g.shape, g, o, None) for g, o in zip(gs, out)]) for out in outs]
ws = xb.alloc_bytes(xb.xconv_orth_workspace_bytes(lists[0], 3, args))
torch.cuda.synchronize()
print("calls", flush=True)
new.set_fail(1)
xb.xconv_orth(lists[0], 3, args, ws)
torch.cuda.synchronize()
new.set_fail(0)
assert new.failures() > 0
for items in lists[1:]:
    xb.xconv_orth(items, 3, args, ws)
    new.set_fail(1)                 # (what the second call takes is put back without memory)
    torch.cuda.synchronize()
new.set_fail(0)
for out in outs[1:]:
    assert all(torch.equal(a, b) and bool(a.any()) for a, b in zip(outs[0], out))
print("the same three times")
"""


def test_several_kinds_without_host_memory(tmp_path):
    src, so = tmp_path / "new.cpp", str(tmp_path / "new.so")
    src.write_text(NEW)
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", str(src), "-o", so, "-ldl"], check=True)
    print("[gpu-case] xconv_orth, three kinds, without host memory", flush=True)
    p = subprocess.run([sys.executable, "-c", CODE, so], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True, timeout=110)
    assert p.returncode == 0 and "the same three times" in p.stdout, (p.returncode, p.stdout)
