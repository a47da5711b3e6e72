"""The attention's workspace when memory is short: a call that could have what it needs has it.

A child process loads a small library ahead of the CUDA runtime that answers allocations above a limit as if there were no memory for them."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHIM = r"""
#define _GNU_SOURCE
#include <dlfcn.h>
#include <stddef.h>
static size_t most = ~(size_t)0, largest = 0;
size_t shim_largest(void) { return largest; }
void shim_limit(size_t bytes) { most = bytes; largest = 0; }
int cudaMalloc(void** p, size_t bytes) {
    static int (*real)(void**, size_t);
    if (!real) *(void**)&real = dlsym(dlopen("libcudart.so.12", RTLD_NOW | RTLD_NOLOAD), "cudaMalloc");
    if (bytes > largest) largest = bytes;
    if (bytes > most) return 2; /* cudaErrorMemoryAllocation */
    return real(p, bytes);
}
"""


def test_workspace_when_there_is_no_memory_for_twice_as_much(tmp_path):
    src, so = os.path.join(str(tmp_path), "shim.c"), os.path.join(str(tmp_path), "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-O1", "-o", so, src, "-ldl"])
    r = subprocess.run([sys.executable, os.path.abspath(__file__), so], env=dict(os.environ, LD_PRELOAD=so), cwd=ROOT,
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    assert "fine" in r.stdout


def _run(shim):
    import ctypes as C
    import torch
    from paper_2608_20375_b200 import Graft, GraftError, KVCache
    shim.shim_limit.argtypes, shim.shim_largest.restype = [C.c_size_t], C.c_size_t
    V, B, Hq, Hk, D, page, rows = 50, 4, 8, 2, 64, 16, 64
    gen = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    c = KVCache.alloc(1, 40, Hk, page, D)
    c.k.copy_(rand(*c.k.shape)), c.v.copy_(rand(*c.v.shape))
    table = torch.arange(40, dtype=torch.int32, device="cuda").view(4, 10)
    table[:, :2] = table[:1, :2].clone()
    q = rand(B, rows, Hq, D).to(torch.bfloat16)

    def call(g, rows, shared):
        out = torch.zeros((B, rows, Hq, D), dtype=torch.bfloat16, device="cuda")
        g.tree_attention(c, 0, table, q[:, :rows].contiguous(), i32([60, 50, 40, 90]), i32([rows] * B), None, out, shared=shared)
        torch.cuda.synchronize()
        return out

    small, large = (8, 0), (64, 32)  # (blocks' pieces of 32 rows, then units of 256)
    sizes, want = [], []
    for what in (small, large):
        shim.shim_limit(2 ** 40)
        want.append(call(Graft(V, 4, 4, 16, 8, B, 1, rows - 1, 1, 0.0), *what))
        sizes.append(shim.shim_largest())
    middle = (24, 0)  # less than twice as much as the large one
    g = Graft(V, 4, 4, 16, 8, B, 1, rows - 1, 1, 0.0)
    shim.shim_limit(2 ** 40)
    first = call(g, *middle)
    begun = shim.shim_largest()
    assert sizes[0] < begun < sizes[1] < 2 * begun, (sizes, begun)
    shim.shim_limit(sizes[1])  # enough for the call, not for twice what it had
    assert torch.equal(call(g, *large), want[1]) and torch.equal(call(g, *middle), first) and torch.equal(call(g, *small), want[0])
    g = Graft(V, 4, 4, 16, 8, B, 1, rows - 1, 1, 0.0)
    shim.shim_limit(sizes[1] - 1)
    try:
        call(g, *large)
        raise SystemExit("a workspace that is not to be had was not reported")
    except GraftError as e:
        assert "scratch" in str(e), e
    assert torch.equal(call(g, *small), want[0])


if __name__ == "__main__":
    import ctypes
    sys.path.insert(0, ROOT)
    _run(ctypes.CDLL(sys.argv[1]))
    print("fine")
