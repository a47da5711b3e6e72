"""Launches of the verifier's calls that fail on the host: the call says so, nothing of it is left for the next launch, and the next calls are right.

No kernel goes wrong here.  A child process loads a small library ahead of the CUDA runtime that answers one call of cudaLaunchKernelExC with
an error instead of handing it on, and leaves CUDA's last error set, as a launch that failed does (by asking for a device that is not there)."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SHIM = r"""
#define _GNU_SOURCE
#include <dlfcn.h>
static int wanted = 0, calls = 0;
static void* cudart(const char* name) { return dlsym(dlopen("libcudart.so.12", RTLD_NOW | RTLD_NOLOAD), name); }
int shim_calls(void) { return calls; }
void shim_fail(int nth) { wanted = nth; calls = 0; }  /* the nth call from here on; 0: none */
int cudaLaunchKernelExC(const void* config, const void* func, void** args) {
    static int (*real)(const void*, const void*, void**);
    if (!real) *(void**)&real = cudart("cudaLaunchKernelExC");
    if (++calls == wanted) {
        int (*set_device)(int);
        *(void**)&set_device = cudart("cudaSetDevice");
        return set_device(100000); /* cudaErrorInvalidDevice, and the last error */
    }
    return real(config, func, args);
}
"""


@pytest.mark.parametrize("call", ["write", "read", "keep", "keep in place", "attention", "few rows", "shared", "verify"])
def test_calls_after_a_launch_that_failed(tmp_path, call):
    src, so = os.path.join(str(tmp_path), "shim.c"), os.path.join(str(tmp_path), "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-O1", "-o", so, src, "-ldl"])
    r = subprocess.run([sys.executable, os.path.abspath(__file__), call, so], env=dict(os.environ, LD_PRELOAD=so), cwd=ROOT,
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    assert "fine" in r.stdout


def _run(call, shim):
    import torch
    from paper_2608_20375_b200 import Graft, GraftError, KVCache, TreeOut
    B, V, L, Hq, Hk, D, page, rows = 3, 500, 4, 8, 2, 64, 16, 9
    gen = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    g = Graft(V, L, 4, 16, 8, B, 1, rows - 1, 1, 0.0)
    c = KVCache.alloc(2, B * 20, Hk, page, D)
    c.k.copy_(rand(*c.k.shape)), c.v.copy_(rand(*c.v.shape))
    table = torch.arange(B * 20, dtype=torch.int32, device="cuda").view(B, 20)
    if call == "shared":
        table[:, :4] = table[:1, :4].clone()
    lens, count = i32([200, 90, 300]), i32([9, 4, 1])
    q, key, value = (rand(B, rows, h, D).to(torch.bfloat16) for h in (Hq, Hk, Hk))
    one = q[:, :1].contiguous()
    tree = TreeOut(count, None, i32([list(range(rows))] * B), i32([[-1, 0, 0, 1, 1, 2, 3, 3, 4]] * B), None, None, None, None, None)
    z, u = rand(B, rows, V), torch.rand((B, rows), generator=gen, device="cuda")
    z[:, :, :rows] += 8.0
    cache0 = c.k.clone(), c.v.clone()

    def step():
        c.k.copy_(cache0[0]), c.v.copy_(cache0[1])
        o, nxt = torch.zeros_like(q), lens.clone()
        outs = [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((B,), (B, L), (B,))]
        path, zeros = i32([[2, 4, 5, 7]] * B), torch.zeros_like(lens)
        torch.cuda.synchronize()
        shim.shim_fail(armed)
        {"write": lambda: g.cache_write(c, 1, table, lens, count, key, value),
         "read": lambda: g.cache_read(c, 1, table, lens, count, o[:, :, :Hk].contiguous(), o[:, :, Hk:2 * Hk].contiguous()),
         "keep": lambda: g.cache_keep(c, table, lens, count.clamp(max=L), path, zeros),
         "keep in place": lambda: g.cache_keep(c, table, nxt, count.clamp(max=L), path, nxt),
         "attention": lambda: g.tree_attention(c, 0, table, q, lens, count, None, o),
         "few rows": lambda: g.tree_attention(c, 0, table, one, lens, count.clamp(max=1), None, o[:, :1].contiguous()),
         "shared": lambda: g.tree_attention(c, 0, table, q, lens, count, None, o, shared=64),
         "verify": lambda: g.verify(tree, z, None, u, *outs)}[call]()
        n = shim.shim_calls()
        shim.shim_fail(0)
        torch.cuda.synchronize()
        return n, [t.clone() for t in (c.k, c.v, o, nxt, zeros, *outs)]

    armed = 0
    launches, want = step()
    assert launches >= 1
    for armed in range(1, launches + 1):
        try:
            step()
            raise SystemExit("the call did not report the launch that failed")
        except GraftError as e:
            assert "CUDA" in str(e), e
        shim.shim_fail(0)
        assert int((lens + 1).sum()) == int(lens.sum()) + B  # (torch looks at the last error behind its launches)
        again, armed = armed, 0
        for _ in range(2):
            assert all(torch.equal(x, y) for x, y in zip(step()[1], want))
        armed = again


if __name__ == "__main__":
    import ctypes
    sys.path.insert(0, ROOT)
    _run(sys.argv[1], ctypes.CDLL(sys.argv[2]))
    print("fine")
