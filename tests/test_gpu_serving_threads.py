"""First calls from several host threads at once, as a C program makes them (ctypes lets go of Python's lock)."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import ctypes, threading
import torch
import paper_2608_12629_b200 as cake
from paper_2608_12629_b200 import serving
L, dev, n = serving._load(), "cuda:0", 8
bf, e4 = torch.bfloat16, torch.float8_e4m3fn
torch.manual_seed(3)
M, N, K = 16, 1024, 2048
x, w = torch.randn(300, K, device=dev).to(e4), torch.randn(N, K, device=dev).to(e4)
xs, ws = torch.rand(300, K // 128, device=dev) + .5, torch.rand(N // 128, K // 128, device=dev) + .5
k, v = (torch.randn(64, 16, 2, 128, device=dev, dtype=bf) for _ in range(2))
cache = cake.PagedCache(k, v)
q = torch.randn(3, 8, 128, device=dev, dtype=bf)
table, lens = torch.arange(48, dtype=torch.int32, device=dev).view(3, 16), torch.tensor([256, 3, 100], dtype=torch.int32, device=dev)
streams = [torch.cuda.Stream() for _ in range(n)]

def buffers():
    return dict(g=torch.zeros(cake.cake_gemm_fp8_workspace_bytes(300, N, K) + (1 << 20), dtype=torch.uint8, device=dev),
                d=cake.alloc_decode_workspace(3, 8, 2, 128, dev), small=torch.zeros(M, N, device=dev), large=torch.zeros(300, N, device=dev),
                out=torch.zeros(3, 8, 128, dtype=bf, device=dev))

def calls(b, stream):
    p = ctypes.c_void_p(stream)
    rc = [L.cake_gemm_fp8(x.data_ptr(), K, xs.data_ptr(), w.data_ptr(), K, ws.data_ptr(), m, N, K, b[o].data_ptr(), N, b["g"].data_ptr(),
                          b["g"].numel(), p, cake.CAKE_GEMM_OUT_FP32) for m, o in ((M, "small"), (300, "large"))]
    rc.append(L.cake_paged_decode(q.data_ptr(), 1024, 128, ctypes.byref(cache._struct), table.data_ptr(), 16, 0, 16, lens.data_ptr(), 1, 0, 3, 8, .1, 0,
                                  b["out"].data_ptr(), None, b["d"].data_ptr(), b["d"].numel(), p))
    return rc

bufs, codes, gate = [buffers() for _ in range(n)], [None] * n, threading.Barrier(n)
torch.cuda.synchronize()

def work(i):
    torch.cuda.set_device(0)
    gate.wait()
    codes[i] = calls(bufs[i], streams[i].cuda_stream)

threads = [threading.Thread(target=work, args=(i,)) for i in range(n)]
[t.start() for t in threads]
[t.join() for t in threads]
torch.cuda.synchronize()
assert all(c == [0, 0, 0] for c in codes), codes
last = buffers()
torch.cuda.synchronize()
assert calls(last, streams[0].cuda_stream) == [0, 0, 0]
torch.cuda.synchronize()
for b in bufs:
    assert all(torch.equal(b[o], last[o]) for o in ("small", "large", "out"))
assert bool(torch.isfinite(last["large"]).all()) and bool((last["out"] != 0).any())
print("same")
"""


def test_first_calls_of_several_threads_at_once():
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stdout + r.stderr
