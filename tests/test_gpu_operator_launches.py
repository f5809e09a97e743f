"""The row operators' launches ask for the shared memory that they use, whatever was called before them and
whatever another thread calls beside them."""

import subprocess
import sys
import threading

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF16, F32 = torch.bfloat16, torch.float32

# Widths whose rings and a kernel's own arrays pass 48 KB together but not alone, each for another kernel,
# in a process that has called none of them at a larger width.
FRESH = r"""
import torch
from paper_1811_12843_gb300 import operators as ops
B, F = torch.bfloat16, torch.float32
def randn(rows, dim, dtype):
    return torch.randn(rows, dim, device="cuda", dtype=F).to(dtype)
def near(a, b, tol):
    assert ((a.double() - b.double()).abs() <= tol * b.double().abs().amax()).all()
x = randn(700, 8136, B)
q, s = ops.quantize_rows(x)
near(q.double() * s.double()[:, None], x, 2.0 ** -4)
for dim, dtype, res in ((6104, B, True), (3056, F, True), (6104, F, False), (5729, B, False), (3749, F, False),
                        (3897, B, True), (2321, F, True)):
    x, r, w = randn(700, dim, dtype), randn(700, dim, dtype), 1 + 0.1 * randn(1, dim, F)[0]
    n = ops.rmsnorm(x, w, residual=r if res else None)
    t = x.double() + (r.double() if res else 0)
    near(n.y, t * (t.square().mean(dim=1, keepdim=True) + 1e-6).rsqrt() * w.double(), 2.0 ** -8)
for dim, dtype, dsum in ((4072, B, False), (2313, B, True), (1875, F, False)):
    s, dy, ds = randn(700, dim, dtype), randn(700, dim, dtype), randn(700, dim, dtype)
    w, rstd = 1 + 0.1 * randn(1, dim, F)[0], (s.float().square().mean(dim=1) + 1e-6).rsqrt()
    dx, dw = ops.rmsnorm_backward(dy, s, rstd, w, dsum=ds if dsum else None)
    g, rr = dy.double() * w.double(), rstd.double()[:, None]
    ref = rr * (g - s.double() * rr * rr * (g * s.double()).mean(dim=1, keepdim=True))
    near(dx, ref + (ds.double() if dsum else 0), 2.0 ** -8)
    near(dw, (dy.double() * s.double() * rr).sum(dim=0), 2.0 ** -12)
torch.cuda.synchronize()
print("all right")
"""


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()


def test_first_calls_at_any_width():
    r = subprocess.run([sys.executable, "-c", FRESH], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "all right" in r.stdout, r.stderr[-2000:]


def test_threads_with_different_widths():
    """Two threads call one kernel, each at a width of its own, on streams of their own."""
    from paper_1811_12843_gb300 import operators as ops
    widths, failures = (16384, 9000), []
    xs = [torch.randn(620, d, device="cuda").to(BF16) for d in widths]
    want = [ops.quantize_rows(x) for x in xs]
    torch.cuda.synchronize()

    def call(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(400):
                    got = ops.quantize_rows(xs[i])
                torch.cuda.current_stream().synchronize()
            assert torch.equal(got[0].float(), want[i][0].float()) and torch.equal(got[1], want[i][1])
        except Exception as e:  # noqa: BLE001 (any failure of the thread is the test's)
            failures.append(repr(e))

    threads = [threading.Thread(target=call, args=(i,)) for i in (0, 1, 0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures


def test_a_narrower_call_between_capture_and_replay():
    from paper_1811_12843_gb300 import operators as ops
    x, narrow = torch.randn(620, 16384, device="cuda").to(BF16), torch.randn(620, 9000, device="cuda").to(BF16)
    want = ops.quantize_rows(x)
    ops.quantize_rows(narrow)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ops.quantize_rows(x)
        ops.quantize_rows(narrow)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0].float(), want[0].float()) and torch.equal(got[1], want[1])
