"""The extension calls are dependent launches: their kernels may become resident while the kernel before them still runs.
However long that takes, no bounded wait of theirs may count it."""
import ctypes
import subprocess

import pytest
import torch

import paper_2609_30884_gb300 as crf
from paper_2609_30884_gb300 import build
from tests.test_gpu_extend import Setup

pytestmark = pytest.mark.gpu

# A caller's kernel that lets its dependents start at once and ends after `ns` (or a bounded number of turns).
DELAY = r"""
#include <cuda_runtime.h>
__global__ void delay_kernel(unsigned long long ns) {
  asm volatile("griddepcontrol.launch_dependents;");
  unsigned long long t0, t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t0));
  for (int i = 0; i < 4000000; ++i) {
    __nanosleep(1000);
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    if (t - t0 >= ns) break;
  }
}
extern "C" int delay(unsigned long long ns, void* stream) {
  delay_kernel<<<1, 1, 0, static_cast<cudaStream_t>(stream)>>>(ns);
  return static_cast<int>(cudaGetLastError());
}
"""
SECONDS = 3.0  # the kernels' wait limit is two


@pytest.fixture(scope="module")
def delay(tmp_path_factory):
    d = tmp_path_factory.mktemp("delay")
    (d / "delay.cu").write_text(DELAY)
    subprocess.run([build.nvcc(), *build.ARCH, "-shared", "-Xcompiler", "-fPIC", "-cudart", "shared", str(d / "delay.cu"),
                    "-o", str(d / "delay.so")], check=True)
    lib = ctypes.CDLL(str(d / "delay.so"))
    lib.delay.argtypes = [ctypes.c_ulonglong, ctypes.c_void_p]

    def call(seconds):
        assert lib.delay(int(seconds * 1e9), torch.cuda.current_stream().cuda_stream) == 0

    return call


# single tokens cut among CTAs (and merged); tiles of 256 rows
@pytest.mark.parametrize("chunks", [[(1, 9000), (2, 700)], [(300, 500), (1, 40)]])
def test_attention_behind_a_long_kernel(delay, chunks):
    ctx = crf.Context(0)
    s = Setup(61, 12, 2, 128, chunks, poison=False)
    want, lse0 = s.run(ctx)
    ctx.check()
    b = s.batch()
    ws = ctx.chunk_attention_workspace(s.pool, b, s.hq)
    out, lse = torch.zeros_like(want), torch.zeros_like(lse0)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    torch.cuda.synchronize()
    start.record()
    delay(SECONDS)
    ctx.chunk_attention(s.pool, 0, b, s.q, out, ws, lse=lse)
    end.record()
    ctx.check()
    assert start.elapsed_time(end) >= 0.9e3 * SECONDS
    assert torch.equal(out, want) and torch.equal(lse, lse0)
    ctx.close()
