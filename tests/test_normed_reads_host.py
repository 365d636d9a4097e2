"""What the threads of the normed heads' kernels read of a row, compiled for the host: every element of every head once, and nothing outside. A
thread that has no head (a block is rounded up to whole warps, a last block of a row's may be part full) has a place behind the last one,
which lies outside what the caller gave."""
import ctypes
import subprocess

import numpy as np
import pytest

from paper_2609_30884_gb300 import build

SHIM = r"""
#include "head_norm.cu"
namespace crf {  // what the launches need and the layout does not
PdlScope::PdlScope() : prev_(false) {}
PdlScope::~PdlScope() {}
bool pdl_active() { return false; }
}  // namespace crf
using namespace crf;
// Reads of one row as (part, head, first element): threads' first units, and second ones as the gradient takes them. Returns how many, -1 where
// heads have no such form; `threads` counts those that read nothing.
template <int VEC, bool INTER, int BATCH>
static int reads(const RotaryDesc& d, bool few, bool gradient, int* out, int most, int* idle) {
  Tiling t = {};
  if (!vector_form(d, VEC, &t)) return -1;
  deal_slots(d, BATCH, few, &t);
  int n = 0;
  *idle = 0;
  for (unsigned column = 0; column < columns_of(t); ++column)
    for (int thread = 0; thread < block_threads(t); ++thread) {
      const Place p = place_of<VEC, INTER, BATCH>(t, d, thread, static_cast<int>(column));
      if (p.rb != 0) continue;
      auto put = [&](int head, int e) {
        if (n < most) out[3 * n] = p.part, out[3 * n + 1] = head, out[3 * n + 2] = e;
        ++n;
      };
      const int was = n;
      if (gradient) {
        if (p.heads > 0) put(p.head, p.e0);
        if (second_unit<INTER>(p)) put(p.head + (INTER ? 1 : 0), INTER ? p.e0 : p.e1);
      } else {
        for (int b = 0; b < p.heads; ++b) {
          put(p.head + b, p.e0);
          if (!INTER && p.turning) put(p.head + b, p.e1);
        }
      }
      *idle += n == was;
    }
  return n;
}
// form: 0 a gradient, 1 and 4 a forward call of that many heads a thread
extern "C" int reads_of_row(int dim, int rot, int inter, int size, int parts, const int* heads, int few, int form, int* out, int most, int* idle) {
  RotaryDesc d = {};
  d.head_dim = dim, d.rot_dim = rot, d.interleaved = inter != 0, d.n_parts = parts;
  for (int i = 0; i < parts; ++i) d.part[i].heads = heads[i], d.part[i].rotate = true;
  const bool g = form == 0;
#define FORM(VEC, INTER, BATCH) reads<VEC, INTER, BATCH>(d, few != 0, g, out, most, idle)
  if (size == 2)
    return g ? (inter ? FORM(8, true, kGradBatch<true>) : FORM(8, false, kGradBatch<false>))
             : form == 1 ? (inter ? FORM(8, true, 1) : FORM(8, false, 1)) : inter ? FORM(8, true, kNormBatch) : FORM(8, false, kNormBatch);
  return g ? (inter ? FORM(4, true, kGradBatch<true>) : FORM(4, false, kGradBatch<false>))
           : form == 1 ? (inter ? FORM(4, true, 1) : FORM(4, false, 1)) : inter ? FORM(4, true, kNormBatch) : FORM(4, false, kNormBatch);
}
"""


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    try:
        nvcc = build.nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    d = tmp_path_factory.mktemp("reads")
    (d / "shim.cu").write_text(SHIM)
    subprocess.run([nvcc, *build.ARCH, "-O1", "-std=c++17", "--expt-relaxed-constexpr", "-I", build.CSRC, "-I", build.INCLUDE,
                    "-shared", "-Xcompiler", "-fPIC", "-cudart", "shared", str(d / "shim.cu"), "-o", str(d / "reads.so")], check=True)
    return ctypes.CDLL(str(d / "reads.so"))


HEADS = [(1,), (3,), (1, 1), (3, 1), (12, 2), (28, 4), (9, 5), (7, 0 + 6), (33,), (40, 8), (70, 9), (130, 3), (5, 3, 3), (28, 4, 4)]


@pytest.mark.parametrize("form", [0, 1, 4])
@pytest.mark.parametrize("size", [2, 4])
@pytest.mark.parametrize("inter", [0, 1])
def test_a_row_is_read_once_and_nothing_beside_it(so, inter, size, form):
    vec, idle, some, spare = 16 // size, ctypes.c_int(), 0, 0
    out = np.zeros((200000, 3), dtype=np.int32)
    for dim, rot in ((64, 64), (128, 128), (128, 64), (128, 32), (256, 256), (96, 96), (96, 48), (80, 80), (64, 16), (256, 128), (16, 16), (32, 16)):
        for heads in HEADS:
            if form == 0 and len(heads) > 2:
                continue
            for few in (0, 1):
                n = so.reads_of_row(dim, rot, inter, size, len(heads), (ctypes.c_int * 3)(*heads), few, form, out.ctypes.data_as(ctypes.c_void_p),
                                    len(out), ctypes.byref(idle))
                assert n <= len(out)
                if n < 0:
                    continue
                some, spare = some + 1, spare + (idle.value > 0)
                met = [np.zeros((h, dim), dtype=int) for h in heads]
                for part, head, e in out[:n]:
                    assert 0 <= part < len(heads) and 0 <= head < heads[part] and 0 <= e <= dim - vec, (dim, rot, heads, few, part, head, e)
                    met[part][head, e:e + vec] += 1
                assert all((m == 1).all() for m in met), (dim, rot, heads, few)
    assert some > 100 and spare > 20
