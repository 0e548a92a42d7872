"""Buffer accesses of the operators, from the compiler's assembly (no GPU)."""
import os
import re
import subprocess

import pytest

from paper_2608_13966_amd import build as B

PIECES = """
#include "ops_common.h"
using namespace quasar;
// rows whose pieces lie past any immediate offset
template <int T>
__device__ void copy(const void* x, void* y, int bytes) {
  const int at = threadIdx.x * 8 * elem_size<T>();
  for (int v = 0; v < 4; v++) {
    Piece<T> p;
    load_piece<T>(p, wave_buffer(const_cast<void*>(x), bytes), at + v * 65536);
    float f[8];
    for (int i = 0; i < 8; i++) f[i] = p.get(i) * 2.0f;
    store_piece<T == kElemBF16>(wave_buffer(y, bytes), at + v * 65536, f);
  }
}
__global__ void pieces(const void* x, void* y, int bytes, bool bf16) {
  bf16 ? copy<kElemBF16>(x, y, bytes) : copy<kElemF32>(x, y, bytes);
}
"""


def _scalar_offsets(asm):
    """The scalar offset operand of every buffer load and store."""
    return re.findall(r"^\s*buffer_(?:load|store)\S*\s+v\S+\s+(?:v\d+|off),\s*s\[\d+:\d+\],\s*([^\s,]+)", asm, flags=re.M)


def _assembly(src, cwd):
    out = os.path.join(cwd, "out.s")
    r = subprocess.run([B.hipcc(), *B.COMMON, "--cuda-device-only", "-S", src, "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return open(out).read()


def test_pieces_have_their_whole_offset_checked(tmp_path):
    """The check against a buffer's end covers the vector and immediate offsets; a scalar one beside them would let the
    pieces past a row's end read past the allocation."""
    src = tmp_path / "pieces.hip"
    src.write_text(PIECES)
    off = _scalar_offsets(_assembly(str(src), str(tmp_path)))
    assert len(off) == 4 * 2 + 4 * 4 and set(off) == {"0"}, off


@pytest.mark.slow
def test_the_distillation_kernels_have_no_scalar_offsets(tmp_path):
    off = _scalar_offsets(_assembly(os.path.join(B.CSRC, "distill_kernel.hip"), str(tmp_path)))
    assert len(off) > 1000 and set(off) == {"0"}, (len(off), set(off))
