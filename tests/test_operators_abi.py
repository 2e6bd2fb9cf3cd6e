"""What of the model's operators runs without a GPU: workspace sizes, refusals before anything is enqueued."""

import ctypes
import subprocess

from paper_2205_13104_b200 import twa


def test_workspace_sizes():
    twa.build_library()
    assert twa.twa_layer_norm_workspace_bytes(0, 4) >= 2 * 4 * 4
    assert twa.twa_layer_norm_workspace_bytes(10, 1000) >= 10 * 2 * 1000 * 4
    assert twa.twa_layer_norm_workspace_bytes(1 << 30, 1000) == twa.twa_layer_norm_workspace_bytes(1 << 20, 1000)
    assert twa.twa_layer_norm_workspace_bytes(-1, 4) == 0
    assert twa.twa_embedding_workspace_bytes(1000, 50272, 64) >= 4 * 4 * 1000 + 50272 // 8
    assert twa.twa_embedding_workspace_bytes(1 << 40, 5, 4) == 0
    assert twa.twa_grad_norm_workspace_bytes(0) > 0
    assert twa.twa_grad_norm_workspace_bytes(513) > twa.twa_grad_norm_workspace_bytes(512)
    assert twa.twa_grad_norm_workspace_bytes(twa.TWA_MAX_TENSORS + 1) == 0


def test_workspaces_of_the_widest_rows_and_the_largest_vocabularies():
    twa.build_library()
    cols = twa.TWA_LAYER_NORM_MAX_COLS
    assert 64 * 2 * 4 * cols <= twa.twa_layer_norm_workspace_bytes(1 << 20, cols) <= 65 * 2 * 4 * cols
    assert twa.twa_embedding_workspace_bytes(4, twa.TWA_EMBEDDING_MAX_VOCAB, 4) > twa.TWA_EMBEDDING_MAX_VOCAB // 8
    assert twa.twa_embedding_workspace_bytes(4, twa.TWA_EMBEDDING_MAX_VOCAB + 1, 4) == 0


def test_calls_without_a_context_are_refused():
    twa.build_library()
    lib = twa.load()
    d = 4096                                   # never looked at
    bad = twa.TWA_ERR_INVALID_ARG
    assert lib.twa_layer_norm(None, d, 8, 0, d, d, 0, 4, 8, 1e-5, d, 8, d, d) == bad
    assert lib.twa_layer_norm_backward(None, d, 8, d, 8, 0, d, 0, d, d, 4, 8, d, 8, d, d, 0, 0, d, 1 << 20) == bad
    assert lib.twa_embedding(None, d, 8, 0, 5, 8, d, 0, 4, 1.0, d, 8, 0) == bad
    assert lib.twa_embedding_backward(None, d, 8, 0, d, 0, 4, 5, 8, 1.0, -1, d, 8, 0, 0, d, 1 << 20) == bad
    assert lib.twa_token_logprobs(None, d, 8, 0, 4, 8, d, 0, -100, d, d, d, 0, None, None) == bad
    assert lib.twa_token_logprobs_backward(None, d, 8, 0, 4, 8, d, 0, -100, d, None, d, None, d, 8) == bad
    t = twa.twa_tensors(None, None, None, 0)
    assert lib.twa_grad_norm(None, ctypes.byref(t), d, d, 1 << 20) == bad
    assert lib.twa_clip_gather(None, ctypes.byref(t), 1.0, 1e-6, d, 0, d, d, 1 << 20) == bad
    assert lib.twa_clip_grads(None, ctypes.byref(t), 1.0, 1e-6, d, d, 1 << 20) == bad


READS = """
#include <stdio.h>
#include "twa_layer_norm.cuh"
// Units of E elements as LnPlace lays them out over a row; a unit that the row has in part is read whole where there are rows before
// and after it.  Prints every read beside the matrix.
int main() {
  for (int size : {2, 4})
    for (int rows = 1; rows <= 5; ++rows)
      for (int cols = 1; cols <= 19; ++cols)
        for (int ld = cols; ld <= cols + 9; ++ld)
          for (int other = ld; other <= ld + 8; other += 8)
            for (int start = 0; start < 8; ++start) {
              const int E = 16 / size;
              const char* at = reinterpret_cast<const char*>(4096) + start * size;
              if (!ln_classes(at, ld, at, other, at, other, rows, cols, size)) continue;
              for (int stride : {ld, other})
                for (int r = 1; r + 1 < rows; ++r) {
                  const int first = r * stride, skew = (start + first) % E, end = (rows - 1) * stride + cols;
                  for (int k = 0; k * E < skew + cols; ++k) {
                    const int from = first - skew + k * E;
                    if (from < 0 || from + E > end)
                      printf("%d bytes, %d x %d, stride %d, start %d: row %d reads %d .. %d of %d\\n", size, rows, cols, stride, start, r,
                             from, from + E - 1, end);
                  }
                }
            }
}
"""


def test_layer_norm_reads_nothing_beside_the_matrix(tmp_path):
    """The rule by which rows are read in units of 16 bytes, compiled for the host."""
    source, program = tmp_path / "reads.cu", tmp_path / "reads"
    source.write_text(READS)
    subprocess.run([twa._nvcc(), *twa.NVCC_FLAGS, "-I", twa.CSRC, "-o", str(program), str(source)], check=True)
    assert subprocess.run([str(program)], check=True, capture_output=True, text=True).stdout == ""
