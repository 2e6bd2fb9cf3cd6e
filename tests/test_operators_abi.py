"""What of the model's operators runs without a GPU: workspace sizes, refusals before anything is enqueued."""

import ctypes
import subprocess

import pytest
import torch

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


def on_device(number):
    """A tensor type whose tensors say that they are on that device."""
    class Elsewhere(torch.Tensor):
        is_cuda = True

        def get_device(self):
            return number

    return lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype).as_subclass(Elsewhere)


def test_tensors_of_another_device_than_the_contexts_are_refused():
    twa.build_library()
    ctx = twa.Context()                        # no handle: a call that gets through the checks is refused as without a context
    ctx.device = 0
    here, there = on_device(0), on_device(1)

    def calls(n):
        """Every call with its n-th tensor on the other device; None from the number on that a call does not have."""
        def t(i, *shape, dtype=torch.float32):
            return (there if i == n else here)(*shape, dtype=dtype)

        ids, space = (dict(dtype=d) for d in (torch.int64, torch.uint8))
        yield 6, lambda: twa.twa_layer_norm(ctx, t(0, 4, 8), t(1, 8), t(2, 8), 1e-5, t(3, 4, 8), t(4, 4), t(5, 4))
        yield 9, lambda: twa.twa_layer_norm_backward(ctx, t(0, 4, 8), t(1, 4, 8), t(2, 8), t(3, 4), t(4, 4), t(5, 4, 8), t(6, 8), t(7, 8),
                                                     t(8, 64, **space))
        yield 3, lambda: twa.twa_embedding(ctx, t(0, 5, 8), t(1, 4, **ids), 1.0, t(2, 4, 8))
        yield 4, lambda: twa.twa_embedding_backward(ctx, t(0, 4, 8), t(1, 4, **ids), 1.0, t(2, 5, 8), t(3, 64, **space))
        yield 7, lambda: twa.twa_token_logprobs(ctx, t(0, 4, 8), t(1, 4, **ids), t(2, 4), t(3, 4), t(4, 4), t(5, 4, 2, dtype=torch.int32),
                                                t(6, 4, 2))
        yield 7, lambda: twa.twa_token_logprobs_backward(ctx, t(0, 4, 8), t(1, 4, **ids), t(2, 4), t(3, 4), t(4, 4, 8), t(5, 4), t(6, 4))
        yield 4, lambda: twa.twa_grad_norm(ctx, twa.Tensors([t(0, 8), t(1, 8)]), t(2, 1), t(3, 64, **space))
        yield 5, lambda: twa.twa_clip_gather(ctx, twa.Tensors([t(0, 8), t(1, 8)]), 1.0, t(2, 16), t(3, 1), t(4, 64, **space))
        yield 4, lambda: twa.twa_clip_grads(ctx, twa.Tensors([t(0, 8), t(1, 8)]), 1.0, t(2, 1), t(3, 64, **space))

    for n in range(9):
        for count, call in calls(n):
            if n < count:
                with pytest.raises(ValueError, match="device"):
                    call()
    for count, call in calls(-1):              # and with all on the context's device the checks let them through
        with pytest.raises(twa.TwaError):
            call()
    twice = twa.Tensors([there(8), there(8)])
    with pytest.raises(ValueError, match="context's device"):
        twa.twa_grad_norm(ctx, twice, here(1), here(64, dtype=torch.uint8))
