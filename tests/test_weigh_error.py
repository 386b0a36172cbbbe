"""A kv_weigh that gives up one of its bounded waits is remembered, with or without a status array.

The kernel's own waits do not run out, and none is made to: the GPU test builds the kernel's source with one kernel more,
a warp that waits as the kernel's roles do, on a barrier that nothing signals, for the second that the wait takes.
"""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2608_03447_gb300 import build

KERNEL = """
#include "asd_weigh_tc.cu"
namespace {
__global__ void give_up(int* waited) {
  __shared__ WeighShared sh;
  if (threadIdx.x == 0) {
    mbar_init(&sh.drain, 1);
    sh.abort = 0;
  }
  __syncthreads();
  const bool came = warp_wait(&sh.drain, 0, sh);
  if (threadIdx.x == 0) *waited = came ? 1 : 2 + sh.abort;
}
}  // namespace
extern "C" int run(void* waited, void* stream) {
  give_up<<<1, 32, 0, static_cast<cudaStream_t>(stream)>>>(static_cast<int*>(waited));
  return static_cast<int>(cudaGetLastError());
}
"""


def test_there_has_to_be_a_place_for_the_answer():
    from paper_2608_03447_gb300 import asd
    assert asd.load().asd_weigh_error(None, None) == 1


@pytest.mark.gpu
def test_a_wait_that_runs_out_is_remembered(asd, tmp_path):
    (tmp_path / "give_up.cu").write_text(KERNEL)
    out = str(tmp_path / "give_up.so")
    subprocess.run([build.nvcc_path(), *build.ARCH, *build.NVCC_FLAGS, f"-I{build.CSRC}", "-shared", "-cudart", "static",
                    str(tmp_path / "give_up.cu"), "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.run.argtypes = lib.asd_weigh_error.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    stream = torch.cuda.current_stream().cuda_stream
    word, waited = ctypes.c_int(7), torch.zeros(1, dtype=torch.int32, device="cuda")

    def error():
        assert lib.asd_weigh_error(ctypes.addressof(word), stream) == 0
        return word.value
    assert error() == 0
    assert lib.run(waited.data_ptr(), stream) == 0
    assert error() == 9 and waited.tolist() == [3]  # gave up, with the CTA's abort mark set
    assert error() == 0  # read once
    assert asd.weigh_error() == 0  # another library's word


@pytest.mark.gpu
def test_ordinary_calls_leave_nothing(asd):
    k = torch.randn(1, 4, 16, 2, 64, device="cuda").bfloat16()
    cache = asd.KVCache(k, k.clone(), torch.arange(4, dtype=torch.int32, device="cuda")[None])
    q = torch.randn(1, 3, 4, 64, device="cuda").bfloat16()
    weight = torch.zeros(1, 2, 64, device="cuda")
    lse, kv_len = torch.full((1, 3, 4), 5.0, device="cuda"), torch.full((1,), 40, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    asd.kv_weigh(q, lse, cache, kv_len, weight, stream=side)
    assert asd.weigh_error(side) == 0 and asd.weigh_error() == 0
    assert int((weight > 0).sum()) == 2 * 43
