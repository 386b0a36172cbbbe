"""What tree attention reports when one of its bounded waits runs out: the call itself flags its requests.

The kernel's own waits do not run out, and none is made to. The GPU test builds a kernel of its own around the pieces
that the attention kernel uses for it: the bounded wait, on a barrier that nothing signals, and the flags.
"""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2608_03447_gb300 import build


def test_the_call_that_gives_up_flags_its_requests():
    """Where a CTA ends with its abort mark set, it flags the requests before it returns."""
    with open(os.path.join(build.CSRC, "asd_attention_tc.cu")) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    end = code[code.index("if (sh.abort) {"):code.index("tcgen05.dealloc")]
    assert re.search(r"attn_incomplete\(p\.status, p\.B, threadIdx\.x, kThreads\)", end)


KERNEL = """
#include "asd_attention.cuh"
using namespace asd_detail;
namespace {
__global__ void give_up(int32_t* status, int B, unsigned* error) {
  __shared__ unsigned long long bar;
  __shared__ int abort;
  if (threadIdx.x == 0) {
    mbar_init(&bar, 1);
    abort = 0;
  }
  __syncthreads();
  if (threadIdx.x == 0 && !mbar_wait(&bar, 0, &abort)) {
    abort = 1;
    atomicExch(error, static_cast<unsigned>(ASD_ERR_TIMEOUT));
  }
  __syncthreads();
  if (abort) attn_incomplete(status, B, threadIdx.x, blockDim.x);
}
}  // namespace
extern "C" int run(void* status, int B, void* error, void* stream) {
  give_up<<<1, 64, 0, static_cast<cudaStream_t>(stream)>>>(static_cast<int32_t*>(status), B,
                                                           static_cast<unsigned*>(error));
  return static_cast<int>(cudaGetLastError());
}
"""


@pytest.mark.gpu
def test_a_wait_that_runs_out(asd, tmp_path):
    (tmp_path / "give_up.cu").write_text(KERNEL)
    out = str(tmp_path / "give_up.so")
    subprocess.run([build.nvcc_path(), *build.ARCH, *build.NVCC_FLAGS, f"-I{build.CSRC}", "-shared", "-cudart", "static",
                    str(tmp_path / "give_up.cu"), "-o", out], check=True)
    run = ctypes.CDLL(out).run
    run.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
    stream = torch.cuda.current_stream().cuda_stream
    status = torch.zeros(130, dtype=torch.int32, device="cuda")
    status[3] = asd.STATUS_PAGE
    error = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert run(status.data_ptr(), 129, error.data_ptr(), stream) == 0
    torch.cuda.synchronize()
    want = torch.full((130,), asd.STATUS_INCOMPLETE, dtype=torch.int32)
    want[3] |= asd.STATUS_PAGE
    want[129] = 0
    assert int(error) == 9 and torch.equal(status.cpu(), want)
    assert run(None, 129, error.data_ptr(), stream) == 0
    torch.cuda.synchronize()
