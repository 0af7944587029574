"""Layer norm called from several host threads at once."""
import threading

import pytest
import torch

from paper_2109_12497_b200 import binding as B
from test_gpu_mx import DT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,dtype,long,short", [("forward", "f32", 16380, 9000), ("forward", "bf16", 16376, 12800),
                                                   ("backward", "f32", 4092, 2100), ("backward", "f32", 16376, 9008)])
def test_host_threads_with_rows_of_two_lengths(kind, dtype, long, short):
    """Both lengths are one kernel's and more than 48 KiB: no thread's request for memory takes away what another's needs.  One
    thread calls with long rows, three with short ones, straight through ctypes, which lets the others run meanwhile."""
    start, refused, lib, code = threading.Barrier(4), [], B.lib(), B.UQ_F32 if dtype == "f32" else B.UQ_BF16

    def calls(cols):
        stream = torch.cuda.Stream()
        x, y = (torch.ones(1, cols, dtype=DT[dtype], device="cuda") for _ in range(2))
        one, ws = torch.ones(1, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        px, py, p1, pw, st = x.data_ptr(), y.data_ptr(), one.data_ptr(), ws.data_ptr(), stream.cuda_stream
        if kind == "forward":
            call, args = lib.uq_layer_norm, (px, 1, cols, cols, code, None, None, 1e-5, py, cols, None, None, None, None, st)
        else:
            call, args = lib.uq_layer_norm_backward, (px, cols, px, cols, 1, cols, code, None, p1, p1, py, cols, None, None, B.UQ_F32, pw, 1 << 20, st)
        start.wait()
        for _ in range(20000):
            if call(*args):
                refused.append(cols)
        stream.synchronize()

    threads = [threading.Thread(target=calls, args=(cols,)) for cols in (long, short, short, short)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert refused == []
