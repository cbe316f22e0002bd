"""grad_b of the linear layer over many rows of one sign: no lane adds up more than 256 numbers in a chain, whatever the layer's width.

The gradient is one number everywhere, chosen so that a longer chain rounds the same way at each of its additions: 1 + 0.49 * 2^-13 added up in fp32 loses
0.49 * 2^-13 with each addition from 1024 on.  Tolerance: a sum of n numbers of one sign, added up in chains of 256, then of the workgroup's rows side by
side (128 at most), then of the runs, 16 side by side, and their 16: as many halves of fp32's steps of the result, and one rounding."""
import ctypes

import pytest
import torch

from paper_2401_06197_amd import binding as dcn

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


# many outputs, few, and many rows of a few
@pytest.mark.parametrize("P,N", [(8192, 131080), (16384, 131072 + 4096), (2 ** 22, 512), (2 ** 20, 264), (2 ** 20, 16)])
def test_chains_are_short(P, N):
    lib, K = dcn.load_library(), 8
    value = float(torch.tensor(1 + 0.49 * 2.0 ** -13))
    gy = torch.full((P, N), value, device="cuda")
    gb = torch.empty(N, device="cuda")
    need = dcn.dcnv4_linear_backward_workspace_bytes(P, K, N, dcn.DCNV4_F32)
    space = torch.empty(need, dtype=torch.uint8, device="cuda")
    rc = lib.dcnv4_linear_backward(None, None, ctypes.c_void_p(gy.data_ptr()), None, None, ctypes.c_void_p(gb.data_ptr()), ctypes.c_void_p(space.data_ptr()), need,
                                   P, K, N, dcn.DCNV4_F32, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0
    want = P * value
    off = float(((gb.double() - want) / want).abs().max())
    runs = -(-P // 1024)
    assert off <= (256 + 128 + runs / 16 + 16 + 1) * E, off / E
    assert bool((gb == gb[0]).all())
