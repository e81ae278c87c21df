"""GPU: a workspace that libw8a8 prepares by itself serves a product whose walk along k is shared."""
import numpy as np
import pytest
import torch

from paper_2505_22179_amd import binding as B
from tests.test_gpu_w8a8 import Linear

pytestmark = pytest.mark.gpu


def test_a_workspace_of_its_own_preparation():
    lin = Linear(41, 40, 128, 16384)   # 40 tokens, a long walk: shared by several workgroups, which count with tickets
    want = lin.linear()
    ws = torch.full((B.w8a8_workspace_bytes(lin.M, lin.N, lin.K),), 0x5B, dtype=torch.uint8, device="cuda")
    print("w4a16_workspace_init of libw8a8", flush=True)
    assert B.load_w8a8().w4a16_workspace_init(ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert not ws[:16384].any()
    for _ in range(2):   # the tickets are zero again behind each call
        np.testing.assert_array_equal(lin.linear(ws=ws).view(np.uint16), want.view(np.uint16))
