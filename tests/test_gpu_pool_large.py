"""Pooling of more than 2^32 outputs from an input off the vector boundaries, which is done an output a thread."""
import gc

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_more_outputs_than_a_launch_has_threads():
    from paper_2502_11407_amd import binding as gs
    planes, side = 65600, 256                    # 2^32 + 2^22 outputs
    flat = torch.empty(planes * side * side + 1, dtype=torch.float16, device="cuda")
    flat[1:].view(planes, side * side)[:] = (torch.arange(planes, device="cuda", dtype=torch.int32) % 2039)[:, None].to(torch.float16)
    I = flat[1:].view(1, planes, side, side)
    O = torch.full((1, planes, side, side), 7.5, dtype=torch.float16, device="cuda")
    gs.avgpool2d("f16", I, O, 1, 1, out_dtype="f16")
    assert torch.equal(O, I)                     # (means of one value)
    del flat, I, O
    gc.collect()
    torch.cuda.empty_cache()
