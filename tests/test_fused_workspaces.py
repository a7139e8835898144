"""The room that a call is told to bring is enough for it, whatever its leading dimensions are (no GPU needed: without one, a call whose
arguments are accepted ends at its first launch)."""
import ctypes
import random

import pytest
import torch

WORKSPACE = 4


@pytest.fixture(scope="module")
def gs():
    if torch.cuda.is_available():
        pytest.skip("the addresses are the host's: nothing may be launched")
    from paper_2502_11407_amd import binding
    return binding


def test_loss_takes_the_room_it_asked_for(gs):
    """Rows side by side and far apart (X = the last token of each sequence), which leads to tiles with more slabs."""
    buf = ctypes.create_string_buffer(4096)
    at = (ctypes.addressof(buf) + 255) // 256 * 256
    rng = random.Random(3)
    cases = [("bf16", 128, 50257, 4096, 2048), ("f16", 64, 32000, 4096, 4096), ("bf16", 512, 50257, 1024, 8192), ("f32", 1, 7, 3, 1)]
    for _ in range(60):
        cases.append((rng.choice(["f16", "bf16", "f32"]),) + tuple(int(10 ** rng.uniform(0, e)) for e in (4, 5, 3.5, 4)))
    for dtype, T, V, D, apart in cases:
        room = gs.xent_workspace_bytes(dtype, T, V, D)
        for ldx, ldw in ((D, D), (D * apart, D), (D, D * apart), (D * apart, D * apart), (D * apart + 1, D + 1)):
            st = gs.lib.gensor_xent_forward(gs.DTYPE[dtype], T, V, D, at, ldx, at, ldw, at, -100, at, at, at, room, None)
            assert st != WORKSPACE and st != 0, (dtype, T, V, D, ldx, ldw)
            st = gs.lib.gensor_xent_forward(gs.DTYPE[dtype], T, V, D, at, ldx, at, ldw, at, -100, at, at, at, (T * 4 + 255) // 256 * 256, None)
            assert st in (WORKSPACE, 2), (dtype, T, V, D, ldx, ldw)
