"""The example that trains and streams a conditioned block, over several sizes.

Streamed and trained tokens come from the same weights through different kernels: each of
the block's three branches rounds some six intermediate results to bf16 (1.7e-3 each in
the mean square) once in either form, so the tokens differ by sqrt(2 * 6 * 3) 1.7e-3 =
1e-2 of the branches, which are at most the tokens' size; 2e-2 allows for twice that."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import conditioned_block
    finally:
        sys.path.pop(0)
    return conditioned_block


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [
    dict(),
    dict(B=1, frames=4, per_frame=55, frames_a_chunk=1, H=2, Hkv=1, d=72, states=20),
    dict(B=3, frames=6, per_frame=48, frames_a_chunk=3, H=4, Hkv=4, d=128, states=301),
])
def test_trains_and_streams(sizes):
    ex = _example()
    losses, off = ex.run(steps=8, z=ex.Sizes(**sizes), say=lambda text: None)
    assert all(b < a for a, b in zip(losses, losses[4:]))
    assert off <= 2e-2
