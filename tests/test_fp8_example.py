"""The example's block with RMS norms and projections in 8 bits: it runs, its gradients are
the formula's, and it streams the tokens that it gives as a whole.

Streamed and whole tokens come from the same 8-bit weights through different kernels, whose
results differ by their rounding to bf16 (test_cond_example.py: 1e-2 of the branches).  A
difference of that size moves a value over the border between two codes, 2^-3 of it apart,
with a probability of 1e-2 / 2^-3, and the square of the difference then is 2^-3 times 1e-2
and not 1e-4: 3.5e-2 a rounding to 8 bits of 1e-2 off inputs; the second and third branch take
inputs that are so far off already.  8e-2 allows for five such roundings one after another."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture()
def ex():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import conditioned_block
    finally:
        sys.path.pop(0)
    return conditioned_block


SIZES = [dict(), dict(B=1, frames=4, per_frame=55, frames_a_chunk=1, H=2, Hkv=2, d=72, states=20),
         dict(B=3, frames=6, per_frame=48, frames_a_chunk=3, H=4, Hkv=4, d=128, states=301)]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", SIZES)
def test_runs_and_streams(ex, sizes):
    losses, off = ex.run(steps=3, z=ex.Sizes(**sizes), say=lambda text: None, eight_bits=True)
    assert len(losses) == 3 and all(0 < x < 1e4 for x in losses)
    assert off <= 8e-2


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", SIZES)
def test_gradients(ex, sizes):
    """Against the block in fp32 with torch's norm, products and attention: every product is of
    two factors rounded to 8 bits, 2.6% each (2^-4 / sqrt(3) of a value from 1 to 2), and a
    gradient passes at most ten of them one after another: sqrt(20) 2.6% = 12%."""
    z = ex.Sizes(**sizes)
    block = ex.EightBitBlock(z)
    x, vectors, states, n, target = ex.batch(z)
    names = [k for k in block.p if k not in ("cross_bias",)]
    dy = torch.randn(x.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(5))
    got = torch.autograd.grad(block.train(x, vectors, states, n), [block.p[k] for k in names], dy.to(ex.BF16),
                              allow_unused=True)
    p = {k: t.detach().clone().requires_grad_(True) for k, t in block.p.items()}

    def norm(t, w=None):
        y = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-5)
        return y if w is None else y * w

    def attend(q, k, v, seen):
        s = (q @ k.transpose(-1, -2) / z.d ** 0.5).masked_fill(~seen, float("-inf"))
        s = s - torch.where(torch.isinf(s.amax(-1, keepdim=True)), 0.0, s.amax(-1, keepdim=True)).detach()
        w = s.exp()
        return w @ v / w.sum(-1, keepdim=True).clamp(min=1e-30)

    def heads(t, count):
        return t.unflatten(-1, (count, z.d)).transpose(1, 2)

    h = x.float()
    m = (vectors.float() @ p["modulate"].T)[..., :z.C].repeat_interleave(z.per_frame, 1)
    q, k, v = (heads(t, z.H) for t in (norm(h, 1 + m) @ p["qkv"].T).chunk(3, -1))
    chunk = torch.arange(z.N, device="cuda") // z.T
    o = attend(q, k, v, chunk[:, None] >= chunk[None])
    h = h + o.transpose(1, 2).flatten(2) @ p["out"].T
    q = heads(norm(h, p["cross_weight"]) @ p["cross_q"].T, z.H)
    k, v = (heads(t, z.Hkv).repeat_interleave(z.H // z.Hkv, 1) for t in (states.float() @ p["cross_kv"].T).chunk(2, -1))
    seen = (torch.arange(z.S, device="cuda") < n[:, None])[:, None, None]
    h = h + attend(q, k, v, seen).transpose(1, 2).flatten(2) @ p["cross_out"].T
    y = h + torch.nn.functional.gelu(norm(h) @ p["up"].T) @ p["down"].T
    want = torch.autograd.grad(y, [p[k] for k in names], dy)
    for name, a, b in zip(names, got, want):
        assert a.dtype == torch.float32 and bool(torch.isfinite(a).all())
        if float(b.norm()) == 0:  # (one sample whose condition is dropped)
            assert float(a.norm()) == 0
        else:
            assert float((a - b).norm() / b.norm()) < 0.12, name
