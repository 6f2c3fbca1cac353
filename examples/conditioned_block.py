"""A conditioned block of a video transformer, trained and then streamed.

    python examples/conditioned_block.py [--steps 20]

The block is x += attention(norm(x)); x += cross(norm(x), states); x += mlp(norm(x)):

- attention: block-causal over the video's chunks, its norm modulated frame by frame
  (a weight and a bias for every frame, from the frame's conditioning vector);
- cross: every token sees its sample's encoder states, of which there are another number
  in each sample and none where the condition is dropped; heads of K and V are shared;
- mlp: plain products.

Training takes one step a batch through BlockCausalAttention, CrossAttention and
LayerNorm.  Streaming takes the same weights through the calls without gradients: a chunk
a step, against a rolling cache of the block-causal keys and values and against K and V of
the states, which are projected once a prompt.  Both give the same tokens, which the
program checks."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_01127_gb300 as mw  # noqa: E402

BF16 = torch.bfloat16


class Sizes:
    def __init__(self, B=2, frames=8, per_frame=32, frames_a_chunk=2, H=6, Hkv=2, d=64, states=77, cond=32):
        self.B, self.frames, self.per_frame = B, frames, per_frame
        self.N = frames * per_frame
        self.T = frames_a_chunk * per_frame  # tokens of a chunk
        self.H, self.Hkv, self.d, self.C = H, Hkv, d, H * d
        self.S, self.cond = states, cond


class Block:
    """Weights in fp32, cast to bf16 for the products."""

    def __init__(self, z: Sizes, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)

        def w(rows, cols, gain=1.0):
            t = torch.randn(rows, cols, generator=g, device="cuda") * (gain / math.sqrt(cols))
            return t.requires_grad_(True)

        C, kv = z.C, z.Hkv * z.d
        self.z = z
        self.p = {
            "modulate": w(2 * C, z.cond, 0.1),  # a frame's vector -> its norm's weight and bias
            "qkv": w(3 * C, C), "out": w(C, C),
            "cross_weight": torch.ones(C, device="cuda", requires_grad=True),
            "cross_bias": torch.zeros(C, device="cuda", requires_grad=True),
            "cross_q": w(C, C), "cross_kv": w(2 * kv, C), "cross_out": w(C, C),
            "up": w(2 * C, C), "down": w(C, 2 * C),
        }

    def __getitem__(self, name):
        return self.p[name].to(BF16)

    def heads(self, x, n):  # [B, rows, n d] -> [B, n, rows, d]
        return x.unflatten(-1, (n, self.z.d)).transpose(1, 2).contiguous()

    def joined(self, x):
        return x.transpose(1, 2).flatten(2)

    def modulation(self, frame_vectors):
        """[B, frames, cond] -> weight and bias of the frames' norms, [B frames, C]."""
        m = (frame_vectors @ self["modulate"].T).flatten(0, 1).float()
        return (1 + m[:, :self.z.C]).contiguous(), m[:, self.z.C:].contiguous()

    def states_kv(self, states):
        k, v = (states @ self["cross_kv"].T).chunk(2, -1)
        return self.heads(k, self.z.Hkv), self.heads(v, self.z.Hkv)

    def train(self, x, frame_vectors, states, n_states):
        z = self.z
        h = mw.LayerNorm.apply(x, *self.modulation(frame_vectors))
        q, k, v = (self.heads(t, z.H) for t in (h @ self["qkv"].T).chunk(3, -1))
        x = x + self.joined(mw.BlockCausalAttention.apply(q, k, v, z.T)) @ self["out"].T
        h = mw.LayerNorm.apply(x, self.p["cross_weight"], self.p["cross_bias"])
        o = mw.CrossAttention.apply(self.heads(h @ self["cross_q"].T, z.H), *self.states_kv(states), n_states)
        x = x + self.joined(o) @ self["cross_out"].T
        h = mw.LayerNorm.apply(x)
        return x + torch.nn.functional.gelu(h @ self["up"].T) @ self["down"].T

    @torch.no_grad()
    def stream(self, x, frame_vectors, states, n_states):
        """The same, a chunk a step."""
        z = self.z
        cross_k, cross_v = self.states_kv(states)
        ring = mw.RingState(z.N)
        k_ring, v_ring = (torch.zeros(z.B, z.H, z.N, z.d, dtype=BF16, device="cuda") for _ in range(2))
        out = []
        per_chunk = z.T // z.per_frame
        for c in range(z.N // z.T):
            y = x[:, c * z.T:(c + 1) * z.T].contiguous()
            weight, bias = self.modulation(frame_vectors[:, c * per_chunk:(c + 1) * per_chunk])
            h, _, _ = mw.mw_layernorm_fwd(y, weight, bias, need_stats=False)
            qkv = (h @ self["qkv"].T).view(z.B, z.T, 3, z.H, z.d)
            q, k, v = mw.mw_qkv_rope_split(qkv)
            head, length = ring.head, ring.length
            o, _ = mw.mw_bca_cache_step(q, k, v, k_ring, v_ring, head, length, ring.commit(z.T), z.T, z.T,
                                        need_lse=False)
            y = y + self.joined(o) @ self["out"].T
            h, _, _ = mw.mw_layernorm_fwd(y, self.p["cross_weight"], self.p["cross_bias"], need_stats=False)
            o, _ = mw.mw_xattn_fwd(self.heads(h @ self["cross_q"].T, z.H), cross_k, cross_v, n_states, need_lse=False)
            y = y + self.joined(o) @ self["cross_out"].T
            h, _, _ = mw.mw_layernorm_fwd(y, need_stats=False)
            out.append(y + torch.nn.functional.gelu(h @ self["up"].T) @ self["down"].T)
        return torch.cat(out, 1)


def batch(z: Sizes, seed=1):
    g = torch.Generator("cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(BF16)

    x, vectors, states = randn(z.B, z.N, z.C), randn(z.B, z.frames, z.cond), randn(z.B, z.S, z.C)
    # the first sample's prompt is whole, the last one's dropped, those between are shorter
    n = torch.linspace(z.S, 0, z.B, device="cuda").to(torch.int32)
    return x, vectors, states, n, 0.5 * x + 0.1 * randn(z.B, z.N, z.C)


def run(steps=20, z=None, say=print):
    """(losses, relative distance of the streamed tokens from the trained block's)."""
    z = z or Sizes()
    block = Block(z)
    x, vectors, states, n, target = batch(z)
    optimizer = torch.optim.Adam(block.p.values(), lr=3e-3)
    losses = []
    for step in range(steps):
        y = block.train(x, vectors, states, n)
        loss = (y.float() - target.float()).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.item())
        say(f"step {step}: loss {losses[-1]:.4f}")
    with torch.no_grad():
        whole = block.train(x, vectors, states, n).float()
    streamed = block.stream(x, vectors, states, n).float()
    off = float((streamed - whole).norm() / whole.norm())
    say(f"streamed against trained: {off:.2e}")
    if mw.mw_device_status() != 0:
        raise RuntimeError("a kernel's bounded wait expired")
    return losses, off


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    losses, off = run(ap.parse_args().steps)
    if not (losses[-1] < losses[0] and off < 2e-2):
        raise SystemExit("the loss did not fall, or streaming gave other tokens")
