"""An attention block between an encoder's frames and the lattice, from the calls of ``binding``: how the residual norm, the products, the
norms of heads with their rotation, attention over a band of frames and the paged cache go together in training and in streaming recognition.

    python -m paper_2304_13134_amd.frame_attention        # trains a small encoder through the globally normalised loss, then streams it

Training keeps the norm's result in 8 bits, queries and keys before and after their norms, values, the attention's result and the logarithms
of its softmax sums, never a matrix of frames by frames.  Streaming keeps keys and values of the frames heard in pages, and gives it one frame
or a chunk at a time.
"""
from __future__ import annotations

import torch

from . import binding as lb
from .frame_block import FrameModel, synthetic_batch


class FrameAttention:
    """y = x + attention(queries, keys, values of norm(x)) wo^T + bo on frames [B, T, H] in bfloat16, of which lengths [B] exist.

    `heads` heads share `kv_heads` heads of keys and values.  A frame sees `left` frames before it and `right` after (None: all), and the first
    `sinks` ones."""

    def __init__(self, hidden, heads, kv_heads=None, left=None, right=0, sinks=0, base=10000.0, device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.heads, self.kv_heads, self.width = heads, kv_heads or heads, hidden // heads
        self.band = {"left": left, "right": right, "sinks": sinks}
        columns = (self.heads + 2 * self.kv_heads) * self.width
        self.split = [self.heads * self.width, self.kv_heads * self.width, self.kv_heads * self.width]
        self.gain = torch.ones(hidden, device=device)
        self.wqkv = (torch.randn(columns, hidden, generator=g, device=device) * hidden ** -0.5).bfloat16()
        self.bqkv = torch.zeros(columns, device=device)
        self.gain_q, self.gain_k = torch.ones(self.width, device=device), torch.ones(self.width, device=device)
        self.wo = (torch.randn(hidden, self.split[0], generator=g, device=device) * self.split[0] ** -0.5).bfloat16()
        self.bo = torch.zeros(hidden, device=device)
        pairs = self.width // 8 * 4
        self.frequencies = base ** (-torch.arange(pairs, device=device, dtype=torch.float32) / pairs)

    def parameters(self):
        return {"gain": self.gain, "wqkv": self.wqkv, "bqkv": self.bqkv, "gain_q": self.gain_q, "gain_k": self.gain_k, "wo": self.wo, "bo": self.bo}

    def forward(self, x, lengths=None, keep=torch.int8):
        """(y, what backward() needs)"""
        n = lb.last_residual_norm(x, self.gain, lengths=lengths, dtype=x.dtype, keep=keep)
        qkv, _ = lb.last_product(n.y, self.wqkv, self.bqkv, lengths=lengths)
        q, k, v = qkv.split(self.split, dim=-1)
        nq, nk = lb.last_head_norm(q, k, self.width, self.gain_q, self.gain_k, self.frequencies, lengths=lengths)
        a, lse = lb.last_attention(nq, nk, v, self.width, lengths=lengths, **self.band)
        y, _ = lb.last_product(a, self.wo, self.bo, residual=x, lengths=lengths)
        return y, (x, n.inv, n.kept, qkv, nq, nk, a, lse)

    def backward(self, dy, saved, lengths=None):
        """(dx, gradients by name) of dy in bfloat16; weights' gradients in float32."""
        x, inv, n, qkv, nq, nk, a, lse = saved
        q, k, v = qkv.split(self.split, dim=-1)
        dwo, dbo = lb.last_product_grad_weight(dy, a, lengths=lengths)
        da = lb.last_product_grad_input(dy, self.wo, lengths=lengths)
        dqkv = torch.empty_like(qkv)
        d = dqkv.split(self.split, dim=-1)
        lb.last_attention_grad(da, nq, nk, v, a, lse, self.width, lengths=lengths, out=d, **self.band)
        _, _, dgain_q, dgain_k = lb.last_head_norm_grad(d[0], d[1], q, k, self.width, self.gain_q, self.gain_k, self.frequencies, lengths=lengths,
                                                        out=d[:2])
        dwqkv, dbqkv = lb.last_product_grad_weight(dqkv, n, lengths=lengths)
        dn = lb.last_product_grad_input(dqkv, self.wqkv, lengths=lengths)
        dx, dgain = lb.last_residual_norm_grad(dn, x, self.gain, inv, ds=dy, lengths=lengths)
        return dx, {"gain": dgain, "wqkv": dwqkv, "bqkv": dbqkv, "gain_q": dgain_q, "gain_k": dgain_k, "wo": dwo, "bo": dbo}

    def pages(self, count, page=64):
        """(keys, values) for a Cache: `count` pages of `page` frames."""
        return tuple(torch.empty(count, self.kv_heads, page, self.width, dtype=torch.bfloat16, device=self.gain.device) for _ in range(2))

    def stream(self, x, cache, lengths=None):
        """forward() of new frames x [B, T, H] of streams whose earlier ones are in `cache`, where these go too (the caller adds them to cache.used).
        A frame sees no later ones than the call brings."""
        n = lb.last_residual_norm(x, self.gain, lengths=lengths, dtype=x.dtype)
        qkv, _ = lb.last_product(n.y, self.wqkv, self.bqkv, lengths=lengths)
        q, k, v = qkv.split(self.split, dim=-1)
        nq = lb.last_cache_append(k, v, cache, q=q, gain_q=self.gain_q, gain_k=self.gain_k, frequencies=self.frequencies, lengths=lengths)
        a = lb.last_cached_attention(nq, cache, lengths=lengths, **self.band)
        return lb.last_product(a, self.wo, self.bo, residual=x, lengths=lengths)[0]


class FrameEncoder(FrameModel):
    """FrameModel with an attention block before its feed-forward one."""

    def __init__(self, hidden=128, inner=512, V=8, heads=4, kv_heads=2, left=16, right=0, sinks=2, device="cuda", seed=0):
        super().__init__(hidden, inner, V, device=device, seed=seed)
        self.attention = FrameAttention(hidden, heads, kv_heads, left, right, sinks, device=device, seed=seed + 2)

    def loss_and_gradients(self, x, lengths, refs, ref_lengths):
        z, saved = self.attention.forward(x, lengths)
        loss, gradients, dz = self.loss_of_frames(z, lengths, refs, ref_lengths)
        _, grads = self.attention.backward(dz, saved, lengths)
        return loss, gradients + [(p, grads[k]) for k, p in self.attention.parameters().items()]


def main(steps=30, chunk=8):
    model = FrameEncoder()
    x, lengths, refs, ref_lengths = synthetic_batch()
    for i in range(steps):
        loss = model.step(x, lengths, refs, ref_lengths)
        if i % 5 == 0 or i == steps - 1:
            print("step %2d  loss %.3f" % (i, loss), flush=True)
    # the same frames as streams, a chunk at a time
    B, T, _ = x.shape
    y, _ = model.attention.forward(x, lengths)
    page, entries = 16, (T + 15) // 16
    table = torch.randperm(B * entries, device=x.device).to(torch.int32).reshape(B, entries)
    cache = lb.Cache(*model.attention.pages(B * entries, page), table, torch.zeros(B, dtype=torch.int32, device=x.device))
    parts = []
    for t in range(0, T, chunk):
        new = (lengths - t).clamp(0, min(chunk, T - t)).to(torch.int32)
        parts.append(model.attention.stream(x[:, t:t + chunk].contiguous(), cache, new))
        lb.check_item_status()
        cache.used.add_(new)
    z = torch.cat(parts, 1)
    print("streamed in chunks of %d: %.5f of the rms off" % (chunk, float((z - y).float().norm() / y.float().norm())), flush=True)


if __name__ == "__main__":
    main()
