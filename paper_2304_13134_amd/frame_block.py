"""A feed-forward block between an encoder's frames and the lattice, from the calls of ``binding``: how the residual norm,
the products and the activations kept in 8 bits go together in training and in recognition.

    python -m paper_2304_13134_amd.frame_block        # trains a small one through the globally normalised loss

Training keeps, beside the frames themselves, the norm's result and what the activation is applied to, both in 8 bits: 8.25
bits a value with the scales instead of 16, for gradients that differ by the codes' rounding (0.8 % of a kept value's rms
with int8, of normal values).  Recognition runs the products on 8-bit operands.
"""
from __future__ import annotations

import torch

from . import binding as lb


class FrameBlock:
    """y = x + act(norm(x) w1^T + b1) w2^T + b2 on frames [B, T, H] in bfloat16, of which lengths [B] exist."""

    def __init__(self, hidden, inner, activation="silu", device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.activation = activation
        self.gain = torch.ones(hidden, device=device)
        self.w1 = (torch.randn(inner, hidden, generator=g, device=device) * hidden ** -0.5).bfloat16()
        self.b1 = torch.zeros(inner, device=device)
        self.w2 = (torch.randn(hidden, inner, generator=g, device=device) * inner ** -0.5).bfloat16()
        self.b2 = torch.zeros(hidden, device=device)

    def parameters(self):
        return {"gain": self.gain, "w1": self.w1, "b1": self.b1, "w2": self.w2, "b2": self.b2}

    def forward(self, x, lengths=None, keep=torch.int8):
        """(y, what backward() needs)"""
        n = lb.last_residual_norm(x, self.gain, lengths=lengths, dtype=x.dtype, keep=keep)
        a, h = lb.last_product(n.y, self.w1, self.b1, self.activation, lengths=lengths, keep=keep)
        y, _ = lb.last_product(a, self.w2, self.b2, residual=x, lengths=lengths)
        return y, (x, n.inv, n.kept, h)

    def backward(self, dy, saved, lengths=None):
        """(dx, gradients by name) of dy in bfloat16; weights' gradients in float32."""
        x, inv, n, h = saved
        dw2, db2 = lb.last_product_grad_weight(dy, h, self.activation, lengths=lengths)
        dh = lb.last_product_grad_input(dy, self.w2, h, self.activation, lengths=lengths)
        dw1, db1 = lb.last_product_grad_weight(dh, n, lengths=lengths)
        dn = lb.last_product_grad_input(dh, self.w1, lengths=lengths)
        dx, dgain = lb.last_residual_norm_grad(dn, x, self.gain, inv, ds=dy, lengths=lengths)
        return dx, {"gain": dgain, "w1": dw1, "b1": db1, "w2": dw2, "b2": db2}

    def eight_bits(self):
        """The weights in 8 bits, for recognise()."""
        return lb.last_keep(self.w1, torch.float8_e4m3fn), lb.last_keep(self.w2, torch.float8_e4m3fn)

    def recognise(self, x, weights, lengths=None):
        """forward() on 8-bit operands: `weights` from eight_bits()."""
        e4m3 = torch.float8_e4m3fn
        n = lb.last_residual_norm(x, self.gain, lengths=lengths, keep=e4m3)
        a, _ = lb.last_product(n.kept, weights[0], self.b1, self.activation, lengths=lengths, dtype=e4m3)
        y, _ = lb.last_product(a, weights[1], self.b2, residual=x, lengths=lengths, dtype=x.dtype)
        return y


class FrameModel:
    """A block, a norm and the shared-embedding weight function of the lattice (two-label contexts, V labels)."""

    def __init__(self, hidden=128, inner=512, V=8, device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed + 1)
        self.block = FrameBlock(hidden, inner, device=device, seed=seed)
        self.gain = torch.ones(hidden, device=device)
        self.e = (0.5 * torch.randn(1 + V + V * V, hidden, generator=g, device=device)).bfloat16()
        self.W = (torch.randn(hidden, V + 1, generator=g, device=device) * hidden ** -0.5).bfloat16()

    def loss_and_gradients(self, x, lengths, refs, ref_lengths):
        """(loss [B], gradients by parameter) of frames x [B, T, H]."""
        return self.loss_of_frames(x, lengths, refs, ref_lengths)[:2]

    def loss_of_frames(self, x, lengths, refs, ref_lengths):
        """(loss [B], gradients by parameter, gradient of x)"""
        y, saved = self.block.forward(x, lengths)
        f = lb.last_residual_norm(y, self.gain, lengths=lengths)
        dist, num, (df, de, dW) = lb.last_globally_normalized_loss(lb.SharedEmb(f.y, self.e, self.W), lengths, refs, ref_lengths, order=2)
        dy, dgain = lb.last_residual_norm_grad(df, y, self.gain, f.inv, lengths=lengths)
        dx, grads = self.block.backward(dy, saved, lengths)
        return dist - num, [(self.gain, dgain), (self.e, de), (self.W, dW)] + [(p, grads[k]) for k, p in self.block.parameters().items()], dx

    def step(self, x, lengths, refs, ref_lengths, rate=0.002):
        """One step down the gradient; the mean loss before it."""
        loss, gradients = self.loss_and_gradients(x, lengths, refs, ref_lengths)
        lb.check_item_status()
        for p, g in gradients:
            p.copy_(p.float() - rate / len(lengths) * g)
        return float(loss.mean())


def synthetic_batch(B=8, T=64, hidden=128, V=8, U=10, device="cuda", seed=0):
    """Frames whose first columns tell the label that is spoken, and the labels."""
    g = torch.Generator().manual_seed(seed)
    refs = torch.randint(1, V + 1, (B, U), generator=g, dtype=torch.int32)
    lengths = torch.randint(3 * T // 4, T + 1, (B,), generator=g, dtype=torch.int32)
    x = torch.randn(B, T, hidden, generator=g)
    for b in range(B):
        at = torch.linspace(0, int(lengths[b]) - 1, U).long()
        x[b, at, refs[b].long() - 1] += 6.0
    return x.bfloat16().to(device), lengths.to(device), refs.to(device), torch.full((B,), U, dtype=torch.int32, device=device)


def main(steps=30):
    model = FrameModel()
    x, lengths, refs, ref_lengths = synthetic_batch()
    for i in range(steps):
        loss = model.step(x, lengths, refs, ref_lengths)
        if i % 5 == 0 or i == steps - 1:
            print("step %2d  loss %.3f" % (i, loss), flush=True)
    y, _ = model.block.forward(x, lengths)
    z = model.block.recognise(x, model.block.eight_bits(), lengths)
    print("8-bit products: %.4f of the rms off" % float((z - y).float().norm() / y.float().norm()), flush=True)


if __name__ == "__main__":
    main()
