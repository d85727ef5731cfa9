"""Trains a small network with every operator of the package: MXFP4 products
forward and backward, the projected step on the weights, AdamW on the other
parameters, one clipping norm over all gradients.

    python examples/train_mxfp4.py [--steps 200]

The network reads a token's embedding, scales it by a gain and takes it through
two linear layers with a ReLU between them; it learns a fixed random network of
the same shape (synthetic data).  The weights are fp32 and quantised, by rows and
by columns, after each step; activations and their gradients are quantised as
they come.  No quantity is read back to the host but the printed losses.
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_15037_gb300 as M  # noqa: E402

VOCAB, WIDTH, HIDDEN, TOKENS, RANK = 512, 256, 512, 1024, 64


class Net:
    def __init__(self, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def draw(*shape, scale):
            return torch.randn(*shape, generator=gen, device="cuda") * scale
        # weights: the projected step owns them; the rest: AdamW, with 8-bit moments for
        # the embedding and a bf16 copy of the bias for the forward pass
        self.group = M.MoaraGroup(block_size=64, clip_norm=1.0, scale=1.0, refresh_interval=50)
        for m, n in ((HIDDEN, WIDTH), (WIDTH, HIDDEN)):
            self.group.add(m, n, RANK, "bf16", W0=draw(m, n, scale=n ** -0.5))
        self.embed, self.gain = draw(VOCAB, WIDTH, scale=1.0), torch.ones(WIDTH, device="cuda")
        self.bias = torch.zeros(WIDTH, device="cuda")
        self.bias16 = self.bias.bfloat16()
        self.rest = M.AdamWGroup(seed=seed)
        self.rest.add(self.embed, state="block8", weight_decay=0.01)
        self.rest.add(self.gain)
        self.rest.add(self.bias, copy=self.bias16)
        self.fp4 = M.Fp4Group()
        self.quantize_weights()

    def quantize_weights(self):
        self.ops = [self.fp4.quantize(b.W, rows=True, cols=True) for b in self.group.modules]

    def forward(self, tokens):
        (w1, _), (w2, _) = self.ops
        e = self.embed[tokens]
        x, self.xt = self.fp4.quantize(e * self.gain, rows=True, cols=True)
        a = self.fp4.product(x, w1, dtype=torch.float32)
        h, self.ht = self.fp4.quantize(a.relu(), rows=True, cols=True)
        self.saved = tokens, e, a
        return self.fp4.product(h, w2, dtype=torch.float32) + self.bias16

    def backward(self, dy):
        """Gradients of the two weights (bf16) and of embedding, gain and bias."""
        (_, w1t), (_, w2t) = self.ops
        tokens, e, a = self.saved
        d, dt = self.fp4.quantize(dy, rows=True, cols=True)
        dw2 = self.fp4.product(dt, self.ht)
        da = self.fp4.product(d, w2t, dtype=torch.float32) * (a > 0)
        d, dt = self.fp4.quantize(da, rows=True, cols=True)
        dw1 = self.fp4.product(dt, self.xt)
        dx = self.fp4.product(d, w1t, dtype=torch.float32)
        de = torch.zeros_like(self.embed).index_add_(0, tokens, dx * self.gain)
        return [dw1, dw2], [de, (dx * e).sum(0), dy.sum(0)]

    def step(self, grads, others, t, lr):
        # one norm over all gradients: that of the others joins the grouped step's, whose
        # coefficient scales both
        norm = self.rest.grad_norm(others)
        self.group.set_clip_extra(norm[:1])
        self.group.step(grads, t, lr, auto_refresh=True, stream=torch.cuda.current_stream().cuda_stream)
        self.rest.step(others, t, lr, grad_scale=self.group.clip_state()[1:])
        self.quantize_weights()

    def close(self):
        self.group.close(), self.rest.close(), self.fp4.close()


def train(steps=200, lr=3e-3, seed=0, report=None):
    """Losses of the first and the last ten steps, averaged."""
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    teach = [torch.randn(*s, generator=gen, device="cuda") * s[1] ** -0.5
             for s in ((VOCAB, WIDTH), (HIDDEN, WIDTH), (WIDTH, HIDDEN))]
    teach[0] *= WIDTH ** 0.5
    net = Net(seed)
    net.embed.copy_(teach[0] + 0.3 * torch.randn(VOCAB, WIDTH, generator=gen, device="cuda"))
    losses = []
    for t in range(1, steps + 1):
        tokens = torch.randint(0, VOCAB, (TOKENS,), generator=gen, device="cuda")
        want = (teach[0][tokens] @ teach[1].t()).relu() @ teach[2].t()
        y = net.forward(tokens)
        diff = y - want
        losses.append(diff.square().mean())
        grads, others = net.backward(diff * (2 / diff.numel()) * WIDTH)
        net.step(grads, others, t, lr * (1 - (t - 1) / steps))
        if report and (t == 1 or t % report == 0):
            print(f"step {t}: loss {losses[-1].item():.4f}")
    if net.group.status() or net.fp4.status():
        raise RuntimeError("a kernel reported an error")
    net.close()
    losses = torch.stack(losses)
    return losses[:10].mean().item(), losses[-10:].mean().item()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    first, last = train(ap.parse_args().steps, report=20)
    print(f"loss of the first ten steps {first:.4f}, of the last ten {last:.4f}")
