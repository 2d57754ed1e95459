"""A residual block x + fc2(relu(fc1(norm(x)))) trained in 8-bit floating point under masks of 128 x 128 blocks.

What a step keeps for its backward pass is 8 bits a value: the norm leaves its result as the codes that fc1 reads, and
relu's output is kept as the codes that fc2 reads; the same two checkpoints then give both layers' weights' gradients and
the gate of the relu.  The masks keep the heavier half of each layer's blocks.  Run it on a GPU: `python examples/train_f8.py`.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2407_09453_amd as bsp


def heavier_half(W):
    """The mask of the blocks of W whose L2 norm is at least the median."""
    O, I = W.shape
    blocks = W.view(O // 128, 128, I // 128, 128).square().sum((1, 3))
    return (blocks >= blocks.median()).to(torch.uint8)


class Block:
    def __init__(self, width, hidden, gen):
        self.master = {"W1": torch.randn(hidden, width, generator=gen, device="cuda") * (2 / width) ** 0.5,
                       "W2": torch.randn(width, hidden, generator=gen, device="cuda") * (1 / hidden) ** 0.5,
                       "b1": torch.zeros(hidden, device="cuda"), "b2": torch.zeros(width, device="cuda"),
                       "w": torch.ones(width, device="cuda"), "b": torch.zeros(width, device="cuda")}
        m = self.master
        self.fc1 = bsp.BspLayerF8(m["W1"], heavier_half(m["W1"]), bias=m["b1"])
        self.fc2 = bsp.BspLayerF8(m["W2"], heavier_half(m["W2"]), bias=m["b2"])

    def forward(self, x):
        """(y, what the backward pass needs)."""
        n, mean, rstd = bsp.layer_norm(x, self.master["w"], self.master["b"], code="e4m3")
        h = bsp.save8(self.fc1.fc(n, relu=True))
        return self.fc2.fc(h, residual=x), (x, mean, rstd, n, h)

    def backward(self, dy, kept):
        """(dx, gradients of the master values)."""
        x, mean, rstd, n, h = kept
        g = {}
        g["W2"], g["b2"] = self.fc2.grad_weight(dy, h)
        dh = self.fc2.grad_input(dy, relu_of=h)
        g["W1"], g["b1"] = self.fc1.grad_weight(dh, n)
        dx, g["w"], g["b"] = bsp.layer_norm_grad(self.fc1.grad_input(dh), x, mean, rstd, self.master["w"])
        return dx + dy, g

    def update(self, g, rate):
        """A plain gradient step on the master values; the layers take the new weights as codes."""
        for k, v in g.items():
            self.master[k] -= rate * v
        for fc, W, b in ((self.fc1, "W1", "b1"), (self.fc2, "W2", "b2")):
            fc.update(self.master[W], bias=self.master[b])


def train(steps=40, rows=512, width=512, hidden=1024, rate=0.05, seed=0):
    """Learns another such block's outputs; the mean squared error of every step."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    teacher, block = Block(width, hidden, gen), Block(width, hidden, gen)
    losses = []
    for _ in range(steps):
        x = torch.randn(rows, width, generator=gen, device="cuda").to(torch.bfloat16)
        want, _ = teacher.forward(x)
        y, kept = block.forward(x)
        err = y.float() - want.float()
        losses.append(float(err.square().mean()))
        _, g = block.backward((err * (2 / rows)).to(torch.bfloat16), kept)
        block.update(g, rate)
    return block, losses


if __name__ == "__main__":
    block, losses = train()
    print("mean squared error: " + " ".join("%.3f" % v for v in losses[::5] + losses[-1:]))
    x = torch.randn(1, 512, device="cuda").to(torch.bfloat16)
    print("one row served:", block.forward(x)[0][0, :4].tolist())
