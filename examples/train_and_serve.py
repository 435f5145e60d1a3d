"""Trains one MoE layer and serves tokens from it: the training step (forward, backward,
orthogonalised updates of every weight matrix, the loss-free bias) and decoding one token or a
few at a time, all on the library's kernels.

    python examples/train_and_serve.py [steps]

The task is a regression: a layer of random weights (the teacher) gives the targets for random
tokens, and another one of the same sizes learns them."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_17402_gb300 import moevie  # noqa: E402

D, E, K, H, HS, TOKENS = 256, 16, 4, 136, 128, 4096


def random_layer(gen):
    def matrix(*shape):
        return torch.randn(*shape, generator=gen, device="cuda") * shape[-2] ** -0.5

    def bf16(w):
        return moevie.moevie_pad_rows(w.to(torch.bfloat16))

    return moevie.LayerWeights(W_r=matrix(D, E), b=torch.zeros(E, device="cuda"), W1=bf16(matrix(E, D, H)),
                               W2=bf16(matrix(E, H, D)), k=K, Ws1=bf16(matrix(D, HS)), Ws2=bf16(matrix(HS, D)))


def tokens(n, gen):
    return torch.randn(n, D, generator=gen, device="cuda").to(torch.bfloat16)


class Muon:
    """fp32 master weights, momentum and the scratch of one weight tensor of the layer."""

    def __init__(self, w):
        self.bf16 = w   # the layer's own tensor, written by every step
        self.master = moevie.moevie_pad_rows(w.float())
        self.momentum = moevie.moevie_pad_rows(torch.zeros_like(w, dtype=torch.float32))
        self.ws = moevie.OrthoWorkspace(w.shape[0] if w.dim() == 3 else 1, *w.shape[-2:])

    def step(self, grad, lr):
        moevie.moevie_muon_update(self.master, self.momentum, grad, self.ws, lr, W_bf16=self.bf16)


def train(layer, teacher, steps, gen, lr=0.02):
    """Returns the loss (mean squared error over the target's mean square) of every step."""
    fwd = moevie.Workspace(TOKENS, D, E, K, H, HS)
    bwd = moevie.BackwardWorkspace(TOKENS, D, E, K, H, HS)
    muon = {name: Muon(getattr(layer, name)) for name in ("W1", "W2", "Ws1", "Ws2")}
    losses = []
    for step in range(steps):
        x = tokens(TOKENS, gen)
        want = moevie.moevie_moe_forward(teacher, x, fwd).float()
        y, routing = moevie.moevie_moe_forward(layer, x, fwd, routing=True)
        err = y.float() - want
        losses.append(float((err ** 2).mean() / (want ** 2).mean()))
        grads = moevie.moevie_moe_backward(layer, x, (err / TOKENS).to(torch.bfloat16), routing["idx"], bwd)
        now = lr * (1 - step / steps)
        for name, opt in muon.items():
            opt.step(grads["d" + name], now)
        layer.W_r -= now * grads["dW_r"]
        moevie.moevie_update_bias(routing["counts"], layer.b, 1e-3, fwd)
    for ws in (fwd, bwd, *(m.ws for m in muon.values())):
        assert moevie.moevie_get_device_status(ws)[0] == 0
    return losses


def serve(layer, x):
    """The tokens one at a time, then up to FEW_MAX_TOKENS at a time."""
    ws = moevie.FewWorkspace(moevie.FEW_MAX_TOKENS, D, E, K, H, HS)
    one = torch.cat([moevie.moevie_moe_few(layer, x[t:t + 1], ws) for t in range(len(x))])
    few = torch.cat([moevie.moevie_moe_few(layer, x[t:t + moevie.FEW_MAX_TOKENS], ws)
                     for t in range(0, len(x), moevie.FEW_MAX_TOKENS)])
    assert moevie.moevie_get_device_status(ws)[0] == 0
    return one, few


def main(steps=150):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    teacher, layer = random_layer(gen), random_layer(gen)
    losses = train(layer, teacher, steps, gen)
    x = tokens(100, gen)
    one, few = serve(layer, x)
    batch = moevie.moevie_moe_forward(layer, x, moevie.Workspace(len(x), D, E, K, H, HS))

    def off(y):
        return float((y.float() - batch.float()).norm() / batch.float().norm())

    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {steps} steps; served one at a time and {min(64, len(x))} at a "
          f"time: {off(one):.1e} and {off(few):.1e} from the batch forward")
    return losses, off(one), off(few)


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:2]))
