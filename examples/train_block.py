"""A training step of residual blocks around the MoE layer, on the library's kernels: the norms, gates
and residual stream, the layers, the balance loss of their routers, and a backward pass that reads the
rows it needs from 8-bit checkpoints.

    python examples/train_block.py [steps]

Two blocks, post-norm of the layer's output and a gate for each image:
    u_i = N_pre(r_i),   r_(i+1) = r_i + gate * N_post(layer_i(u_i)).
Their last stream is held against a target; the gates, the norms' weights and the routers learn."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_17402_gb300 import moevie  # noqa: E402

D, E, K, H, BLOCKS = 256, 16, 4, 136, 2
IMAGES, TOKENS, PADDED = 5, 1200, 1280   # rows behind the last image are padding
COEF = 0.01                              # of the balance loss


class Blocks:
    """Weights, runs of rows (images) and scratch."""

    def __init__(self, gen):
        def matrix(*shape, std=None):
            return torch.randn(*shape, generator=gen, device="cuda") * (shape[-2] ** -0.5 if std is None else std)

        def bf16(w):
            return moevie.moevie_pad_rows(w.to(torch.bfloat16))

        ends = torch.linspace(0, TOKENS, IMAGES + 1).to(torch.int32)
        ends[1:-1] += torch.tensor([17, -30, 8, 1], dtype=torch.int32)
        self.seg = ends.cuda()
        self.layers = [moevie.LayerWeights(W_r=matrix(D, E), b=torch.zeros(E, device="cuda"), W1=bf16(matrix(E, D, H)),
                                           W2=bf16(matrix(E, H, D)), k=K) for _ in range(BLOCKS)]

        def norm(pre, post):
            both = {"w_pre": torch.ones(D, device="cuda"), "b_pre": torch.zeros(D, device="cuda")} if pre else {}
            if post:
                both |= {"w_post": torch.ones(D, device="cuda"), "gate": 0.3 + matrix(IMAGES, D, std=0.1)}
            return moevie.ResidualNorm(D, pre, post, seg=self.seg, **both)

        # the first norm, then what lies between layers, then the last join
        self.norms = [norm("layer", None)] + [norm("layer", "rms") for _ in range(BLOCKS - 1)] + [norm(None, "rms")]
        self.fwd = moevie.Workspace(PADDED, D, E, K, H)
        self.bwd = moevie.BackwardWorkspace(PADDED, D, E, K, H)
        self.norm_ws = moevie.ResidualNormWorkspace(PADDED, D, IMAGES)
        self.balance_ws = moevie.BalanceWorkspace(PADDED, E, K, IMAGES)

    def forward(self, r):
        """r fp32 [PADDED, D] -> the last stream, and what the backward keeps of each block.  Rows of padding go
        through the layers (as zeros), and nowhere else."""
        kept = []
        out = self._buffers(self.norms[0], join=False)
        moevie.moevie_residual_norm(self.norms[0], r, None, self.norm_ws, out=out)
        balance = 0.0
        for layer, norms in zip(self.layers, self.norms[1:]):
            f, routing = moevie.moevie_moe_forward(layer, out.u, self.fwd, routing=True)
            s = moevie.moevie_router_logits(out.u, layer.W_r, self.fwd)
            ds = moevie.BalanceOut.empty(PADDED, E, IMAGES)
            ds.ds.zero_()   # rows of padding have no gradient
            moevie.moevie_balance_loss(s, routing["idx"], self.balance_ws, COEF, seg=self.seg, out=ds)
            balance = balance + ds.loss
            after = self._buffers(norms, save=True)
            after.r = torch.zeros_like(r)
            moevie.moevie_residual_norm(norms, r, f, self.norm_ws, out=after)
            # of r and f only the 8-bit checkpoints stay; u is formed again from that of r
            kept.append((routing["idx"], ds.ds, out.stats_pre, after))
            out, r = after, after.r
        return r, balance, kept

    def _buffers(self, norms, save=False, join=True):
        out = moevie.ResidualNormOut.empty(norms, PADDED, torch.float32, save, join)
        if out.u is not None:
            out.u.zero_()
        return out

    def backward(self, dr, kept):
        """dr fp32 [PADDED, D], the gradient of the last stream -> that of r, and of the weights, block by block."""
        grads = [None] * (BLOCKS + 1)
        du, r1 = None, None   # of the norm behind the block in hand, and its rows
        layers = [None] * BLOCKS
        for i in reversed(range(BLOCKS)):
            idx, ds, stats_pre, after = kept[i]
            grads[i + 1] = self._join_back(self.norms[i + 1], dr, du, r1, after)
            dr = grads[i + 1].dr
            first = moevie.ResidualNorm(D, self.norms[i].pre, w_pre=self.norms[i].w_pre, b_pre=self.norms[i].b_pre,
                                        seg=self.seg)
            again = self._buffers(first, join=False)
            u = moevie.moevie_residual_norm(first, after.save_r, None, self.norm_ws, out=again).u
            layers[i] = moevie.moevie_moe_backward(self.layers[i], u, grads[i + 1].df, idx, self.bwd, ds=ds)
            du, r1 = layers[i]["dx"], after.save_r
        out = moevie.ResidualNormGrads.empty(self.norms[0], PADDED, torch.float32, join=False)
        grads[0] = moevie.moevie_residual_norm_backward(self.norms[0], dr, du, r1, None, kept[0][2], None, self.norm_ws,
                                                        out=out)
        return grads, layers

    def _join_back(self, norms, dr, du, r1, after):
        out = moevie.ResidualNormGrads.empty(norms, PADDED, torch.float32)
        out.dr.zero_()
        out.df.zero_()
        return moevie.moevie_residual_norm_backward(norms, dr, du, r1, after.save_f, after.stats_pre, after.stats_post,
                                                    self.norm_ws, out=out)

    def loss(self, r, target):
        """Mean squared error of the images' rows plus the balance loss, its gradient by the last stream, and what
        the backward keeps."""
        got, balance, kept = self.forward(r)
        err = torch.zeros_like(got)
        err[:TOKENS] = got[:TOKENS] - target[:TOKENS]
        return (err ** 2).sum() / (TOKENS * D) + balance, 2 * err / (TOKENS * D), kept

    def weights(self, grads, layers):
        """Every learning tensor with its gradient."""
        for norms, g in zip(self.norms, grads):
            for name in ("w_pre", "b_pre", "w_post", "gate"):
                if getattr(norms, name) is not None and getattr(g, "d" + name) is not None:
                    yield getattr(norms, name), getattr(g, "d" + name)
        for layer, g in zip(self.layers, layers):
            yield layer.W_r, g["dW_r"]


def inputs(gen):
    r = torch.zeros(PADDED, D, device="cuda")
    r[:TOKENS] = torch.randn(TOKENS, D, generator=gen, device="cuda")
    target = torch.randn(PADDED, D, generator=gen, device="cuda")
    return r, target


def main(steps=20, lr=30.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    blocks = Blocks(gen)
    losses = []
    r, target = inputs(gen)
    for _ in range(steps):
        loss, dr, kept = blocks.loss(r, target)
        losses.append(float(loss))
        for w, g in blocks.weights(*blocks.backward(dr, kept)):
            w -= lr * g
    for ws in (blocks.fwd, blocks.bwd, blocks.norm_ws, blocks.balance_ws):
        assert moevie.moevie_get_device_status(ws)[0] == 0
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {steps} steps")
    return losses


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:2]))
