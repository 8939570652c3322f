"""Tunes the router of one MoE layer whose experts stay as they are.

    python examples/tune_router.py [--steps 60] [--tokens 3000] [--seed 0]

The layer (64 experts of which a token takes 6, 2 shared experts) starts with a router that a bias skews towards a few experts, and
learns to give the outputs that the same experts give under another router, while the balance loss spreads the tokens.  A tenth of the
tokens is padding.  Each step is one accumulated batch:

    route (with logits) -> permute -> grouped_ffn -> combine            the layer, stage by stage
    dout = gradient of the mean squared error
    combine_backward -> balance_loss -> route_backward                  gradients of gate matrix and bias
    clip_gradients                                                      over all tuned tensors
    an update of the fp32 master copies in torch
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2503_09716_amd import Moe, make_shape  # noqa: E402

BALANCE_COEF, Z_COEF, MAX_NORM = 1e-2, 1e-4, 1.0


class Layer:
    """An MoE layer's weights and the buffers of one batch, kept from step to step."""

    def __init__(self, moe: Moe, shape, generator):
        T, H, F, E, k, Ns = shape.T, shape.H, shape.F, shape.E, shape.top_k, shape.num_shared
        self.moe, self.shape = moe, shape

        def normal(n, std):
            return torch.empty(n, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=generator)
        self.w = moe.pack_experts([normal((H, F), H ** -0.5) for _ in range(E + Ns)], [normal((H, F), H ** -0.5) for _ in range(E + Ns)],
                                  [normal((F, H), F ** -0.5) for _ in range(E + Ns)])
        i32 = dict(dtype=torch.int32, device="cuda")
        f32 = dict(dtype=torch.float32, device="cuda")
        self.topk_idx, self.topk_w, self.logits = torch.empty((T, k), **i32), torch.empty((T, k), **f32), torch.empty((T, E), **f32)
        self.offsets, self.perm, self.inv_perm, self.row_token = (torch.empty(n, **i32) for n in (E + 1, T * k, T * k, T * k))
        self.y_perm, self.y_shared = torch.empty((T * k, H), **f32), torch.empty((T, H), **f32) if Ns else None
        self.out = torch.empty((T, H), **f32)
        self.h, self.ws, self.back = moe.new_h_scratch(shape), moe.new_workspace(shape), moe.new_backward_workspace(shape)
        self.dtopk_w, self.dlogits = torch.empty((T, k), **f32), torch.empty((T, E), **f32)
        self.counts, self.loss = torch.empty(E, **i32), torch.empty(2, **f32)
        self.dwg, self.dbias = torch.empty((H, E), **f32), torch.empty(E, **f32)

    def forward(self, x, wg, bias):
        m, s = self.moe, self.shape
        m.route(s, x, wg, bias, self.topk_idx, self.topk_w, self.logits, self.ws)
        m.permute(s, x, self.topk_idx, None, self.offsets, self.perm, self.inv_perm, self.row_token, self.ws)
        m.grouped_ffn(s, None, self.row_token, x, self.offsets, *self.w, self.h, self.y_perm, self.y_shared, self.ws)
        m.combine(s, self.y_perm, self.inv_perm, self.topk_w, self.y_shared, self.out)
        return self.out

    def backward(self, x, wg, keep, dout):
        """Gradients of <dout, out> and of the balance losses in dwg and dbias.  Nothing before the layer is tuned: no gradient of x."""
        m, s = self.moe, self.shape
        m.combine_backward(s, dout, self.y_perm, self.inv_perm, self.topk_w, self.dtopk_w, None)
        m.balance_loss(s, self.logits, self.topk_idx, keep, BALANCE_COEF, Z_COEF, self.counts, self.loss, self.dlogits, self.back)
        m.route_backward(s, x, wg, self.logits, self.topk_idx, self.dtopk_w, self.dlogits, keep, None, self.dwg, self.dbias, False, self.back)


def tune(steps=60, tokens=3000, seed=0, lr=0.02, say=print):
    """Runs the steps; per step the mean squared error, the balance loss and the norm of the gradients before clipping."""
    moe = Moe(0)
    moe.set_option("out_fp32", 1)   # out and dout in fp32
    gen = torch.Generator(device="cuda").manual_seed(seed)
    shape = make_shape(tokens, 256, 192, 64, 6, 2, renormalize=False, routed_scale=8.0)
    T, H, E = shape.T, shape.H, shape.E
    layer = Layer(moe, shape, gen)
    x = torch.empty((T, H), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    keep = torch.rand(T, device="cuda", generator=gen) >= 0.1
    teacher = torch.empty((H, E), dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.06, generator=gen)
    target = layer.forward(x, teacher, None).clone()

    gate = teacher.float() + torch.empty((H, E), device="cuda").normal_(0.0, 0.03, generator=gen)   # fp32 masters
    bias = -1.1 * torch.log(torch.arange(1, E + 1, device="cuda").float())
    params, grads = [gate, bias], [layer.dwg, layer.dbias]
    first, second = [torch.zeros_like(p) for p in params], [torch.zeros_like(p) for p in params]
    clipped = [torch.empty_like(g) for g in grads]
    listed, norm = moe.gradient_list(grads, clipped), torch.empty(1, device="cuda")
    n = keep.sum().clamp(min=1)
    history = []
    for step in range(1, steps + 1):
        wg = gate.bfloat16()
        off = torch.where(keep[:, None], layer.forward(x, wg, bias) - target, torch.zeros_like(target))
        layer.backward(x, wg, keep, off * (2.0 / (n * H)))
        moe.clip_gradients(listed, MAX_NORM, norm)
        for p, g, m, v in zip(params, clipped, first, second):
            m.lerp_(g, 0.1)
            v.lerp_(g * g, 0.01)
            p -= lr * (m / (1 - 0.9 ** step)) / ((v / (1 - 0.99 ** step)).sqrt() + 1e-8)
        history.append(torch.stack([off.square().sum() / (n * H), layer.loss[0], norm[0]]))
        if step == 1 or step % 10 == 0:
            mse, balance, size = history[-1].tolist()
            say("step %3d  error %.5f  balance %.3f  most tokens on an expert %d  norm %.4f" % (step, mse, balance, int(layer.counts.max()), size))
    out = torch.stack(history).cpu()
    moe.close()
    return out


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--tokens", type=int, default=3000)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    tune(a.steps, a.tokens, a.seed)
