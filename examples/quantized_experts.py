"""Keeps the experts of one MoE layer in MXFP4 and runs a long batch and single steps on them.

    python examples/quantized_experts.py [--tokens 3000] [--steps 20] [--seed 0]

The long batch goes stage by stage, with activations in MXFP4, too:

    route -> permute -> mx_quantize of x -> mx_grouped_product (gate and up) -> mx_quantize of h -> mx_grouped_product (down) -> combine

and a few tokens through the whole layer in one call (layer_few), with activations as they are.  Prints how far both are from
the layer on the experts' values, and what they take.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2503_09716_amd import Moe, make_shape, workspace_bytes  # noqa: E402


class QuantizedLayer:
    """The weights of a layer in MXFP4.  Shared experts are summed, so in a long batch they are one expert of their width together, packed a second time; the layer for few
    tokens takes them one by one."""

    def __init__(self, moe: Moe, wg, w1, w3, w2, k, num_shared):
        self.moe, self.wg, self.k, self.num_shared = moe, wg, k, num_shared
        self.H, self.F, self.E = w1[0].shape[0], w1[0].shape[1], len(w1) - num_shared
        packed = [[moe.mx_pack_weight(w) for w in ws] for ws in (w1, w3, w2)]
        self.all = moe.weight_list(*packed)
        self.routed = moe.weight_list(*[ws[:self.E] for ws in packed])
        if num_shared:
            joined = (torch.cat(w1[self.E:], dim=1), torch.cat(w3[self.E:], dim=1), torch.cat(w2[self.E:], dim=0))
            shared = [[moe.mx_pack_weight(w.contiguous())] for w in joined]
            self.shared_up, self.shared_down = moe.weight_list(*shared[:2]), moe.weight_list(shared[2])

    def values(self):
        """The matrices as the layer has them, in bf16."""
        sizes = ((self.H, self.F), (self.H, self.F), (self.F, self.H))
        return [[self.moe.mx_unpack_weight(w, torch.empty(s, dtype=torch.bfloat16, device=w.device)) for w in ws] for ws, s in zip(self.all.weights, sizes)]

    def _ffn(self, q, row_index, offsets, up, down, down_at, rows, F):
        m = self.moe
        ws = m.new_mx_workspace(rows, up.struct.experts)
        h = torch.empty((rows, F), dtype=torch.bfloat16, device="cuda")
        m.mx_grouped_product(q, row_index, offsets, up, h, ws, gated=True)
        hq = m.new_mx_rows(rows, F)
        m.mx_quantize(h, hq)
        y = torch.empty((rows, self.H), device="cuda")
        m.mx_grouped_product(hq, None, offsets, down, y, ws, first=down_at)
        return y

    def long_batch(self, x):
        m, T, k, E = self.moe, x.shape[0], self.k, self.E
        s = make_shape(T, self.H, self.F, E, k, self.num_shared)
        i32 = dict(dtype=torch.int32, device="cuda")
        idx, w = torch.empty((T, k), **i32), torch.empty((T, k), device="cuda")
        offsets, perm, inv_perm, row_token = (torch.empty(n, **i32) for n in (E + 1, T * k, T * k, T * k))
        ws = m.new_workspace(s)
        m.route(s, x, self.wg, None, idx, w, None, ws)
        m.permute(s, x, idx, None, offsets, perm, inv_perm, row_token, ws)
        q = m.new_mx_rows(T, self.H)
        m.mx_quantize(x, q)
        y = self._ffn(q, row_token, offsets, self.routed, self.routed, 2, T * k, self.F)
        y_shared = None
        if self.num_shared:
            y_shared = self._ffn(q, None, torch.tensor([0, T], **i32), self.shared_up, self.shared_down, 0, T, self.F * self.num_shared)
        out = torch.empty((T, self.H), dtype=m.out_dtype, device="cuda")
        m.combine(s, y, inv_perm, w, y_shared, out)
        return out

    def few(self, x):
        m = self.moe
        s = make_shape(x.shape[0], self.H, self.F, self.E, self.k, self.num_shared)
        out = torch.empty(x.shape, dtype=m.out_dtype, device="cuda")
        m.layer_few(s, x, self.wg, None, self.all, out, m.new_few_workspace(s))
        return out


def relative(a, b):
    return ((a.float() - b.float()).square().mean() / b.float().square().mean()).sqrt().item()


def main(argv=None):
    p = argparse.ArgumentParser()
    p.add_argument("--tokens", type=int, default=3000)
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args(argv)
    H, F, E, k, shared = 1024, 704, 32, 4, 2
    gen = torch.Generator(device="cuda").manual_seed(a.seed)

    def normal(shape, std):
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, std, generator=gen)
    moe = Moe(0)
    w = [[normal(s, s[0] ** -0.5) for _ in range(E + shared)] for s in ((H, F), (H, F), (F, H))]
    layer = QuantizedLayer(moe, normal((H, E), 2 * H ** -0.5), *w, k, shared)
    values = [[moe.pack_weight(m) for m in ms] for ms in layer.values()]

    def reference(x):
        s = make_shape(x.shape[0], H, F, E, k, shared)
        out = torch.empty(x.shape, dtype=torch.bfloat16, device="cuda")
        moe.layer(s, x, layer.wg, None, *values, out, torch.empty(workspace_bytes(s), dtype=torch.uint8, device="cuda"))
        return out
    x = normal((a.tokens, H), 1.0)
    result = {"long": relative(layer.long_batch(x), reference(x)), "few": relative(layer.few(x[:5]), reference(x[:5]))}
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for name, call in (("long_us", lambda: layer.long_batch(x)), ("few_us", lambda: layer.few(x[:5]))):
        call()
        start.record()
        for _ in range(a.steps):
            call()
        end.record()
        end.synchronize()
        result[name] = start.elapsed_time(end) * 1e3 / a.steps
    moe.close()
    print("relative difference from the layer on the experts' values: %(long).4f (activations in MXFP4), %(few).4f; %(long_us).0f us, %(few_us).0f us" % result)
    return result


if __name__ == "__main__":
    main()
