"""A stack of routed residual blocks on the library: each block's feed-forward layer is one of
several sparse FFN experts per token choice.

Between two blocks one sfl_norm_forward does the norm, gate and residual sum of the block behind and
the norm of the block ahead; inside a block the router picks the experts, sfl_expert_dispatch brings
the rows into expert order, every expert runs sfl_ffn_forward on its rows, and sfl_expert_combine
brings them back. `backward` walks the same way back and leaves fp32 gradients, which `step` clips
by their global norm and applies. torch is used for memory and for the router's two small matrix
products.

    python examples/routed_block.py --tokens 2048 --width 1024 --hidden 4096 --experts 8 --steps 10
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2603_23198_amd import binding as b  # noqa: E402


class RoutedStack:
    """`layers` blocks of width d; each has `experts` non-gated FFNs of hidden width f, of which
    every token takes k. d % 512 == 0 and f % 64 == 0, as the layer's backward needs."""

    def __init__(self, layers, d, f, experts, k, *, ell_width=None, lambda_l1=0.0, res_scale=1.0, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def normal(*shape, std=0.02):
            return torch.randn(shape, generator=g, device="cuda") * std

        self.d, self.f, self.E, self.k, self.res_scale, self.lambda_l1 = d, f, experts, k, res_scale, lambda_l1
        self.cfg = b.make_cfg(tile_cols=256, tile_slots=128, ell_width=ell_width or f)
        # fp32 masters; the layer's matrices also as bf16 copies that the kernels read
        self.blocks = [dict(w_pre=torch.ones(d, device="cuda"), w_post=torch.ones(d, device="cuda"),
                            gate_c=torch.full((d,), 0.5, device="cuda"), router=normal(d, experts),
                            W_up=normal(experts, d, f), W_down=normal(experts, f, d)) for _ in range(layers)]
        self.w_out = torch.ones(d, device="cuda")  # the norm behind the last block
        self.grads = [{n: torch.zeros_like(p) for n, p in blk.items()} for blk in self.blocks]
        self.dw_out = torch.zeros_like(self.w_out)
        self.halves = [{n: blk[n].bfloat16() for n in ("W_up", "W_down")} for blk in self.blocks]
        self.sumsq = torch.empty(1, dtype=torch.float64, device="cuda")
        self.norm = torch.empty(1, device="cuda")
        self.clip_list = b.grad_list(self.all_grads())
        self._spaces = {}

    def all_grads(self):
        return [g for blk in self.grads for g in blk.values()] + [self.dw_out]

    def _space(self, name, nbytes):
        """A workspace of at least nbytes, kept from call to call."""
        t = self._spaces.get(name)
        if t is None or t.numel() < nbytes:
            t = self._spaces[name] = torch.empty(max(1, nbytes), dtype=torch.uint8, device="cuda")
        return t

    # -- one block's layer ---------------------------------------------------------------------
    def _experts_forward(self, i, N):
        T = N.shape[0]
        logits = N.float() @ self.blocks[i]["router"]
        expert = torch.empty((T, self.k), dtype=torch.int32, device="cuda")
        weight = torch.empty((T, self.k), device="cuda")
        b.sfl_route_forward(logits, expert, weight)
        pos, offsets = torch.empty_like(expert), torch.empty(self.E + 1, dtype=torch.int32, device="cuda")
        Xs = N.new_empty((T * self.k, self.d))
        ws = self._space("order", b.sfl_expert_workspace_size(T, self.k, self.E))
        b.sfl_expert_dispatch(expert, self.E, pos, offsets, X=N, Xs=Xs, workspace=ws)
        rows = offsets.tolist()  # the launches below need the experts' row counts on the host
        Ys, kept = torch.empty_like(Xs), {}
        for e in range(self.E):
            x, y = Xs[rows[e]:rows[e + 1]], Ys[rows[e]:rows[e + 1]]
            if x.shape[0] == 0:
                continue
            bufs = kept[e] = b.alloc_twell(x.shape[0], self.f, "bf16", self.cfg)
            W_up, W_down = (self.halves[i][n][e] for n in ("W_up", "W_down"))
            args = b.ffn_args(x, W_up, W_down, self.cfg, Y=y, bufs=bufs)
            ws = self._space("forward", b.sfl_forward_workspace_size(args))
            b.sfl_ffn_forward(b.ffn_args(x, W_up, W_down, self.cfg, Y=y, bufs=bufs, workspace=ws))
        Y = torch.empty_like(N)
        b.sfl_expert_combine(Ys, pos, Y, weight=weight)
        return Y, dict(N=N, logits=logits, expert=expert, weight=weight, pos=pos, rows=rows, Xs=Xs, Ys=Ys, kept=kept, Y=Y)

    def _experts_backward(self, i, s, dY):
        """dN from dY; the layer's gradients go to self.grads[i]."""
        g = self.grads[i]
        dYs, dweight = torch.empty_like(s["Ys"]), torch.empty_like(s["weight"])
        b.sfl_expert_combine_backward(dY, s["Ys"], s["pos"], s["weight"], dYs=dYs, dweight=dweight)
        dXs = torch.empty_like(s["Xs"])
        for e in range(self.E):
            at = slice(s["rows"][e], s["rows"][e + 1])
            if e not in s["kept"]:
                g["W_up"][e].zero_()
                g["W_down"][e].zero_()
                continue
            W_up, W_down = (self.halves[i][n][e] for n in ("W_up", "W_down"))
            pos = (s["Xs"][at], W_up, W_down, dYs[at], self.cfg, s["kept"][e], self.lambda_l1, dXs[at], g["W_up"][e],
                   g["W_down"][e])
            ws = self._space("backward", b.sfl_backward_workspace_size(b.bwd_args(*pos)))
            b.sfl_ffn_backward(b.bwd_args(*pos, workspace=ws))
        dN = torch.empty_like(dY)
        b.sfl_expert_combine(dXs, s["pos"], dN)
        dlogits = torch.empty_like(s["logits"])
        b.sfl_route_backward(s["logits"], s["expert"], dweight, dlogits)
        torch.mm(s["N"].float().t(), dlogits, out=g["router"])
        return dN.add_((dlogits @ self.blocks[i]["router"].t()).to(dN.dtype))

    # -- the stack ------------------------------------------------------------------------------
    def forward(self, X):
        """The normed output [T][d] of a bf16 batch, and what `backward` needs."""
        N = torch.empty_like(X)
        b.sfl_norm_forward(X, N=N, norms=b.SFL_NORM_PRE, w_pre=self.blocks[0]["w_pre"])
        state = dict(X=[X], layers=[])
        for i, blk in enumerate(self.blocks):
            Y, s = self._experts_forward(i, N)
            ahead = self.blocks[i + 1]["w_pre"] if i + 1 < len(self.blocks) else self.w_out
            X_out, N = torch.empty_like(X), torch.empty_like(X)
            b.sfl_norm_forward(state["X"][-1], Y, X_out=X_out, N=N, w_pre=ahead, w_post=blk["w_post"],
                               gate_c=blk["gate_c"], res_scale=self.res_scale)
            state["X"].append(X_out)
            state["layers"].append(s)
        return N, state

    def backward(self, state, dN):
        """The gradient of the input; those of the parameters are in self.grads and self.dw_out."""
        T, dX = dN.shape[0], None
        ws = self._space("norm", b.sfl_norm_workspace_size(T, self.d, dN.dtype))
        for i in reversed(range(len(self.blocks))):
            blk, g = self.blocks[i], self.grads[i]
            last = i + 1 == len(self.blocks)
            dX_in, dY = torch.empty_like(dN), torch.empty_like(dN)
            b.sfl_norm_backward(state["X"][i + 1], state["layers"][i]["Y"], dX, dN, dX=dX_in, dY=dY,
                                w_pre=self.w_out if last else self.blocks[i + 1]["w_pre"],
                                dw_pre=self.dw_out if last else self.grads[i + 1]["w_pre"], w_post=blk["w_post"],
                                dw_post=g["w_post"], gate_c=blk["gate_c"], dgate_c=g["gate_c"],
                                res_scale=self.res_scale, workspace=ws)
            dX, dN = dX_in, self._experts_backward(i, state["layers"][i], dY)
        b.sfl_norm_backward(state["X"][0], None, dX, dN, dX=dX, norms=b.SFL_NORM_PRE, w_pre=self.blocks[0]["w_pre"],
                            dw_pre=self.grads[0]["w_pre"], workspace=ws)
        return dX

    def step(self, lr, max_norm):
        """Clips the gradients by their global norm and applies them; returns the norm (device). Where
        it is not finite, nothing was scaled and the step is left out."""
        ws = self._space("clip", b.sfl_grad_workspace_size(self.clip_list))
        b.sfl_grad_sumsq(self.clip_list, self.sumsq, workspace=ws)
        b.sfl_grad_clip(self.clip_list, self.sumsq, max_norm, self.norm)
        if not self.norm.isfinite().item():
            return self.norm
        for blk, g, half in zip(self.blocks, self.grads, self.halves):
            for n in blk:
                blk[n].sub_(g[n], alpha=lr)
            for n in half:
                half[n].copy_(blk[n])
        self.w_out.sub_(self.dw_out, alpha=lr)
        return self.norm


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("tokens", 2048), ("width", 1024), ("hidden", 4096), ("experts", 8), ("choices", 2),
                          ("layers", 2), ("steps", 10)):
        p.add_argument("--" + name, type=int, default=default)
    p.add_argument("--lr", type=float, default=1.0)
    p.add_argument("--max-norm", type=float, default=0.1)
    a = p.parse_args(argv)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    X = torch.randn((a.tokens, a.width), generator=g, device="cuda").bfloat16()
    target = torch.randn((a.tokens, a.width), generator=g, device="cuda")
    m = RoutedStack(a.layers, a.width, a.hidden, a.experts, a.choices)
    losses = []
    for i in range(a.steps):
        torch.cuda.synchronize()
        start = time.perf_counter()
        out, state = m.forward(X)
        off = out.float() - target
        m.backward(state, (2 / off.numel() * off).bfloat16())
        norm = m.step(a.lr, a.max_norm)
        losses.append(off.square().mean().item())
        print(f"step {i}: loss {losses[-1]:.5f}  gradient norm {norm.item():.4f}  "
              f"{(time.perf_counter() - start) * 1e3:.2f} ms", flush=True)
    return losses


if __name__ == "__main__":
    main()
