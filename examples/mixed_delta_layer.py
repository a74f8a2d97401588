"""A gated delta-rule layer whose projections are mixed along time before the heads are formed, trained for a few steps, then asked for the next tokens.

    python examples/mixed_delta_layer.py

A token's way through the layer (H heads, d_k = d_v = D / H):

    p, m     projection of the normed stream to queries, keys and values side by side, and one gate for each of its columns
    y        y_t = a y_(t-1) + (1 - a) p_t with a = sigmoid(m): gated_scan, from columns of one projection
    q, k     the heads of y, to unit length where they stand: qk_norm_rope
    o        the delta rule of them and of y's values, as in gated_delta_layer.py

A prompt goes through gated_scan, qk_norm_rope, gdn_chunk_tri_solve_multi and gdn_chunk_attn; one more token through gated_scan_step, qk_norm_rope and gdn_step, with both states in
the same slots.  Training goes back through gated_scan_bwd and qk_norm_rope_bwd, which write the projection's gradient column by column.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_21325_amd as tri  # noqa: E402
from examples.gated_delta_layer import C, Delta, Norm, answer, local, train  # noqa: E402


class Mix(torch.autograd.Function):
    """y of a projection [B, T, 2 W]: its first W columns are mixed, its last W are the gates."""

    @staticmethod
    def forward(ctx, both):
        x, g = both.chunk(2, -1)
        y, _ = tri.gated_scan(x, g, logit=True, mix=True)
        ctx.save_for_backward(both, y)
        return y

    @staticmethod
    def backward(ctx, dy):
        both, y = ctx.saved_tensors
        d = torch.empty_like(both)
        (x, g), (dx, dg) = both.chunk(2, -1), d.chunk(2, -1)
        tri.gated_scan_bwd(x, g, y, dy.contiguous(), logit=True, mix=True, dx=dx, dg=dg)
        return d


class UnitHeads(torch.autograd.Function):
    """(q, k, v) of columns [..., 3 H d]: queries and keys to unit length."""

    @staticmethod
    def forward(ctx, y, H):
        q, k, v = y.unflatten(-1, (3, H, -1)).unbind(-3)
        ctx.save_for_backward(y)
        ctx.H = H
        return (*tri.qk_norm_rope(q, k, unit=True), v.contiguous())

    @staticmethod
    def backward(ctx, dq, dk, dv):
        y, = ctx.saved_tensors
        d = torch.empty_like(y)
        (q, k, _), (to_q, to_k, to_v) = (t.unflatten(-1, (3, ctx.H, -1)).unbind(-3) for t in (y, d))
        tri.qk_norm_rope_bwd(dq.contiguous(), dk.contiguous(), q, k, unit=True, dq=to_q, dk=to_k)
        to_v.copy_(dv)
        return d, None


class MixedLayer(torch.nn.Module):
    def __init__(self, D, H, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.H = H
        par = lambda *s: torch.nn.Parameter((torch.randn(*s, device=device) * s[-1] ** -0.5).to(dtype))
        self.norm = torch.nn.Parameter(torch.ones(D, dtype=dtype, device=device))
        self.mixed, self.gates, self.out = par(6 * D, D), par(2 * H, D), par(D, D)

    def rates(self, n):
        beta, r = (n @ self.gates.t()).float().unflatten(-1, (2, self.H)).unbind(-2)
        return torch.sigmoid(beta).contiguous(), -torch.nn.functional.softplus(r - 3).contiguous()

    def forward(self, x, residual):
        """Of whole chunks, for training: (what the layer adds, the stream)."""
        n, s = Norm.apply(x, residual, self.norm)
        q, k, v = UnitHeads.apply(Mix.apply(n @ self.mixed.t()), self.H)
        beta, r = self.rates(n)
        return Delta.apply(q, k, v, beta, local(r)).flatten(-2) @ self.out.t(), s

    @torch.no_grad()
    def prompt(self, x, residual):
        """Of any length: the layer's outputs, the stream and the two states behind it."""
        n, s = tri.add_rms_norm(x, self.norm, residual)
        y, mixed = tri.gated_scan(*(n @ self.mixed.t()).chunk(2, -1), logit=True, mix=True)
        q, k, v = UnitHeads.apply(y, self.H)
        beta, r = self.rates(n)
        g = local(r)
        U, W = tri.gdn_chunk_tri_solve_multi(k, beta, g, [v, k], C, row_scales=[beta, beta * g.exp()])
        O, state = tri.gdn_chunk_attn(q, k, U, g, C, W=W)
        return O.flatten(-2) @ self.out.t(), s, (mixed, state)

    @torch.no_grad()
    def step(self, x, residual, states):
        """Of one token [B, D]; the states are updated."""
        n, s = tri.add_rms_norm(x, self.norm, residual)
        mixed, state = states
        y = tri.gated_scan_step(*(n @ self.mixed.t()).chunk(2, -1), mixed, logit=True, mix=True)
        q, k, v = UnitHeads.apply(y, self.H)
        beta, r = self.rates(n)
        return tri.gdn_step(q, k, v, r, state, beta=beta).flatten(-2) @ self.out.t(), s


if __name__ == "__main__":
    torch.manual_seed(0)
    layer = MixedLayer(256, 4)
    losses = train(layer)
    print("loss %.3f -> %.3f" % (losses[0], losses[-1]))
    print("tokens one by one against one prompt: %.1e" % answer(layer))
