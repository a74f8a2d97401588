"""A gated delta-rule layer out of the library's operators: trained for a few steps, then asked for the next tokens.

    python examples/gated_delta_layer.py

A token's way through the layer (pre-norm, H heads, d_k = d_v = D / H):

    s, n     add_rms_norm of the stream and what the layer before added to it
    q, k     projections of n, to unit length; v a projection
    beta, r  sigmoid and -softplus of projections: how much of a value is written, the log-decay of the state
    state    S <- exp(r) S + beta k (v - exp(r) S^T k)^T,   o = S^T q

A prompt is taken in chunks (gdn_chunk_tri_solve_multi, gdn_chunk_attn), one more token by gdn_step; both leave the same state behind.
Training goes back through gdn_chunk_attn_bwd and add_rms_norm_bwd; the chunk inverse itself is differentiated here, from its stored matrices.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2605_21325_amd as tri  # noqa: E402

C = 64  # tokens of a chunk


def chunks(x):
    """[B, T, H, ...] as [B * T / C * H, C, ...], in the order of the chunk matrices."""
    B, T, H = x.shape[:3]
    return x.reshape(B, T // C, C, H, *x.shape[3:]).transpose(2, 3).reshape(B * (T // C) * H, C, *x.shape[3:])


def tokens(x, B, T, H):
    """The way back."""
    return x.reshape(B, T // C, H, C, *x.shape[2:]).transpose(2, 3).reshape(B, T, H, *x.shape[2:])


def local(r):
    """Log-decays [B, T, H] summed up from each chunk's first token on."""
    B, T, H = r.shape
    full = torch.nn.functional.pad(r, (0, 0, 0, -T % C))
    return full.reshape(B, -1, C, H).cumsum(2).reshape(B, -1, H)[:, :T].contiguous()


class Norm(torch.autograd.Function):
    """(y, s): s = x + residual, y its norm."""

    @staticmethod
    def forward(ctx, x, residual, weight):
        y, s = tri.add_rms_norm(x, weight, residual)
        ctx.save_for_backward(s, weight)
        return y, s

    @staticmethod
    def backward(ctx, dy, ds):
        s, weight = ctx.saved_tensors
        dx, dweight = tri.add_rms_norm_bwd(dy.contiguous(), s, weight, dsum=ds.contiguous())
        return dx, dx, dweight.to(weight.dtype)


class Delta(torch.autograd.Function):
    """Outputs of the delta rule over whole chunks, from unit keys."""

    @staticmethod
    def forward(ctx, q, k, v, beta, g):
        U, W = tri.gdn_chunk_tri_solve_multi(k, beta, g, [v, k], C, row_scales=[beta, beta * g.exp()])
        O, _ = tri.gdn_chunk_attn(q, k, U, g, C, W=W)
        ctx.save_for_backward(q, k, v, beta, g, U, W)
        return O

    @staticmethod
    def backward(ctx, dO):
        q, k, v, beta, g, U, W = ctx.saved_tensors
        B, T, H = beta.shape
        dQ, dK, dU, dW, dg, _ = tri.gdn_chunk_attn_bwd(q, k, U, g, dO.contiguous(), C, W=W)
        # U = (I + A)^{-1} diag(beta) V,  W = (I + A)^{-1} diag(beta e^g) K,  A_ij = beta_i e^(g_i - g_j) <k_i, k_j> for i > j
        Tt = tri.gdn_chunk_tri_inv(k, beta, g, C).transpose(1, 2)
        kc, vc, uc, wc = (chunks(x).float() for x in (k, v, U, W))
        bc, gc = chunks(beta), chunks(g)
        xv, xk = Tt @ chunks(dU).float(), Tt @ chunks(dW).float()
        keep = torch.ones(C, C, device=k.device).tril(-1)
        decay = torch.exp((gc[:, :, None] - gc[:, None, :]).masked_fill(keep == 0, -torch.inf))
        dA = -(xv @ uc.transpose(1, 2) + xk @ wc.transpose(1, 2)) * decay  # times what else A_ij has of <k_i, k_j>
        kk = kc @ kc.transpose(1, 2)
        of_g = dA * kk * bc[:, :, None]
        rk = (xk * kc).sum(-1) * gc.exp()
        dv = bc[..., None] * xv
        dk = (bc * gc.exp())[..., None] * xk + (bc[:, :, None] * dA) @ kc + (bc[:, :, None] * dA).transpose(1, 2) @ kc
        dbeta = (xv * vc).sum(-1) + rk + (dA * kk).sum(-1)
        dgc = bc * rk + of_g.sum(2) - of_g.sum(1)
        back = lambda x: tokens(x, B, T, H)
        return dQ, (dK.float() + back(dk)).to(k.dtype), back(dv).to(v.dtype), back(dbeta), dg + back(dgc)


class Layer(torch.nn.Module):
    def __init__(self, D, H, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.H = H
        par = lambda *s: torch.nn.Parameter((torch.randn(*s, device=device) * s[-1] ** -0.5).to(dtype))
        self.norm = torch.nn.Parameter(torch.ones(D, dtype=dtype, device=device))
        self.qkv, self.gates, self.out = par(3 * D, D), par(2 * H, D), par(D, D)

    def split(self, n):
        """q, k, v, beta, r of the normed stream."""
        q, k, v = (n @ self.qkv.t()).unflatten(-1, (3, self.H, -1)).unbind(-3)
        beta, r = (n @ self.gates.t()).float().unflatten(-1, (2, self.H)).unbind(-2)
        unit = lambda x: torch.nn.functional.normalize(x.float(), dim=-1).to(x.dtype)
        return unit(q), unit(k), v.contiguous(), torch.sigmoid(beta).contiguous(), -torch.nn.functional.softplus(r - 3).contiguous()

    def forward(self, x, residual):
        """Of whole chunks, for training: (what the layer adds, the stream)."""
        n, s = Norm.apply(x, residual, self.norm)
        q, k, v, beta, r = self.split(n)
        return Delta.apply(q, k, v, beta, local(r)).flatten(-2) @ self.out.t(), s

    @torch.no_grad()
    def prompt(self, x, residual):
        """Of any length: the layer's outputs, the stream and the state behind it."""
        n, s = tri.add_rms_norm(x, self.norm, residual)
        q, k, v, beta, r = self.split(n)
        g = local(r)
        U, W = tri.gdn_chunk_tri_solve_multi(k, beta, g, [v, k], C, row_scales=[beta, beta * g.exp()])
        O, state = tri.gdn_chunk_attn(q, k, U, g, C, W=W)
        return O.flatten(-2) @ self.out.t(), s, state

    @torch.no_grad()
    def step(self, x, residual, state):
        """Of one token [B, D]; state is updated."""
        n, s = tri.add_rms_norm(x, self.norm, residual)
        q, k, v, beta, r = self.split(n)
        return tri.gdn_step(q, k, v, r, state, beta=beta).flatten(-2) @ self.out.t(), s


def train(layer, steps=100, B=4, T=256, seed=0):
    """The layer learns to give back the token four places before; the losses."""
    D = layer.norm.numel()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    words = torch.randn(16, D, generator=gen, device="cuda").bfloat16()
    opt = torch.optim.Adam(layer.parameters(), lr=3e-3)
    losses = []
    for _ in range(steps):
        ids = torch.randint(16, (B, T), generator=gen, device="cuda")
        said, wanted = words[ids], words[ids.roll(4, 1)]
        added, s = layer(said, torch.zeros_like(said))
        loss = ((added.float() - wanted.float())[:, 4:] ** 2).mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
    return losses


def answer(layer, B=2, T=150, more=20, seed=1):
    """A prompt and `more` tokens one by one, against the same tokens as one longer prompt: the largest relative distance of a token's output."""
    D = layer.norm.numel()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x, residual = (torch.randn(B, T + more, D, generator=gen, device="cuda").bfloat16() for _ in range(2))
    whole, _, _ = layer.prompt(x, residual)
    head, _, state = layer.prompt(x[:, :T].contiguous(), residual[:, :T].contiguous())
    got = [head] + [layer.step(x[:, t].contiguous(), residual[:, t].contiguous(), state)[0][:, None] for t in range(T, T + more)]
    got = torch.cat(got, 1).double()
    return ((got - whole.double()).norm(dim=-1) / whole.double().norm(dim=-1)).max().item()


if __name__ == "__main__":
    torch.manual_seed(0)
    layer = Layer(256, 4)
    losses = train(layer)
    print("loss %.3f -> %.3f" % (losses[0], losses[-1]))
    print("tokens one by one against one prompt: %.1e" % answer(layer))
    y, scales, _ = tri.add_rms_norm_fp8(torch.randn(3, 256, device="cuda").bfloat16(), layer.norm.detach())
    print("8-bit norm for the projection behind:", tuple(y.shape), y.dtype, tuple(scales.shape))
