"""A block of a sequence model on channel-last rows: layer norm, a fused projection, linear attention, a projection back, a residual sum.

The same block three ways: over whole prompts (packed ones of different lengths, whose last states stay in a cache), over one token
of each request out of that cache, and over a training batch with its gradients.  Projections are 1 x 1 convolutions of the library;
their gradients are plain matrix products.

    python examples/sequence_block.py           # prompts, then tokens, against the same tokens as one prompt; a training step
"""
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2310_05218_amd as sw  # noqa: E402


class SequenceBlock:
    def __init__(self, channels=512, heads=8, kv_heads=2, dk=64, dv=64, dtype=torch.bfloat16, device="cuda", seed=0):
        g = torch.Generator().manual_seed(seed)
        self.heads, self.kv_heads, self.dk, self.dv = heads, kv_heads, dk, dv
        wide = heads * dk + kv_heads * (dk + dv)
        draw = lambda n, c: (torch.randn(n, 1, 1, c, generator=g) * c ** -0.5).to(device, dtype)
        self.w_in, self.w_out = draw(wide, channels), draw(channels, heads * dv)
        self.weight = (1 + 0.1 * torch.randn(channels, generator=g)).to(device)
        self.bias = (0.1 * torch.randn(channels, generator=g)).to(device)
        # heads that look back over a few tokens to a few hundred
        self.log_decay = torch.log1p(-torch.exp2(-torch.linspace(2, 8, heads))).to(device)

    def states(self, requests, device="cuda"):
        """A cache of states for that many requests."""
        return torch.zeros(requests, self.heads, self.dk, self.dv, device=device)

    @staticmethod
    def project(x, w):
        """Rows [..., channels] times a filter of one tap."""
        return sw.sw_conv2d_nhwc(x.reshape(1, 1, -1, x.shape[-1]), w).reshape(*x.shape[:-1], w.shape[0])

    def parts(self, fused):
        """q, k and v of a fused projection's rows, where they lie."""
        at, out = 0, []
        for heads, width in ((self.heads, self.dk), (self.kv_heads, self.dk), (self.kv_heads, self.dv)):
            out.append(fused[..., at:at + heads * width].unflatten(-1, (heads, width)))
            at += heads * width
        return out

    def prompt(self, x, starts=None, state=None, slots=None):
        """x [B,T,channels], or [T,channels] of packed sequences (starts); the sequences go on from their entries of `state`, which are brought up to date."""
        q, k, v = self.parts(self.project(sw.sw_layer_norm(x, self.weight, self.bias), self.w_in))
        o = sw.sw_linear_attention(q, k, v, self.log_decay, starts=starts, state=state, final_state=state, slots=slots)
        return x + self.project(o.flatten(-2), self.w_out)

    def token(self, x, state, slots=None):
        """x [B,channels]: one token of each request."""
        q, k, v = self.parts(self.project(sw.sw_layer_norm(x, self.weight, self.bias), self.w_in))
        return x + self.project(sw.sw_linear_attention_step(q, k, v, self.log_decay, state, slots).flatten(-2), self.w_out)

    def train(self, x, dy):
        """The block's output for x [B,T,channels] and, from its gradient dy, those of x and of the parameters."""
        rows = lambda t: t.reshape(-1, t.shape[-1])
        h, mean, rstd = sw.sw_layer_norm(x, self.weight, self.bias, stats=True)
        fused = self.project(h, self.w_in)
        q, k, v = self.parts(fused)
        o = sw.sw_linear_attention(q, k, v, self.log_decay).flatten(-2)
        y = x + self.project(o, self.w_out)
        w_in, w_out = rows(self.w_in), rows(self.w_out)
        d_o = (rows(dy) @ w_out).reshape(o.shape).unflatten(-1, (self.heads, self.dv))
        d_fused = torch.empty_like(fused)
        sw.sw_linear_attention_backward(d_o, q, k, v, self.log_decay, out=self.parts(d_fused))
        dh = (rows(d_fused) @ w_in).reshape(h.shape)
        dx, dweight, dbias = sw.sw_layer_norm_backward(dh, x, self.weight, mean, rstd)
        return y, {"x": dx + dy, "weight": dweight, "bias": dbias, "w_in": (rows(d_fused).t() @ rows(h)).reshape(self.w_in.shape),
                   "w_out": (rows(dy).t() @ rows(o)).reshape(self.w_out.shape)}


def main():
    block = SequenceBlock()
    lengths, tokens = [700, 1, 2300, 90], 5
    x = torch.randn(sum(lengths) + len(lengths) * tokens, 512, device="cuda").to(torch.bfloat16)
    ends = torch.tensor([n + tokens for n in lengths]).cumsum(0).tolist()
    rows = [list(range(e - n - tokens, e)) for e, n in zip(ends, lengths)]

    # all tokens as one prompt each, in entries 3, 0, 5 and 1 of a cache of six
    slots = torch.tensor([3, 0, 5, 1], dtype=torch.int32, device="cuda")
    starts = lambda n: torch.tensor([0, *torch.tensor(n).cumsum(0).tolist()], dtype=torch.int32, device="cuda")
    whole = block.states(6)
    want = block.prompt(x, starts([n + tokens for n in lengths]), whole, slots)

    # ... and as prompts with the last few one by one
    cache = block.states(6)
    first = torch.tensor([r for seq in rows for r in seq[:-tokens]], device="cuda")
    got = torch.empty_like(want)
    got[first] = block.prompt(x[first], starts(lengths), cache, slots)
    for i in range(tokens):
        at = torch.tensor([seq[len(seq) - tokens + i] for seq in rows], device="cuda")
        got[at] = block.token(x[at], cache, slots)
    off = lambda a, b: float((a.float() - b.float()).norm() / b.float().norm())
    print(f"{sum(lengths)} tokens of {len(lengths)} packed prompts, then {tokens} of each: outputs {off(got, want):.2e} apart, states {off(cache, whole):.2e}")

    xs, dy = (torch.randn(4, 512, 512, device="cuda").to(torch.bfloat16) for _ in range(2))
    _, grads = block.train(xs, dy)
    print("training step of 4 x 512 tokens, gradients:", ", ".join(f"{n} {tuple(g.shape)}" for n, g in grads.items()))


if __name__ == "__main__":
    main()
