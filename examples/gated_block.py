"""A block of a sequence model with two mixers on channel-last rows: layer norm and a fused projection, from which one half goes through linear attention
on normed and turned queries and keys, the other through a gated recurrence; a projection back and a residual sum.  Both projections have
low-rank adapters, one for each request.

The same block three ways: over packed prompts of different lengths, whose states stay in a cache, over one token of each request out of that cache, and over
a training batch with its gradients (without adapters).

    python examples/gated_block.py              # prompts, then tokens, against the same tokens as one prompt; a training step
"""
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2310_05218_amd as sw  # noqa: E402


class GatedBlock:
    def __init__(self, channels=512, heads=8, kv_heads=2, d=64, width=320, rank=8, adapters=3, dtype=torch.bfloat16, device="cuda", seed=0):
        g = torch.Generator().manual_seed(seed)
        self.heads, self.kv_heads, self.d, self.width = heads, kv_heads, d, width
        # rows of the fused projection: q, k, v; the recurrence's input and its two gates
        self.parts_of = [(heads, d), (kv_heads, d), (kv_heads, d), (width,), (width,), (width,)]
        wide, inner = (heads + 2 * kv_heads) * d + 3 * width, heads * d + width
        draw = lambda *s: torch.randn(s, generator=g)
        self.w_in, self.w_out = (draw(wide, 1, 1, channels) * channels ** -0.5).to(device, dtype), (draw(channels, 1, 1, inner) * inner ** -0.5).to(device, dtype)
        # two factors a projection and adapter
        self.a_in, self.b_in = (draw(adapters, rank, channels) * channels ** -0.5).to(device, dtype), (draw(adapters, wide, rank) * 0.1).to(device, dtype)
        self.a_out, self.b_out = (draw(adapters, rank, inner) * inner ** -0.5).to(device, dtype), (draw(adapters, channels, rank) * 0.1).to(device, dtype)
        self.weight, self.bias = (1 + 0.1 * draw(channels)).to(device), (0.1 * draw(channels)).to(device)
        self.q_weight, self.k_weight = (1 + 0.1 * draw(d)).to(device), (1 + 0.1 * draw(d)).to(device)
        self.frequencies = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).float().to(device)
        self.head_decay = torch.log1p(-torch.exp2(-torch.linspace(2, 8, heads))).to(device)
        self.log_decay = torch.log1p(-torch.exp2(-2 - 6 * torch.rand(width, generator=g))).to(device)

    def states(self, requests, device="cuda"):
        """A cache for that many requests: attention's states and the recurrence's."""
        return torch.zeros(requests, self.heads, self.d, self.d, device=device), torch.zeros(requests, self.width, device=device)

    @staticmethod
    def project(x, w):
        """Rows [..., channels] times a filter of one tap."""
        return sw.sw_conv2d_nhwc(x.reshape(1, 1, -1, x.shape[-1]), w).reshape(*x.shape[:-1], w.shape[0])

    def adapted(self, x, w, a, b, adapter, starts):
        """The projection and, where requests have them, their adapters."""
        y = self.project(x, w)
        return y if adapter is None else sw.sw_adapters(x, a, b, y, None, adapter, starts, out=y)

    def parts(self, fused):
        """q, k, v, the recurrence's input and gates of a fused projection's rows, where they lie."""
        at, out = 0, []
        for shape in self.parts_of:
            n = shape[0] * (shape[1] if len(shape) == 2 else 1)
            part = fused[..., at:at + n]
            out.append(part.unflatten(-1, shape) if len(shape) == 2 else part)
            at += n
        return out

    def prompt(self, x, starts, positions, cache, slots=None, adapter=None):
        """x [T,channels] of packed sequences, positions [T] int32; the sequences go on from their entries of the cache, which are brought up to date."""
        fused = self.adapted(sw.sw_layer_norm(x, self.weight, self.bias), self.w_in, self.a_in, self.b_in, adapter, starts)
        q, k, v, r, decay, gate = self.parts(fused)
        sw.sw_head_norm(q, k, self.q_weight, self.k_weight, self.frequencies, positions, out=(q, k))
        o = sw.sw_linear_attention(q, k, v, self.head_decay, starts=starts, state=cache[0], final_state=cache[0], slots=slots)
        h = sw.sw_gated_recurrence(r, decay, gate, self.log_decay, starts=starts, state=cache[1], final_state=cache[1], slots=slots)
        return x + self.adapted(torch.cat((o.flatten(-2), h), -1), self.w_out, self.a_out, self.b_out, adapter, starts)

    def token(self, x, positions, cache, slots=None, adapter=None):
        """x [B,channels]: one token of each request."""
        fused = self.adapted(sw.sw_layer_norm(x, self.weight, self.bias), self.w_in, self.a_in, self.b_in, adapter, None)
        q, k, v, r, decay, gate = self.parts(fused)
        sw.sw_head_norm(q, k, self.q_weight, self.k_weight, self.frequencies, positions, out=(q, k))
        o = sw.sw_linear_attention_step(q, k, v, self.head_decay, cache[0], slots)
        h = sw.sw_gated_recurrence_step(r, decay, gate, self.log_decay, cache[1], slots)
        return x + self.adapted(torch.cat((o.flatten(-2), h), -1), self.w_out, self.a_out, self.b_out, adapter, None)

    def train(self, x, dy):
        """The block's output for x [B,T,channels] and, from its gradient dy, those of x and of the parameters."""
        rows = lambda t: t.reshape(-1, t.shape[-1])
        norm, mean, rstd = sw.sw_layer_norm(x, self.weight, self.bias, stats=True)
        fused = self.project(norm, self.w_in)
        q, k, v, r, decay, gate = self.parts(fused)
        nq, nk = sw.sw_head_norm(q, k, self.q_weight, self.k_weight, self.frequencies)
        o = sw.sw_linear_attention(nq, nk, v, self.head_decay)
        h = sw.sw_gated_recurrence(r, decay, gate, self.log_decay)
        mixed = torch.cat((o.flatten(-2), h), -1)
        y = x + self.project(mixed, self.w_out)
        w_in, w_out = rows(self.w_in), rows(self.w_out)
        d_mixed = (rows(dy) @ w_out).reshape(mixed.shape)
        d_o, d_h = d_mixed[..., :self.heads * self.d].unflatten(-1, (self.heads, self.d)), d_mixed[..., self.heads * self.d:]
        d_fused = torch.empty_like(fused)
        dq, dk, dv, *d_rest = self.parts(d_fused)
        sw.sw_linear_attention_backward(d_o, nq, nk, v, self.head_decay, out=(dq, dk, dv))
        *_, d_log_decay = sw.sw_gated_recurrence_backward(d_h, r, decay, gate, self.log_decay, h, out=d_rest)
        *_, dq_weight, dk_weight = sw.sw_head_norm_backward(dq, dk, q, k, self.q_weight, self.k_weight, self.frequencies, out=(dq, dk))
        d_norm = (rows(d_fused) @ w_in).reshape(norm.shape)
        dx, dweight, dbias = sw.sw_layer_norm_backward(d_norm, x, self.weight, mean, rstd)
        return y, {"x": dx + dy, "weight": dweight, "bias": dbias, "q_weight": dq_weight, "k_weight": dk_weight, "log_decay": d_log_decay,
                   "w_in": (rows(d_fused).t() @ rows(norm)).reshape(self.w_in.shape), "w_out": (rows(dy).t() @ rows(mixed)).reshape(self.w_out.shape)}


def main():
    block = GatedBlock()
    lengths, tokens = [700, 1, 2300, 90], 5
    x = torch.randn(sum(lengths) + len(lengths) * tokens, 512, device="cuda").to(torch.bfloat16)
    ends = torch.tensor([n + tokens for n in lengths]).cumsum(0).tolist()
    rows = [list(range(e - n - tokens, e)) for e, n in zip(ends, lengths)]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")

    # all tokens as one prompt each, in entries 3, 0, 5 and 1 of a cache of six, with adapters 2, 0 and none
    slots, adapter = ints([3, 0, 5, 1]), ints([2, 0, -1, 2])
    starts = lambda n: ints([0, *torch.tensor(n).cumsum(0).tolist()])
    places = lambda n: torch.cat([torch.arange(k) for k in n]).int().cuda()
    whole = block.states(6)
    all_lengths = [n + tokens for n in lengths]
    want = block.prompt(x, starts(all_lengths), places(all_lengths), whole, slots, adapter)

    # ... and as prompts with the last few one by one
    cache = block.states(6)
    first = torch.tensor([r for seq in rows for r in seq[:-tokens]], device="cuda")
    got = torch.empty_like(want)
    got[first] = block.prompt(x[first], starts(lengths), places(lengths), cache, slots, adapter)
    for i in range(tokens):
        at = torch.tensor([seq[len(seq) - tokens + i] for seq in rows], device="cuda")
        got[at] = block.token(x[at], ints([n + i for n in lengths]), cache, slots, adapter)
    off = lambda a, b: float((a.float() - b.float()).norm() / b.float().norm())
    print(f"{sum(lengths)} tokens of {len(lengths)} packed prompts, then {tokens} of each: outputs {off(got, want):.2e} apart, "
          f"states {off(cache[0], whole[0]):.2e} and {off(cache[1], whole[1]):.2e}")

    xs, dy = (torch.randn(4, 512, 512, device="cuda").to(torch.bfloat16) for _ in range(2))
    _, grads = block.train(xs, dy)
    print("training step of 4 x 512 tokens, gradients:", ", ".join(f"{n} {tuple(g.shape)}" for n, g in grads.items()))


if __name__ == "__main__":
    main()
