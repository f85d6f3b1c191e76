"""The example block (examples/sequence_block.py): prompts, tokens and gradients against autograd of the same block in 64 bits on the CPU.

A tensor passes through at most ten roundings to its format on the way (norm, projections, attention, products, sums), each off by at
most e = eps / 2 of a value: 2-norms are held to 10 e; in fp32 sums of a few hundred terms count, 256 u."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TOLERANCE = {torch.float32: 256 * 2.0 ** -24, torch.bfloat16: 10 * 2.0 ** -8, torch.float16: 10 * 2.0 ** -11}


@pytest.fixture(scope="module")
def SequenceBlock():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "sequence_block.py")
    spec = importlib.util.spec_from_file_location("sequence_block", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module.SequenceBlock


def definition(block, x, p):
    """The block over x [T,channels], 64 bits, every pair of tokens; p: its parameters."""
    T, H = x.shape[0], block.heads
    d = x - x.mean(-1, keepdim=True)
    h = d / torch.sqrt((d * d).mean(-1, keepdim=True) + 1e-5) * p["weight"] + p["bias"]
    q, k, v = block.parts(h @ p["w_in"].reshape(-1, x.shape[1]).t())
    share = H // block.kv_heads
    k, v = k.repeat_interleave(share, 1), v.repeat_interleave(share, 1)
    gap = torch.arange(T)[:, None] - torch.arange(T)[None, :]
    fade = torch.exp(block.log_decay.double().cpu()[:, None, None] * gap.clamp(min=0)) * (gap >= 0)
    pairs = (q.transpose(0, 1) @ k.transpose(0, 1).transpose(1, 2).contiguous()) * fade * block.dk ** -0.5
    return x + (pairs @ v.transpose(0, 1)).transpose(0, 1).flatten(1) @ p["w_out"].reshape(x.shape[1], -1).t()


def parameters(block):
    return {n: getattr(block, n).double().cpu().requires_grad_(True) for n in ("weight", "bias", "w_in", "w_out")}


def near(got, want, dtype, what):
    got = got.double().cpu()
    assert float((got - want).norm()) <= TOLERANCE[dtype] * float(want.norm()), what


SIZES = [dict(channels=64, heads=4, kv_heads=2, dk=16, dv=24), dict(channels=96, heads=2, kv_heads=2, dk=48, dv=32)]


@pytest.mark.parametrize("dtype", TOLERANCE)
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("T", [1, 70, 300])
def test_gradients(SequenceBlock, T, size, dtype):
    block = SequenceBlock(dtype=dtype, seed=T, **size)
    g = torch.Generator().manual_seed(T)
    x, dy = (torch.randn(2, T, size["channels"], generator=g).to(dtype) for _ in range(2))
    y, grads = block.train(x.cuda(), dy.cuda())
    p, xs = parameters(block), x.double().requires_grad_(True)
    want = torch.stack([definition(block, xs[b], p) for b in range(2)])
    wanted = torch.autograd.grad(want, (xs, *p.values()), dy.double())
    near(y, want.detach(), dtype, "y")
    for name, w in zip(("x", *p), wanted):
        near(grads[name], w, dtype, name)


@pytest.mark.parametrize("dtype", TOLERANCE)
@pytest.mark.parametrize("size", SIZES)
def test_prompts_then_tokens(SequenceBlock, size, dtype):
    block = SequenceBlock(dtype=dtype, seed=3, **size)
    lengths, tokens = [40, 1, 150], 3
    g = torch.Generator().manual_seed(5)
    seqs = [torch.randn(n + tokens, size["channels"], generator=g).to(dtype) for n in lengths]
    slots = torch.tensor([4, 0, 2], dtype=torch.int32, device="cuda")
    cache = block.states(5)
    starts = torch.tensor([0, 40, 41, 191], dtype=torch.int32, device="cuda")
    out = block.prompt(torch.cat([s[:-tokens] for s in seqs]).cuda(), starts, cache, slots)
    steps = [block.token(torch.stack([s[len(s) - tokens + i] for s in seqs]).cuda(), cache, slots) for i in range(tokens)]
    assert not cache[1].any() and not cache[3].any()
    for b, s in enumerate(seqs):
        want = definition(block, s.double(), parameters(block)).detach()
        near(out[int(starts[b]):int(starts[b + 1])], want[:-tokens], dtype, f"prompt {b}")
        near(torch.stack([y[b] for y in steps]), want[-tokens:], dtype, f"tokens {b}")
