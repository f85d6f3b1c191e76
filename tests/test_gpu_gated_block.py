"""The example block of two mixers (examples/gated_block.py): prompts, tokens and gradients against autograd of the same block in 64 bits on the CPU.

A tensor passes through at most sixteen roundings to its format on the way (norms, projections, adapters, mixers, their gradients, products, sums), each off by at
most e = eps / 2 of a value: 2-norms are held to 16 e; in fp32 sums of a few hundred terms count, 512 u."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TOLERANCE = {torch.float32: 512 * 2.0 ** -24, torch.bfloat16: 16 * 2.0 ** -8, torch.float16: 16 * 2.0 ** -11}


@pytest.fixture(scope="module")
def GatedBlock():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_block.py")
    spec = importlib.util.spec_from_file_location("gated_block", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module.GatedBlock


def definition(block, x, p, adapter=-1):
    """The block over x [T,channels] of one sequence, 64 bits, token by token and pair by pair."""
    T, H, d = x.shape[0], block.heads, block.d
    low = lambda name, v: 0 if adapter < 0 else v @ getattr(block, "a_" + name)[adapter].double().cpu().t() @ getattr(block, "b_" + name)[adapter].double().cpu().t()
    c = x - x.mean(-1, keepdim=True)
    norm = c / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-5) * p["weight"] + p["bias"]
    q, k, v, r, decay, gate = block.parts(norm @ p["w_in"].reshape(-1, x.shape[1]).t() + low("in", norm))
    angle = torch.arange(T)[:, None, None] * block.frequencies.double().cpu()
    cos, sin = torch.cos(angle), torch.sin(angle)

    def heads(t, w):
        n = t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * w
        one, two = n[..., :d // 2], n[..., d // 2:]
        return torch.cat((one * cos - two * sin, one * sin + two * cos), -1)

    q, k = heads(q, p["q_weight"]), heads(k, p["k_weight"])
    share = H // block.kv_heads
    k, v = k.repeat_interleave(share, 1), v.repeat_interleave(share, 1)
    gap = torch.arange(T)[:, None] - torch.arange(T)[None, :]
    fade = torch.exp(block.head_decay.double().cpu()[:, None, None] * gap.clamp(min=0)) * (gap >= 0)
    pairs = (q.transpose(0, 1) @ k.transpose(0, 1).transpose(1, 2).contiguous()) * fade * d ** -0.5
    o = (pairs @ v.transpose(0, 1)).transpose(0, 1).flatten(1)
    a = torch.exp(p["log_decay"] * torch.sigmoid(decay))
    new = torch.sqrt(1 - a * a) * torch.sigmoid(gate) * r
    now, h = torch.zeros(block.width, dtype=torch.float64), []
    for t in range(T):
        now = a[t] * now + new[t]
        h.append(now)
    mixed = torch.cat((o, torch.stack(h)), 1)
    return x + mixed @ p["w_out"].reshape(x.shape[1], -1).t() + low("out", mixed)


NAMES = "weight", "bias", "q_weight", "k_weight", "log_decay", "w_in", "w_out"


def parameters(block):
    return {n: getattr(block, n).double().cpu().requires_grad_(True) for n in NAMES}


def near(got, want, dtype, what):
    got = got.double().cpu()
    assert float((got - want).norm()) <= TOLERANCE[dtype] * float(want.norm()), what


SIZES = [dict(channels=64, heads=4, kv_heads=2, d=16, width=40, rank=4), dict(channels=96, heads=2, kv_heads=2, d=48, width=130, rank=9)]


@pytest.mark.parametrize("dtype", TOLERANCE)
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("T", [1, 70, 300])
def test_gradients(GatedBlock, T, size, dtype):
    block = GatedBlock(dtype=dtype, seed=T, **size)
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
def test_prompts_then_tokens(GatedBlock, size, dtype):
    block = GatedBlock(dtype=dtype, seed=3, **size)
    lengths, tokens, adapters = [40, 1, 150], 3, [1, -1, 0]
    g = torch.Generator().manual_seed(5)
    seqs = [torch.randn(n + tokens, size["channels"], generator=g).to(dtype) for n in lengths]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    slots, adapter, starts = ints([4, 0, 2]), ints(adapters), ints([0, 40, 41, 191])
    cache = block.states(5)
    out = block.prompt(torch.cat([s[:-tokens] for s in seqs]).cuda(), starts, torch.cat([torch.arange(n) for n in lengths]).int().cuda(), cache, slots, adapter)
    steps = [block.token(torch.stack([s[len(s) - tokens + i] for s in seqs]).cuda(), ints([n + i for n in lengths]), cache, slots, adapter) for i in range(tokens)]
    assert not any(c[1].any() or c[3].any() for c in cache)
    for b, s in enumerate(seqs):
        want = definition(block, s.double(), parameters(block), adapters[b]).detach()
        near(out[int(starts[b]):int(starts[b + 1])], want[:-tokens], dtype, f"prompt {b}")
        near(torch.stack([y[b] for y in steps]), want[-tokens:], dtype, f"tokens {b}")


def test_a_captured_step(GatedBlock):
    """Prompt and token of the whole block in a graph, replayed with eager work between, on a cache that goes on."""
    block = GatedBlock(channels=64, heads=4, kv_heads=2, d=16, width=40, rank=4)
    g = torch.Generator().manual_seed(1)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    x, token = torch.randn(300, 64, generator=g).bfloat16().cuda(), torch.randn(2, 64, generator=g).bfloat16().cuda()
    starts, places, slots, adapter, at = ints([0, 210, 300]), torch.cat((torch.arange(210), torch.arange(90))).int().cuda(), ints([1, 0]), ints([2, 0]), ints([210, 90])
    cache, eager = block.states(2), block.states(2)

    def both(c):
        return block.prompt(x, starts, places, c, slots, adapter), block.token(token, at, c, slots, adapter)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(block.states(2))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(cache)
    for turn in range(4):
        x.copy_(torch.randn(300, 64, generator=g).bfloat16())
        graph.replay()
        want = both(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*out, *cache), (*want, *eager)))
