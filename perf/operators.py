"""Layer norm and linear attention with a decay for each head, as cases to time and to compare.

Each case is one call that a user's program makes of these operators: a layer norm over the rows of a channel-last
tensor, its backward pass, linear attention over whole sequences (equal ones or packed ones of different lengths),
its backward pass, or its recurrent form for one token of each request on a cache of states.  `listed()` names
twelve; `draw(rng)` gives more of the same ranges: rows of 32 to 8192 channels, one row to a hundred thousand,
sequences of one token to 8192, head widths of 16 to 128 (odd multiples of eight among them), keys and values
shared by groups of heads, fp32, bf16 and half.

Activations are N(0, 1), norms' inputs off centre, norms' weights near one; the heads' decays run from 3/4 to 255/256
a token, as in layers whose heads look back over a few tokens to a few hundred.

With `own` false the operators run in their plain form: elementary torch operations in 32 bits, one rounding at the end.
"""
import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_EPS = 1e-5


def listed():
    return [
        # the norm of a decode step: one row for each of a few requests, all latency
        {"name": "norm_tokens", "kind": "norm", "rows": 4, "C": 2048, "dtype": "bf16", "stats": False},
        # the norm over the channels of a channel-last image layer (32 images of 56 x 56 pixels, 64 channels), statistics kept
        {"name": "norm_pixels", "kind": "norm", "rows": 32 * 56 * 56, "C": 64, "dtype": "f32", "stats": True},
        # the norm of a large training batch of wide rows, statistics kept for the backward pass
        {"name": "norm_wide", "kind": "norm", "rows": 16384, "C": 4096, "dtype": "bf16", "stats": True},
        # its backward pass
        {"name": "norm_back_wide", "kind": "norm_back", "rows": 16384, "C": 4096, "dtype": "bf16"},
        # a small fine-tuning batch of rows whose length is no multiple of anything
        {"name": "norm_back_odd", "kind": "norm_back", "rows": 3001, "C": 999, "dtype": "f32"},
        # one long prompt, its final state kept for decoding
        {"name": "prompt_long", "kind": "prompt", "B": 1, "T": 8192, "H": 16, "Hk": 16, "Dk": 128, "Dv": 128, "dtype": "bf16",
         "packed": False, "initial": False},
        # a serving batch: prompts of different lengths packed one after the other, shared keys and values, states continued
        {"name": "prompt_packed", "kind": "prompt", "B": 24, "T": 6100, "H": 8, "Hk": 2, "Dk": 64, "Dv": 64, "dtype": "f16",
         "packed": True, "initial": True},
        # a short prompt on narrow odd heads in full precision: latency
        {"name": "prompt_short", "kind": "prompt", "B": 1, "T": 37, "H": 4, "Hk": 4, "Dk": 48, "Dv": 80, "dtype": "f32",
         "packed": False, "initial": False},
        # a training step's attention
        {"name": "train_long", "kind": "train", "B": 4, "T": 4096, "H": 16, "Hk": 16, "Dk": 128, "Dv": 128, "dtype": "bf16",
         "packed": False, "initial": False},
        # a small training batch: odd lengths, values wider than keys, keys and values shared by two heads, state and its gradient passed on
        {"name": "train_odd", "kind": "train", "B": 3, "T": 777, "H": 6, "Hk": 3, "Dk": 64, "Dv": 96, "dtype": "f32",
         "packed": False, "initial": True},
        # one token of one request: latency
        {"name": "token_one", "kind": "token", "B": 1, "slots": 1, "idle": 0, "H": 16, "Hk": 16, "Dk": 128, "Dv": 128, "dtype": "bf16"},
        # one token for a full batch out of a larger cache, a few rows of the batch unused
        {"name": "token_batch", "kind": "token", "B": 128, "slots": 160, "idle": 3, "H": 16, "Hk": 16, "Dk": 128, "Dv": 128, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    """A case's work on one scale: microseconds at 5 TB/s or 500 TFLOP/s, whichever is more."""
    w = work(case)
    return max(w["bytes"] / 5e6, w["flops"] / 5e8)


def draw(rng):
    """One more case of the listed kinds, of at most its kind's largest listed cost."""
    while True:
        kind = rng.choice(["norm", "norm", "norm_back", "norm_back", "prompt", "prompt", "train", "train", "token"])
        c = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"])}
        if kind in ("norm", "norm_back"):
            c.update(rows=_log(rng, 1, 100000), C=_log(rng, 32, 8192))
            if rng.random() < 0.6:
                c["C"] = -(-c["C"] // 8) * 8
            if kind == "norm":
                c["stats"] = rng.random() < 0.5
        else:
            group = rng.choice([1, 1, 1, 2, 4])
            hk = _log(rng, 1, 16)
            width = lambda: 8 * rng.randint(2, 16) if rng.random() < 0.5 else rng.choice([32, 64, 128])
            c.update(H=hk * group, Hk=hk, Dk=width())
            c["Dv"] = c["Dk"] if rng.random() < 0.6 else width()
            if kind == "token":
                c["B"] = _log(rng, 1, 256)
                c["slots"] = c["B"] + rng.choice([0, 1, c["B"] // 4])
                c["idle"] = rng.choice([0, 0, c["B"] // 8])
            else:
                c["packed"] = rng.random() < 0.5
                c["B"] = _log(rng, 1, 32) if c["packed"] else _log(rng, 1, 8)
                c["T"] = _log(rng, 1, 8192)            # tokens of a sequence, or of all the packed ones
                c["initial"] = rng.random() < 0.4
        top = max(_cost(x) for x in listed() if x["kind"] == kind)
        if _cost(c) <= top and c.get("H", 1) <= 32:
            return c


def _rows(case):
    return case["T"] if case["packed"] else case["B"] * case["T"]


def work(case):
    """Each input read once and each output written once; multiply-adds of the recurrence."""
    e = _BYTES[case["dtype"]]
    kind = case["kind"]
    if kind in ("norm", "norm_back"):
        n, c = case["rows"], case["C"]
        if kind == "norm":
            return {"bytes": 2 * n * c * e + 8 * c + (8 * n if case["stats"] else 0), "flops": 8 * n * c}
        return {"bytes": 3 * n * c * e + 8 * n + 12 * c, "flops": 14 * n * c}
    h, hk, dk, dv = case["H"], case["Hk"], case["Dk"], case["Dv"]
    if kind == "token":
        n = case["B"] - case["idle"]
        return {"bytes": n * h * 8 * dk * dv + n * e * (h * dk + hk * dk + hk * dv + h * dv), "flops": 5 * n * h * dk * dv}
    n, state = _rows(case), 4 * case["B"] * h * dk * dv
    if kind == "prompt":
        return {"bytes": n * e * (h * dk + hk * dk + hk * dv + h * dv) + state * (2 if case["initial"] else 1), "flops": 4 * n * h * dk * dv}
    return {"bytes": n * e * (2 * h * dk + 2 * hk * dk + 2 * hk * dv + h * dv) + (3 * state if case["initial"] else 0),
            "flops": 10 * n * h * dk * dv}


def _lengths(case, seed):
    """Lengths of packed sequences that add up to T: an empty one and a single token among them where there are several."""
    rng = random.Random(seed * 7919 + 17)
    b, t = case["B"], case["T"]
    if b == 1:
        return [t]
    fixed = [0, 1] if b > 2 and t > 1 else []
    share = [rng.expovariate(1.0) + 0.02 for _ in range(b - len(fixed))]
    left = t - sum(fixed)
    cut, at = [], 0.0
    for s in share[:-1]:
        at += s
        cut.append(int(left * at / sum(share)))
    ends = cut + [left]
    lens = [y - x for x, y in zip([0] + ends[:-1], ends)] + fixed
    rng.shuffle(lens)
    return lens


def prepare(case, seed):
    kind, dt = case["kind"], _TYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    s = {"case": case}
    if kind in ("norm", "norm_back"):
        n, c = case["rows"], case["C"]
        s["x"] = normal(n, c).mul_(1.5).add_(normal(n, 1)).to(dt)
        s["weight"] = 1.0 + 0.1 * normal(c)
        s["bias"] = 0.1 * normal(c)
        if kind == "norm_back":
            s["dy"] = normal(n, c).to(dt)
            x = s["x"].float()                 # what the forward pass leaves for the backward one
            s["mean"] = x.mean(1)
            s["rstd"] = (x - s["mean"][:, None]).square_().mean(1).add_(_EPS).rsqrt_()
        return s
    b, h, hk, dk, dv = (case[k] for k in ("B", "H", "Hk", "Dk", "Dv"))
    s["scale"] = dk ** -0.5
    s["log_decay"] = torch.tensor([math.log1p(-2.0 ** -(2 + 6 * i / max(1, h - 1))) for i in range(h)], dtype=torch.float64).float().cuda()
    if kind == "token":
        s["q"], s["k"], s["v"] = normal(b, h, dk).to(dt), normal(b, hk, dk).to(dt), normal(b, hk, dv).to(dt)
        s["state"] = normal(case["slots"], h, dk, dv)
        at = torch.randperm(case["slots"], generator=torch.Generator().manual_seed(seed))[:b]
        at[torch.randperm(b, generator=torch.Generator().manual_seed(seed + 1))[:case["idle"]]] = -1
        s["slots"] = at.int().cuda()
        s["rows_used"], s["slots_used"] = (at >= 0).nonzero()[:, 0].cuda(), at[at >= 0].cuda()
        return s
    if case["packed"]:
        lens = _lengths(case, seed)
        shape = (case["T"],)
        starts = torch.tensor([0] + lens).cumsum(0)
        s["starts"] = starts.int().cuda()
    else:
        lens = [case["T"]] * b
        shape = (b, case["T"])
        starts = torch.arange(b + 1) * case["T"]
        s["starts"] = None
    s["lens"] = lens
    # positions of every sequence's tokens among the rows, padded at the end: what an unpacked program works with
    longest = max(1, max(lens))
    place = torch.arange(longest)[None, :]
    there = place < torch.tensor(lens)[:, None]
    s["there"], s["place"] = there.cuda(), torch.where(there, starts[:-1, None] + place, 0).cuda()
    s["q"], s["k"], s["v"] = normal(*shape, h, dk).to(dt), normal(*shape, hk, dk).to(dt), normal(*shape, hk, dv).to(dt)
    s["state"] = normal(b, h, dk, dv) if case["initial"] else None
    if kind == "prompt":
        s["final"] = torch.empty(b, h, dk, dv, device="cuda")
    else:
        s["do"] = normal(*shape, h, dv).to(dt)
        s["d_final"] = normal(b, h, dk, dv) if case["initial"] else None
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------------------


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1 / torch.sqrt((d * d).mean(1) + _EPS)
    y = (d * rstd[:, None] * s["weight"] + s["bias"]).to(s["x"].dtype)
    return {"y": y, "mean": mean, "rstd": rstd} if s["case"]["stats"] else {"y": y}


def _plain_norm_back(s):
    x, dy, r = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
    hat = (x - s["mean"][:, None]) * r
    g = dy * s["weight"]
    dx = r * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * hat).sum(0), "dbias": dy.sum(0)}


def _spread(t, s, heads):
    """Rows of tokens [..., heads, width] as fp32 [sequence, head, place, width], zeros where a sequence has ended."""
    x = t.reshape(-1, t.shape[-2], t.shape[-1]).float()[s["place"]] * s["there"][:, :, None, None]
    return x.transpose(1, 2).repeat_interleave(heads // t.shape[-2], 1)


def _gather(x, s, like):
    """The way back of _spread; heads that share a row are summed."""
    b, h, n, d = x.shape
    x = x.reshape(b, like.shape[-2], -1, n, d).sum(2).transpose(1, 2)
    return x[s["there"]].reshape(like.shape).to(like.dtype)


def _power(s, n):
    """decay^n for each head in front: [heads, *n.shape]; zero for negative n."""
    g = s["log_decay"].double().reshape(-1, *[1] * n.dim())
    return torch.where(n >= 0, torch.exp(g * n.clamp(min=0)), 0.0).float()


def _fading(a, b, c, s, chunk=64):
    """sum over j <= i of decay^(i - j) (a_i . b_j) c_j, in chunks: products within a chunk, states between them."""
    n = a.shape[2]
    m = -(-n // chunk)
    a, b, c = (torch.nn.functional.pad(x, (0, 0, 0, m * chunk - n)).reshape(*x.shape[:2], m, chunk, x.shape[3]) for x in (a, b, c))
    at, step = torch.arange(chunk, device=a.device), torch.arange(m, device=a.device)
    within = torch.matmul(torch.matmul(a, b.transpose(-1, -2)) * _power(s, at[:, None] - at[None, :])[None, :, None], c)
    added = torch.matmul((b * _power(s, chunk - 1 - at)[None, :, None, :, None]).transpose(-1, -2), c)
    before = torch.matmul(_power(s, (step[:, None] - step[None, :] - 1) * chunk)[None], added.reshape(*added.shape[:3], -1)).reshape(added.shape)
    between = torch.matmul(a * _power(s, at + 1)[None, :, None, :, None], before)
    return (within + between).reshape(*a.shape[:2], m * chunk, -1)[:, :, :n]


def _ends(s):
    """decay^(places up to and with each token) and decay^(places after it), [sequence, head, place, 1]; decay^length."""
    place = torch.arange(s["there"].shape[1], device=s["there"].device)
    lens = s["there"].sum(1)
    return (_power(s, place + 1)[None, :, :, None], _power(s, lens[:, None] - 1 - place[None, :]).transpose(0, 1)[..., None],
            _power(s, lens).transpose(0, 1)[..., None, None])


def _plain_prompt(s):
    h = s["q"].shape[-2]
    q, k, v = (_spread(s[n], s, h) for n in "qkv")
    up, after, whole = _ends(s)
    o = _fading(q, k, v, s)
    final = torch.matmul((k * after).transpose(-1, -2), v)
    if s["state"] is not None:
        o = o + torch.matmul(q * up, s["state"])
        final = final + whole * s["state"]
    like = s["q"].new_empty(*s["q"].shape[:-1], v.shape[-1], device="meta")
    return {"o": _gather(o * s["scale"], s, like), "final": final}


def _plain_train(s):
    h, a = s["q"].shape[-2], s["scale"]
    q, k, v, do = (_spread(s[n], s, h) for n in ("q", "k", "v", "do"))
    up, after, whole = _ends(s)
    back = lambda x, y, z: _fading(x.flip(2), y.flip(2), z.flip(2), s).flip(2)
    dq, dk, dv = a * _fading(do, v, k, s), a * back(v, do, q), a * back(k, q, do)
    out = {}
    if s["state"] is not None:
        dq = dq + a * torch.matmul(do * up, s["state"].transpose(-1, -2))
        dk = dk + torch.matmul(v * after, s["d_final"].transpose(-1, -2))
        dv = dv + torch.matmul(k * after, s["d_final"])
        out["d_state"] = a * torch.matmul((q * up).transpose(-1, -2), do) + whole * s["d_final"]
    return {"dq": _gather(dq, s, s["q"]), "dk": _gather(dk, s, s["k"]), "dv": _gather(dv, s, s["v"]), **out}


def _plain_token(s):
    rows, at = s["rows_used"], s["slots_used"]
    h = s["q"].shape[1]
    q, k, v = (s[n][rows].float().repeat_interleave(h // s[n].shape[1], 1) for n in "qkv")
    new = torch.exp(s["log_decay"])[:, None, None] * s["state"][at] + k[..., None] * v[..., None, :]
    s["state"][at] = new
    o = torch.zeros(s["q"].shape[0], h, v.shape[-1], device=q.device)
    o[rows] = s["scale"] * (q[..., None] * new).sum(-2)
    return {"o": o.to(s["q"].dtype), "state": s["state"]}


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"norm": _plain_norm, "norm_back": _plain_norm_back, "prompt": _plain_prompt, "train": _plain_train, "token": _plain_token}[kind](s)
    import paper_2310_05218_amd as sw

    if kind == "norm":
        if s["case"]["stats"]:
            y, mean, rstd = sw.sw_layer_norm(s["x"], s["weight"], s["bias"], _EPS, stats=True)
            return {"y": y, "mean": mean, "rstd": rstd}
        return {"y": sw.sw_layer_norm(s["x"], s["weight"], s["bias"], _EPS)}
    if kind == "norm_back":
        dx, dweight, dbias = sw.sw_layer_norm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"])
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    if kind == "token":
        o = sw.sw_linear_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], s["slots"], s["scale"])
        return {"o": o, "state": s["state"]}
    if kind == "prompt":
        o = sw.sw_linear_attention(s["q"], s["k"], s["v"], s["log_decay"], s["scale"], starts=s["starts"], state=s["state"], final_state=s["final"])
        return {"o": o, "final": s["final"]}
    d_state = torch.empty_like(s["state"]) if s["state"] is not None else None
    dq, dk, dv = sw.sw_linear_attention_backward(s["do"], s["q"], s["k"], s["v"], s["log_decay"], s["scale"], starts=s["starts"],
                                                 state=s["state"], d_final_state=s["d_final"], d_state=d_state)
    return {"dq": dq, "dk": dk, "dv": dv, **({"d_state": d_state} if d_state is not None else {})}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------------


def _exact_attention(s, train):
    """Sequence by sequence and head by head, every pair of tokens: no chunks, no padding."""
    q, k, v = (s[n].reshape(-1, *s[n].shape[-2:]).double() for n in "qkv")
    h, group = q.shape[1], q.shape[1] // k.shape[1]
    state = s["state"].double() if s["state"] is not None else None
    if train:
        do = s["do"].reshape(-1, *s["do"].shape[-2:]).double()
        grads = [torch.zeros_like(x) for x in (q, k, v)]
        d_final = s["d_final"].double() if state is not None else None
        d_state = torch.zeros_like(d_final) if state is not None else None
    else:
        o = torch.zeros(q.shape[0], h, v.shape[2], dtype=torch.float64, device=q.device)
        final = torch.zeros(len(s["lens"]), h, q.shape[2], v.shape[2], dtype=torch.float64, device=q.device)
    first = 0
    for b, n in enumerate(s["lens"]):
        t = torch.arange(n, device=q.device, dtype=torch.float64)
        gap = t[:, None] - t[None, :]
        rows = slice(first, first + n)
        first += n
        for i in range(h):
            g, u = s["log_decay"][i].double(), i // group
            fade = torch.exp(g * gap.clamp(min=0)).masked_fill_(gap < 0, 0.0)
            up, after, whole = torch.exp(g * (t + 1))[:, None], torch.exp(g * (n - 1 - t))[:, None], torch.exp(g * n)
            qi, ki, vi = q[rows, i], k[rows, u], v[rows, u]
            if not train:
                o[rows, i] = ((qi @ ki.T) * fade) @ vi
                final[b, i] = ki.T @ (after * vi)
                if state is not None:
                    o[rows, i] += up * (qi @ state[b, i])
                    final[b, i] += whole * state[b, i]
                continue
            d = s["scale"] * do[rows, i]
            pair, dpair = (qi @ ki.T) * fade, (d @ vi.T) * fade
            grads[0][rows, i] += dpair @ ki
            grads[1][rows, u] += dpair.T @ qi
            grads[2][rows, u] += pair.T @ d
            if state is not None:
                grads[0][rows, i] += up * (d @ state[b, i].T)
                grads[1][rows, u] += after * (vi @ d_final[b, i].T)
                grads[2][rows, u] += after * (ki @ d_final[b, i])
                d_state[b, i] = qi.T @ (up * d) + whole * d_final[b, i]
    if train:
        named = {n: x.reshape(s[m].shape) for n, m, x in zip(("dq", "dk", "dv"), "qkv", grads)}
        return named if state is None else {**named, "d_state": d_state}
    return {"o": (s["scale"] * o).reshape(*s["q"].shape[:-1], v.shape[2]), "final": final}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("prompt", "train"):
        return _exact_attention(s, kind == "train")
    if kind == "token":
        o = torch.zeros(*s["q"].shape[:2], s["v"].shape[2], dtype=torch.float64, device="cuda")
        state = s["state"].double()
        group = s["q"].shape[1] // s["k"].shape[1]
        for row, slot in zip(s["rows_used"].tolist(), s["slots_used"].tolist()):
            k, v = (s[n][row].double().repeat_interleave(group, 0) for n in "kv")
            state[slot] = torch.exp(s["log_decay"].double())[:, None, None] * state[slot] + torch.einsum("hk,hv->hkv", k, v)
            o[row] = s["scale"] * torch.einsum("hk,hkv->hv", s["q"][row].double(), state[slot])
        return {"o": o, "state": state}
    x = s["x"].double()
    if kind == "norm":
        mean, var = x.mean(1), x.var(1, unbiased=False)
        y = (x - mean[:, None]) / torch.sqrt(var + _EPS)[:, None] * s["weight"].double() + s["bias"].double()
        return {"y": y, "mean": mean, "rstd": (var + _EPS) ** -0.5} if case["stats"] else {"y": y}
    dy, w, mean, r = s["dy"].double(), s["weight"].double(), s["mean"].double()[:, None], s["rstd"].double()[:, None]
    hat = (x - mean) * r
    c = x.shape[1]
    dx = r / c * (c * dy * w - (dy * w).sum(1, keepdim=True) - hat * (dy * w * hat).sum(1, keepdim=True))
    return {"dx": dx, "dweight": torch.einsum("nc,nc->c", dy, hat), "dbias": dy.sum(0)}
