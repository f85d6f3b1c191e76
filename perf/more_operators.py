"""A gated linear recurrence, norms of queries and keys with their rotation, and low-rank adapters, as cases to time and to compare.

Each case is one call that a user's program makes of these operators: the recurrence over whole sequences (equal ones or packed
ones of different lengths), its gradients, or one token of each request on a cache of states; the norms of the heads of
queries and keys with the rotation by their positions, forward or gradients; the adapters of a batch of requests beside
a projection that they share, over whole prompts or for single tokens.  `listed()` names twelve; `draw(rng)` gives more of the
same ranges: one row to a hundred thousand, sequences of one token to 8192, 32 to 8192 channels, heads of 32 to 256,
rotations of a part of a head's elements or all, ranks of 4 to 64, fp32, bf16 and half.

Activations and gates are N(0, 1), the recurrence's decays at an open gate 3/4 to 1023/1024 a token, norms' weights near one,
positions those of prompts that begin anywhere in the first hundred thousand; queries and keys are slices of a fused
projection's rows, as a block has them in hand.

With `own` false the operators run in their plain form: elementary torch operations in 32 bits (angles and sums over
all rows in 64), one rounding at the end.
"""
import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_EPS = 1e-6


def listed():
    return [
        # one long prompt on a wide layer, its last state kept for decoding
        {"name": "recurrence_long", "kind": "recurrence", "B": 1, "T": 8192, "C": 4096, "dtype": "bf16", "packed": False, "initial": False},
        # a serving batch: prompts of different lengths packed one after the other, states continued
        {"name": "recurrence_packed", "kind": "recurrence", "B": 24, "T": 6100, "C": 2048, "dtype": "f16", "packed": True, "initial": True},
        # a short prompt on a narrow layer in full precision: latency
        {"name": "recurrence_short", "kind": "recurrence", "B": 1, "T": 37, "C": 320, "dtype": "f32", "packed": False, "initial": False},
        # a training step's gradients
        {"name": "recurrence_train", "kind": "recurrence_train", "B": 4, "T": 4096, "C": 2048, "dtype": "bf16", "packed": False, "initial": False},
        # a small training batch: odd lengths and channels, the state and its gradient passed on
        {"name": "recurrence_train_odd", "kind": "recurrence_train", "B": 3, "T": 777, "C": 999, "dtype": "f32", "packed": False, "initial": True},
        # one token for a full batch out of a larger cache, a few rows of the batch unused
        {"name": "recurrence_tokens", "kind": "recurrence_token", "B": 128, "slots": 160, "idle": 3, "C": 4096, "dtype": "bf16"},
        # the queries and keys of a decode step, keys shared by four heads: latency
        {"name": "heads_tokens", "kind": "heads", "rows": 4, "H": 16, "Hk": 4, "D": 128, "pairs": 64, "interleaved": False, "dtype": "bf16"},
        # those of a long prompt
        {"name": "heads_long", "kind": "heads", "rows": 8192, "H": 32, "Hk": 8, "D": 128, "pairs": 64, "interleaved": False, "dtype": "bf16"},
        # the gradients of a large training batch
        {"name": "heads_train", "kind": "heads_train", "rows": 16384, "H": 16, "Hk": 16, "D": 128, "pairs": 64, "interleaved": False, "dtype": "bf16"},
        # a small one: heads of an odd width, half of it rotated, neighbours as pairs, full precision
        {"name": "heads_train_odd", "kind": "heads_train", "rows": 3001, "H": 6, "Hk": 3, "D": 80, "pairs": 20, "interleaved": True, "dtype": "f32"},
        # the adapters of a decode step: 64 requests, 40 adapters of rank 16
        {"name": "adapters_tokens", "kind": "adapters", "B": 64, "T": 64, "single": True, "n": 40, "idle": 4, "C_in": 2048, "C_out": 2048, "rank": 16,
         "dtype": "bf16"},
        # those of packed prompts of different lengths, a wide rank
        {"name": "adapters_prompts", "kind": "adapters", "B": 24, "T": 6100, "single": False, "n": 16, "idle": 2, "C_in": 2048, "C_out": 4096, "rank": 64,
         "dtype": "f16"},
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
        kind = rng.choice(["recurrence", "recurrence", "recurrence_train", "recurrence_token", "heads", "heads_train", "adapters", "adapters"])
        c = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"])}
        width = lambda: 8 * _log(rng, 4, 1024) if rng.random() < 0.7 else _log(rng, 32, 8192)
        if kind in ("recurrence", "recurrence_train"):
            c["packed"] = rng.random() < 0.5
            c["B"] = _log(rng, 1, 32) if c["packed"] else _log(rng, 1, 8)
            c.update(T=_log(rng, 1, 8192), C=width(), initial=rng.random() < 0.4)      # (T: of a sequence, or of all the packed ones)
        elif kind == "recurrence_token":
            b = _log(rng, 1, 256)
            c.update(B=b, slots=b + rng.choice([0, 1, b // 4]), idle=rng.choice([0, 0, b // 8]), C=width())
        elif kind in ("heads", "heads_train"):
            hk = _log(rng, 1, 16)
            d = rng.choice([64, 128, 128, 256]) if rng.random() < 0.6 else 2 * rng.randint(16, 128)
            c.update(rows=_log(rng, 1, 100000), H=hk * rng.choice([1, 1, 2, 4]), Hk=hk, D=d, pairs=d // rng.choice([2, 2, 4]), interleaved=rng.random() < 0.3)
        else:
            b = _log(rng, 1, 64)
            single = rng.random() < 0.5
            c.update(B=b, T=b if single else _log(rng, 1, 8192), single=single, n=_log(rng, 1, 64), idle=rng.choice([0, 0, b // 8]), C_in=width(),
                     C_out=width(), rank=rng.choice([4, 8, 16, 32, 64]) if rng.random() < 0.7 else rng.randint(4, 64))
        top = max(_cost(x) for x in listed() if x["kind"] == kind)
        if _cost(c) <= top:
            return c


def _rows(case):
    return case["T"] if case.get("packed", True) else case["B"] * case["T"]


def work(case):
    """Each input read once and each output written once; the operations of the formulas."""
    e = _BYTES[case["dtype"]]
    kind = case["kind"]
    if kind == "recurrence":
        n, c = _rows(case), case["C"]
        return {"bytes": 4 * n * c * e + 4 * c + 4 * case["B"] * c * (2 if case["initial"] else 1), "flops": 16 * n * c}
    if kind == "recurrence_train":
        n, c = _rows(case), case["C"]
        return {"bytes": 8 * n * c * e + 8 * c + (12 * case["B"] * c if case["initial"] else 0), "flops": 40 * n * c}
    if kind == "recurrence_token":
        n, c = case["B"] - case["idle"], case["C"]
        return {"bytes": n * c * (4 * e + 8) + 4 * c, "flops": 16 * n * c}
    if kind in ("heads", "heads_train"):
        n = case["rows"] * (case["H"] + case["Hk"]) * case["D"]
        small = 4 * case["rows"] + 8 * case["D"] + 4 * case["pairs"]
        return {"bytes": 2 * n * e + small, "flops": 8 * n} if kind == "heads" else {"bytes": 3 * n * e + small + 8 * case["D"], "flops": 18 * n}
    n, wide = case["T"], case["C_in"] + case["C_out"]
    some = max(0, case["B"] - case["idle"])
    return {"bytes": e * (n * (wide + case["C_out"]) + min(some, case["n"]) * case["rank"] * wide), "flops": 2 * n * some // case["B"] * case["rank"] * wide}


def _lengths(case, seed):
    """Lengths of packed sequences that add up to T: an empty one and a single token among them where there are several."""
    rng = random.Random(seed * 6271 + 5)
    b, t = case["B"], case["T"]
    if case.get("single"):
        return [1] * b
    if b == 1:
        return [t]
    few = [0, 1] if b > 2 and t > 1 else []
    weights = [rng.expovariate(1.0) + 0.02 for _ in range(b - len(few))]
    left, total, at, ends = t - sum(few), sum(weights), 0.0, [0]
    for w in weights[:-1]:
        at += w
        ends.append(int(left * at / total))
    ends.append(left)
    out = [y - x for x, y in zip(ends, ends[1:])] + few
    rng.shuffle(out)
    return out


def _chosen(count, of, idle, seed):
    """`count` different numbers below `of` (the numbers again where there are fewer), -1 in `idle` places."""
    g = torch.Generator().manual_seed(seed)
    at = torch.randperm(max(count, of), generator=g)[:count] % of
    at[torch.randperm(count, generator=g)[:idle]] = -1
    return at


def prepare(case, seed):
    kind, dt = case["kind"], _TYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    s = {"case": case}
    if kind in ("heads", "heads_train"):
        n, h, hk, d = (case[k] for k in ("rows", "H", "Hk", "D"))
        fused = normal(n, (h + 2 * hk) * d).mul_(1.5).to(dt)             # rows of queries, keys and values
        s["q"], s["k"] = fused[:, :h * d].unflatten(1, (h, d)), fused[:, h * d:(h + hk) * d].unflatten(1, (hk, d))
        s["wq"], s["wk"] = 1.0 + 0.1 * normal(d), 1.0 + 0.1 * normal(d)
        rng = random.Random(seed)
        at, left = [], n
        while left:                                                      # prompts of up to a few thousand tokens
            m = min(left, rng.randint(1, 1 + n // 2))
            at.append(torch.arange(m) + rng.randint(0, 100000))
            left -= m
        s["positions"] = torch.cat(at).int().cuda()
        s["frequencies"] = (10000.0 ** (-torch.arange(case["pairs"], dtype=torch.float64) / case["pairs"])).float().cuda()
        if kind == "heads_train":
            s["dq"], s["dk"] = normal(n, h, d).to(dt), normal(n, hk, d).to(dt)
        return s
    if kind == "adapters":
        b, ci, co, r = (case[k] for k in ("B", "C_in", "C_out", "rank"))
        s["lens"] = lens = _lengths(case, seed)
        s["x"], s["y"] = normal(case["T"], ci).to(dt), normal(case["T"], co).to(dt)
        s["a"], s["b"] = (normal(case["n"], r, ci) * ci ** -0.5).to(dt), (normal(case["n"], co, r) * r ** -0.5).to(dt)
        s["scales"] = 0.5 + 0.25 * normal(case["n"]).abs()
        at = _chosen(b, case["n"], case["idle"], seed)
        s["slots"], s["of"] = at.int().cuda(), at.tolist()
        s["starts"] = None if case["single"] else torch.tensor([0] + lens).cumsum(0).int().cuda()
        # an unpacked program's places of the tokens with an adapter among the rows
        first, there = torch.tensor([0] + lens).cumsum(0)[:-1], torch.tensor(lens)
        used = [i for i in range(b) if at[i] >= 0 and lens[i] > 0]
        longest = max([lens[i] for i in used], default=0)
        place = torch.arange(longest)[None, :]
        inside = place < there[used][:, None]
        s["used"], s["inside"], s["place"] = at[used].cuda(), inside.cuda(), torch.where(inside, first[used][:, None] + place, 0).cuda()
        return s
    c = case["C"]
    s["log_decay"] = torch.log1p(-torch.exp2(-2 - 8 * torch.rand(c, generator=g, device="cuda")))
    if kind == "recurrence_token":
        b = case["B"]
        s["x"], s["decay_gate"], s["input_gate"] = (normal(b, c).to(dt) for _ in range(3))
        s["state"] = normal(case["slots"], c)
        at = _chosen(b, case["slots"], case["idle"], seed)
        s["slots"] = at.int().cuda()
        s["rows_used"], s["slots_used"] = (at >= 0).nonzero()[:, 0].cuda(), at[at >= 0].cuda()
        return s
    b, t = case["B"], case["T"]
    lens = _lengths(case, seed) if case["packed"] else [t] * b
    starts = torch.tensor([0] + lens).cumsum(0)
    shape = (t, c) if case["packed"] else (b, t, c)
    s["starts"] = starts.int().cuda() if case["packed"] else None
    s["lens"] = lens
    some = [i for i in range(b) if lens[i] > 0]
    s["some"], s["firsts"], s["lasts"] = torch.tensor(some).cuda(), starts[some].cuda(), (starts[1:][some] - 1).cuda()
    s["x"], s["decay_gate"], s["input_gate"] = (normal(*shape).to(dt) for _ in range(3))
    s["state"] = normal(b, c) if case["initial"] else None
    if kind == "recurrence":
        s["final"] = torch.empty(b, c, device="cuda")
        return s
    s["h"] = _plain_recurrence(s)["h"]                                   # what the forward pass leaves for the backward one
    s["dh"] = normal(*shape).to(dt)
    s["d_final"] = normal(b, c) if case["initial"] else None
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------------------


def _gates(s):
    """The decay, its logarithm, its gate, the input's weight sqrt(1 - decay^2) and the input's gate, as rows of channels."""
    x, r, i = (s[n].reshape(-1, s[n].shape[-1]).float() for n in ("x", "decay_gate", "input_gate"))
    open_ = torch.sigmoid(r)
    log_a = s["log_decay"] * open_
    return x, torch.exp(log_a), log_a, open_, torch.sqrt(-torch.expm1(2 * log_a)), torch.sigmoid(i)


def _scan(a, b):
    """h_t = a_t h_(t-1) + b_t down the rows, by steps of 1, 2, 4 ... rows."""
    step = 1
    while step < a.shape[0]:
        b = torch.cat([b[:step], b[step:] + a[step:] * b[:-step]])
        a = torch.cat([a[:step], a[step:] * a[:-step]])
        step *= 2
    return b


def _plain_recurrence(s):
    x, a, _, _, weight, gate = _gates(s)
    b = weight * gate * x
    if s["state"] is not None:
        b[s["firsts"]] += a[s["firsts"]] * s["state"][s["some"]]
    a[s["firsts"]] = 0
    h = _scan(a, b)
    final = torch.zeros(len(s["lens"]), x.shape[1], device=x.device) if s["state"] is None else s["state"].clone()
    final[s["some"]] = h[s["lasts"]]
    return {"h": h.reshape(s["x"].shape).to(s["x"].dtype), "final": final}


def _plain_recurrence_train(s):
    x, a, log_a, open_, weight, gate = _gates(s)
    h = s["h"].reshape(x.shape).float()
    before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    before[s["firsts"]] = 0 if s["state"] is None else s["state"][s["some"]]
    up = s["dh"].reshape(x.shape).float().clone()
    if s["d_final"] is not None:
        up[s["lasts"]] += s["d_final"][s["some"]]
    next_a = torch.cat([a[1:], torch.zeros_like(a[:1])])
    next_a[s["lasts"]] = 0
    up = _scan(next_a.flip(0), up.flip(0)).flip(0)
    d_log = up * (a * before - gate * x * a * a / weight)
    out = {"dx": up * weight * gate, "d_decay_gate": d_log * log_a * (1 - open_), "d_input_gate": up * weight * x * gate * (1 - gate)}
    out = {n: v.reshape(s["x"].shape).to(s["x"].dtype) for n, v in out.items()}
    out["d_log_decay"] = (d_log * open_).sum(0, dtype=torch.float64).float()
    if s["state"] is not None:
        out["d_state"] = s["d_final"].clone()
        out["d_state"][s["some"]] = (a * up)[s["firsts"]]
    return out


def _plain_recurrence_token(s):
    rows, at = s["rows_used"], s["slots_used"]
    x, a, _, _, weight, gate = _gates({**{n: s[n][rows] for n in ("x", "decay_gate", "input_gate")}, "log_decay": s["log_decay"]})
    new = a * s["state"][at] + weight * gate * x
    s["state"][at] = new
    h = torch.zeros_like(s["x"])
    h[rows] = new.to(h.dtype)
    return {"h": h, "state": s["state"]}


def _turn(x, s, sign):
    """Pairs of elements turned by their row's position times their frequency."""
    p = s["case"]["pairs"]
    angle = s["positions"].double()[:, None] * s["frequencies"].double()
    cos, sin = torch.cos(angle).float()[:, None], sign * torch.sin(angle).float()[:, None]
    at = torch.arange(p, device=x.device)
    one, two = (2 * at, 2 * at + 1) if s["case"]["interleaved"] else (at, at + p)
    u, v = x[..., one], x[..., two]
    y = x.clone()
    y[..., one], y[..., two] = u * cos - v * sin, u * sin + v * cos
    return y


def _plain_heads(s):
    def one(x, w):
        x = x.float()
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + _EPS) * w
        return _turn(y, s, 1.0)

    return {"q": one(s["q"], s["wq"]).to(s["q"].dtype), "k": one(s["k"], s["wk"]).to(s["k"].dtype)}


def _plain_heads_train(s):
    def one(dy, x, w):
        x, dy = x.float(), _turn(dy.float(), s, -1.0)
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + _EPS)
        hat, g = x * r, dy * w
        return r * (g - hat * (g * hat).mean(-1, keepdim=True)), (dy * hat).sum((0, 1), dtype=torch.float64).float()

    dq, dwq = one(s["dq"], s["q"], s["wq"])
    dk, dwk = one(s["dk"], s["k"], s["wk"])
    return {"dq": dq.to(s["q"].dtype), "dk": dk.to(s["k"].dtype), "dwq": dwq, "dwk": dwk}


def _plain_adapters(s):
    y = s["y"].float()
    if s["place"].numel():
        x = s["x"].float()[s["place"]]
        low = torch.matmul(x, s["a"][s["used"]].float().transpose(1, 2).contiguous())
        more = torch.matmul(low, s["b"][s["used"]].float().transpose(1, 2).contiguous()) * s["scales"][s["used"]][:, None, None]
        y[s["place"][s["inside"]]] += more[s["inside"]]
    return {"y": y.to(s["y"].dtype)}


_PLAIN = {"recurrence": _plain_recurrence, "recurrence_train": _plain_recurrence_train, "recurrence_token": _plain_recurrence_token,
          "heads": _plain_heads, "heads_train": _plain_heads_train, "adapters": _plain_adapters}


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return _PLAIN[kind](s)
    import paper_2310_05218_amd as sw

    if kind == "recurrence":
        h = sw.sw_gated_recurrence(s["x"], s["decay_gate"], s["input_gate"], s["log_decay"], starts=s["starts"], state=s["state"], final_state=s["final"])
        return {"h": h, "final": s["final"]}
    if kind == "recurrence_train":
        d_state = torch.empty_like(s["state"]) if s["state"] is not None else None
        dx, dr, di, dl = sw.sw_gated_recurrence_backward(s["dh"], s["x"], s["decay_gate"], s["input_gate"], s["log_decay"], s["h"], starts=s["starts"],
                                                         state=s["state"], d_final_state=s["d_final"], d_state=d_state)
        return {"dx": dx, "d_decay_gate": dr, "d_input_gate": di, "d_log_decay": dl, **({"d_state": d_state} if d_state is not None else {})}
    if kind == "recurrence_token":
        h = sw.sw_gated_recurrence_step(s["x"], s["decay_gate"], s["input_gate"], s["log_decay"], s["state"], s["slots"])
        return {"h": h, "state": s["state"]}
    if kind == "heads":
        q, k = sw.sw_head_norm(s["q"], s["k"], s["wq"], s["wk"], s["frequencies"], s["positions"], _EPS, interleaved=case["interleaved"])
        return {"q": q, "k": k}
    if kind == "heads_train":
        dq, dk, dwq, dwk = sw.sw_head_norm_backward(s["dq"], s["dk"], s["q"], s["k"], s["wq"], s["wk"], s["frequencies"], s["positions"], _EPS,
                                                    interleaved=case["interleaved"])
        return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
    return {"y": sw.sw_adapters(s["x"], s["a"], s["b"], s["y"], s["scales"], s["slots"], starts=s["starts"])}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------------


def _exact_terms(s):
    """Row by row what the recurrence is made of, from exponentials alone."""
    x, r, i = (s[n].reshape(-1, s[n].shape[-1]).double() for n in ("x", "decay_gate", "input_gate"))
    opened, let_in = 1 / (1 + torch.exp(-r)), 1 / (1 + torch.exp(-i))
    decay = torch.exp(s["log_decay"].double() * opened)
    return x, opened, let_in, decay, ((1 - decay) * (1 + decay)) ** 0.5


def _exact_recurrence(s, train):
    x, opened, let_in, decay, weight = _exact_terms(s)
    zero = torch.zeros(x.shape[1], dtype=torch.float64, device=x.device)
    at, new = 0, weight * let_in * x
    if not train:
        h, final = torch.empty_like(x), torch.empty(len(s["lens"]), x.shape[1], dtype=torch.float64, device=x.device)
        for b, n in enumerate(s["lens"]):
            now = zero if s["state"] is None else s["state"][b].double()
            for t in range(at, at + n):
                now = torch.addcmul(new[t], decay[t], now)
                h[t] = now
            final[b] = now
            at += n
        return {"h": h.reshape(s["x"].shape), "final": final}
    h, dh = s["h"].reshape(x.shape).double(), s["dh"].reshape(x.shape).double()
    up, before = torch.empty_like(x), torch.empty_like(x)
    d_state = torch.empty(len(s["lens"]), x.shape[1], dtype=torch.float64, device=x.device)
    for b, n in enumerate(s["lens"]):
        later = zero if s["d_final"] is None else s["d_final"][b].double()
        for t in range(at + n - 1, at - 1, -1):
            up[t] = dh[t] + later
            later = decay[t] * up[t]
        d_state[b] = later
        if n:
            before[at] = zero if s["state"] is None else s["state"][b].double()
            before[at + 1:at + n] = h[at:at + n - 1]
        at += n
    # d(sqrt(1 - decay^2)) = -decay / sqrt(1 - decay^2) d(decay), d(decay) = decay d(log decay)
    d_decay = up * (before - let_in * x * decay / weight)
    shaped = lambda v: v.reshape(s["x"].shape)
    g = s["log_decay"].double()
    out = {"dx": shaped(up * weight * let_in), "d_decay_gate": shaped(d_decay * decay * g * (opened - opened ** 2)),
           "d_input_gate": shaped(up * weight * x * (let_in - let_in ** 2)), "d_log_decay": torch.einsum("nc,nc,nc->c", d_decay, decay, opened)}
    return out if s["state"] is None else {**out, "d_state": d_state}


def _exact_heads(x, w, s):
    """As complex numbers: pairs times e^(i angle)."""
    p = s["case"]["pairs"]
    y = x * (x.square().mean(-1, keepdim=True) + _EPS) ** -0.5 * w
    head, rest = y[..., :2 * p], y[..., 2 * p:]
    pairs = head.unflatten(-1, (p, 2)) if s["case"]["interleaved"] else head.unflatten(-1, (2, p)).transpose(-1, -2)
    angle = torch.outer(s["positions"].double(), s["frequencies"].double())[:, None]
    z = torch.complex(pairs[..., 0], pairs[..., 1]) * torch.polar(torch.ones_like(angle), angle)
    turned = torch.stack([z.real, z.imag], -1 if s["case"]["interleaved"] else -2).flatten(-2)
    return torch.cat([turned, rest], -1)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("recurrence", "recurrence_train"):
        return _exact_recurrence(s, kind == "recurrence_train")
    if kind == "recurrence_token":
        x, _, let_in, decay, weight = _exact_terms(s)
        h, state = torch.zeros_like(x), s["state"].double()
        for row, slot in zip(s["rows_used"].tolist(), s["slots_used"].tolist()):
            h[row] = state[slot] = decay[row] * state[slot] + weight[row] * let_in[row] * x[row]
        return {"h": h, "state": state}
    if kind == "adapters":
        y, at = s["y"].double(), 0
        for n, slot in zip(s["lens"], s["of"]):
            if n and slot >= 0:
                y[at:at + n] += s["scales"][slot].double() * (s["x"][at:at + n].double() @ s["a"][slot].double().T @ s["b"][slot].double().T)
            at += n
        return {"y": y}
    out = {}
    for n in "qk":
        x, w = s[n].double(), s["w" + n].double()
        if kind == "heads":
            out[n] = _exact_heads(x, w, s)
        else:
            x, w = x.requires_grad_(True), w.requires_grad_(True)
            out["d" + n], out["dw" + n] = torch.autograd.grad(_exact_heads(x, w, s), (x, w), s["d" + n].double())
    return out
