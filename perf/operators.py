"""Operators beside the quantised projections of an attention block or an FFN, on real sizes: what they are, their inputs,
their plain form in elementary torch operations, and the calls that a program makes of the library.

  adapters     y = base + scale_a (x A_a^T) B_a^T: low-rank adapters of many requests beside one shared projection (or the
               stacked q / k / v or gate / up one); every row of the batch names its adapter, or none
  norm_rotate  the RMS norm of every query and key head, and the position rotation, on the stacked projection's output
  rotate       the position rotation alone

Sizes are those of the repository's configurations (Qwen3-4B-shaped blocks: 32 query and 8 key heads of 128, hidden 2560,
9728 FFN channels) and generic ones; `draw` spreads them over the ranges in between.
"""
import math

import torch

own = False

QKV = "4096,1024,1024"


def listed():
    return [
        # one sequence being decoded, its adapter on q / k / v: launches and latency
        {"name": "adapters_qkv_1", "kind": "adapters", "M": 1, "K": 2560, "parts": QKV, "R": 16, "S": 8, "requests": 1, "bare": 0,
         "mixed": False, "y": "bf16"},
        # a served decode batch in which most requests bring an adapter of their own: the adapters' bytes count
        {"name": "adapters_qkv_64", "kind": "adapters", "M": 64, "K": 2560, "parts": QKV, "R": 16, "S": 64, "requests": 64, "bare": 6,
         "mixed": False, "y": "bf16"},
        # a decode batch that shares a dozen adapters of unequal rank, down projection, fp32 output
        {"name": "adapters_down_97_f32", "kind": "adapters", "M": 97, "K": 9728, "parts": "2560", "R": 32, "S": 12, "requests": 97,
         "bare": 9, "mixed": True, "y": "f32"},
        # three short prompts of odd lengths through the o projection
        {"name": "adapters_o_387", "kind": "adapters", "M": 387, "K": 4096, "parts": "2560", "R": 32, "S": 4, "requests": 3, "bare": 0,
         "mixed": False, "y": "bf16"},
        # a prefill chunk of nine requests (one of them bare) through q / k / v
        {"name": "adapters_qkv_4096", "kind": "adapters", "M": 4096, "K": 2560, "parts": QKV, "R": 16, "S": 8, "requests": 9, "bare": 1,
         "mixed": False, "y": "bf16"},
        # the same chunk through gate / up with adapters of a high rank: the most bytes and products of all
        {"name": "adapters_gate_up_4096", "kind": "adapters", "M": 4096, "K": 2560, "parts": "9728,9728", "R": 64, "S": 8, "requests": 8,
         "bare": 0, "mixed": False, "y": "bf16"},
        # one token's heads: latency
        {"name": "norm_rotate_1", "kind": "norm_rotate", "M": 1, "q": 32, "k": 8, "D": 128, "rot": 128, "layout": "half",
         "scaling": "none", "far": 40960, "requests": 1, "inplace": True, "dtype": "bf16"},
        # a served decode batch in a long context (YaRN), heads handed to the attention in buffers of their own
        {"name": "norm_rotate_64", "kind": "norm_rotate", "M": 64, "q": 32, "k": 8, "D": 128, "rot": 128, "layout": "half",
         "scaling": "yarn", "far": 131072, "requests": 64, "inplace": False, "dtype": "bf16"},
        # a prefill chunk of five requests, in the place where the projection left it
        {"name": "norm_rotate_4096", "kind": "norm_rotate", "M": 4096, "q": 32, "k": 8, "D": 128, "rot": 128, "layout": "half",
         "scaling": "none", "far": 40960, "requests": 5, "inplace": True, "dtype": "bf16"},
        # a batch of decoding sequences, interleaved pairs in half of the head
        {"name": "rotate_48_pairs", "kind": "rotate", "M": 48, "q": 16, "k": 2, "D": 128, "rot": 64, "layout": "pairs",
         "scaling": "linear", "far": 32768, "requests": 48, "inplace": True, "dtype": "bf16"},
        # a ragged chunk, fp32, heads of 80 of which 32 turn
        {"name": "rotate_1533_f32", "kind": "rotate", "M": 1533, "q": 20, "k": 20, "D": 80, "rot": 32, "layout": "half",
         "scaling": "none", "far": 4096, "requests": 4, "inplace": False, "dtype": "f32"},
        # a long chunk far out in a context stretched by wavelength
        {"name": "rotate_8192_far", "kind": "rotate", "M": 8192, "q": 32, "k": 8, "D": 128, "rot": 128, "layout": "half",
         "scaling": "bands", "far": 1048576, "requests": 2, "inplace": False, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("adapters", "adapters", "norm_rotate", "rotate"))
    if kind == "adapters":
        parts = [8 * _log(rng, 32, 1216) for _ in range(rng.randint(1, 3))]
        parts[-1] += rng.choice((0, 0, 3))
        R = 8 * _log(rng, 1, 8)
        M = _log(rng, 1, 4096)
        requests = rng.choice((M, min(M, _log(rng, 1, 64))))
        S = min(_log(rng, 2, 96), max(2, requests))
        return {"kind": kind, "M": M, "K": 32 * _log(rng, 8, 304 if M < 1024 else 80), "parts": ",".join(map(str, parts)), "R": R, "S": S,
                "requests": requests, "bare": rng.choice((0, requests // 10)), "mixed": rng.random() < 0.3,
                "y": "f32" if sum(parts) < 9728 and rng.random() < 0.3 else "bf16"}
    D = rng.choice((64, 80, 96, 128, 128, 128, 192, 256))
    k = rng.choice((1, 2, 4, 8))
    M = _log(rng, 1, 8192)
    q = k * rng.choice((1, 4, 8))
    q = min(q, 32 * 128 // D)
    scaling = rng.choice(("none", "linear", "ntk", "yarn", "bands"))
    # (pass upon pass in one place must not grow, as a rotation alone does by YaRN's factor)
    inplace = rng.random() < 0.5 and not (kind == "rotate" and scaling == "yarn")
    return {"kind": kind, "M": M, "q": q, "k": k, "D": D, "rot": rng.choice((D, D, D // 2, D // 4)), "layout": rng.choice(("half", "half", "pairs")),
            "scaling": scaling, "far": max(M + 1, _log(rng, 2048, 1048576)),
            "requests": rng.choice((M, min(M, _log(rng, 1, 16)))), "inplace": inplace, "dtype": "f32" if M <= 4096 and rng.random() < 0.3 else "bf16"}


# ---- inputs -------------------------------------------------------------------------------------------------

_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
BASE = 1000000.0
ORIGINAL = 32768        # positions that the frequencies were trained for
FACTOR = 4.0


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _lengths(c, g):
    """Rows of each request: all of them one, or a random cut of M."""
    M, n = c["M"], c["requests"]
    if n >= M:
        return torch.ones(M, dtype=torch.int64, device="cuda")
    cuts = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), torch.randperm(M - 1, generator=g, device="cuda")[: n - 1].sort().values + 1,
                      torch.full((1,), M, dtype=torch.int64, device="cuda")])
    return cuts[1:] - cuts[:-1]


def _parts(c):
    return [int(n) for n in c["parts"].split(",")]


def _used(c):
    return min(c["S"], c["requests"] - c["bare"])


def _ranks(c):
    return [c["R"] if s % 2 == 0 or not c["mixed"] else max(1, c["R"] // 2) for s in range(c["S"])]


def _scaling(c):
    """Names and numbers of the frequencies' scaling, as a model's configuration holds them."""
    kind = c["scaling"]
    o = {"head_dim": c["D"], "rot_dim": c["rot"], "layout": c["layout"], "scaling": kind, "base": BASE, "factor": FACTOR if kind != "none" else 1.0}
    if kind in ("yarn", "bands"):
        o["original_positions"] = ORIGINAL
    if kind == "yarn":
        o.update(beta_fast=32.0, beta_slow=1.0)
    if kind == "bands":
        o.update(low_factor=1.0, high_factor=4.0)
    return o


def prepare(case, seed):
    s = (_prepare_adapters if case["kind"] == "adapters" else _prepare_heads)(case, _generator(seed))
    s["case"] = case
    return s


def _prepare_adapters(c, g):
    M, K, R, S, parts = c["M"], c["K"], c["R"], c["S"], _parts(c)
    N = sum(parts)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    # activations: heavy-tailed, one channel in a hundred loud; weights N(0, 0.02^2)
    gain = torch.exp(normal(K))
    gain[torch.randperm(K, generator=g, device="cuda")[: round(0.01 * K)]] *= 30.0
    x = (normal(M, K) / torch.sqrt(normal(3, M, K).square_().sum(0) / 3) * gain).to(torch.bfloat16)
    ranks = torch.tensor(_ranks(c), dtype=torch.int32, device="cuda")
    kept = (torch.arange(R, device="cuda") < ranks[:, None]).float()
    A = (normal(S, len(parts), R, K) * 0.02 * kept[:, None, :, None]).to(torch.bfloat16)
    B = (normal(S, N, R) * 0.02 * kept[:, None, :]).to(torch.bfloat16)
    scale = 1.0 + torch.rand(S, generator=g, device="cuda")
    # the projection's own output: as large as a product of x with such weights is
    ld = -(-N // 8) * 8
    base, out = (torch.zeros((M, ld), dtype=_DTYPE[c["y"]], device="cuda")[:, :N] for _ in range(2))
    base.copy_(normal(M, N) * (0.02 * x.float().square().sum(1, keepdim=True).sqrt()))
    # every used adapter serves a request; `bare` requests have none
    slot = torch.arange(c["requests"], device="cuda") % max(1, _used(c))
    slot[c["requests"] - c["bare"]:] = -1
    slot = slot[torch.randperm(c["requests"], generator=g, device="cuda")]
    rows = torch.repeat_interleave(slot, _lengths(c, g)).to(torch.int32)
    s = {"x": x, "A": A, "B": B, "scale": scale, "ranks": ranks if c["mixed"] else None, "base": base, "out": out, "rows": rows}
    if own:
        from paper_2609_22106_b200 import binding as prq

        s["adapters"] = prq.Adapters(A, B, parts, scale=scale, ranks=s["ranks"])
        s["workspace"] = prq.adapters_workspace(s["adapters"], M)
    return s


def _positions(c, g):
    """Decoding sequences stand anywhere in their contexts; the rows of a prompt follow one another."""
    n = _lengths(c, g)
    start = (torch.rand(n.numel(), generator=g, device="cuda", dtype=torch.float64) * (c["far"] - n).clamp(min=1)).long()
    first = torch.cumsum(n, 0) - n
    return (torch.repeat_interleave(start - first, n) + torch.arange(c["M"], device="cuda")).to(torch.int32)


def _prepare_heads(c, g):
    M, q, k, D = c["M"], c["q"], c["k"], c["D"]
    # q, k and v side by side, as the stacked projection writes them
    y = torch.randn(M, (q + 2 * k) * D, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(M, 1, generator=g, device="cuda"))
    y = y.to(_DTYPE[c["dtype"]])
    heads = y[:, : q * D].view(M, q, D), y[:, q * D:(q + k) * D].view(M, k, D)
    to = heads if c["inplace"] else tuple(torch.zeros(t.shape, dtype=y.dtype, device="cuda") for t in heads)
    weights = tuple(0.5 + torch.rand(D, generator=g, device="cuda") for _ in range(2)) if c["kind"] == "norm_rotate" else (None, None)
    s = {"heads": heads, "to": to, "weights": weights, "positions": _positions(c, g), "frequencies": _frequencies(c)}
    if own:
        from paper_2609_22106_b200 import binding as prq

        s["rope"] = prq.Rope(**_scaling(c))
    return s


# ---- the plain form -----------------------------------------------------------------------------------------

def _frequencies(c):
    """Angle per position of every pair, in 64 bits, and the factor that goes with the scaling."""
    o = _scaling(c)
    d, base, factor = o["rot_dim"], o["base"], o["factor"]
    i = torch.arange(d // 2, dtype=torch.float64, device="cuda")
    if o["scaling"] == "ntk":
        base = base * factor ** (d / (d - 2))
    f = torch.exp(-math.log(base) * 2 * i / d)
    if o["scaling"] == "linear":
        return f / factor, 1.0
    if o["scaling"] == "yarn":
        low, high = (d * math.log(o["original_positions"] / (b * 2 * math.pi)) / (2 * math.log(base)) for b in (o["beta_fast"], o["beta_slow"]))
        low, high = max(math.floor(low), 0), min(math.ceil(high), d - 1)
        ramp = ((i - low) / max(high - low, 0.001)).clamp(0, 1)
        return f / factor * ramp + f * (1 - ramp), 0.1 * math.log(factor) + 1
    if o["scaling"] == "bands":
        turns = o["original_positions"] * f / (2 * math.pi)      # within the trained context
        smooth = ((turns - o["low_factor"]) / (o["high_factor"] - o["low_factor"])).clamp(0, 1)
        return f / factor * (1 - smooth) + f * smooth, 1.0
    return f, 1.0


def _plain_adapters(s):
    c, parts = s["case"], _parts(s["case"])
    S, P, R, K = s["A"].shape
    mine = (s["rows"][:, None] == torch.arange(S, device="cuda")).float() * s["scale"]
    h = (s["x"].float() @ s["A"].float().view(S * P * R, K).T).view(-1, S, P, R) * mine[:, :, None, None]
    B = s["B"].float().split(parts, dim=1)
    delta = torch.cat([h[:, :, p].reshape(-1, S * R) @ b.transpose(1, 2).reshape(S * R, -1) for p, b in enumerate(B)], dim=1)
    s["out"].copy_(s["base"].float() + delta)
    return s["out"]


def _plain_heads(s):
    c = s["case"]
    f, attention = s["frequencies"]
    rot = c["rot"]
    angle = (s["positions"].double()[:, None] * f).remainder(2 * math.pi)
    cos, sin = ((t * attention).float()[:, None] for t in (angle.cos(), angle.sin()))
    first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if c["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))

    def one(t, w, to):
        t = t.float()
        if w is not None:
            t = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * w
        r = t.clone()
        a, b = t[..., first], t[..., second]
        r[..., first] = a * cos - b * sin
        r[..., second] = b * cos + a * sin
        return to.copy_(r)

    return [one(*v) for v in zip(s["heads"], s["weights"], s["to"])]


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return _plain_adapters(state) if kind == "adapters" else _plain_heads(state)
    from paper_2609_22106_b200 import binding as prq

    if kind == "adapters":
        return prq.linear_adapters(state["adapters"], state["x"], state["rows"], state["base"], out=state["out"], workspace=state["workspace"])
    q, k = state["heads"]
    if kind == "rotate":
        return prq.rotate_heads(state["rope"], state["positions"], q, k, out=state["to"])
    return prq.norm_rotate_heads(state["rope"], state["positions"], q, k, *state["weights"], eps=EPS, out=state["to"])


def work(case):
    c = case
    if c["kind"] == "adapters":
        M, K, R, P, N = c["M"], c["K"], c["R"], len(_parts(c)), sum(_parts(c))
        ranks = sum(_ranks(c)[: _used(c)])
        size = 2 if c["y"] == "bf16" else 4
        rows = M * (c["requests"] - c["bare"]) / c["requests"]
        mean = ranks / max(1, _used(c))
        return {"bytes": 2 * M * K + 2 * M * N * size + 2 * ranks * (P * K + N) + 4 * M, "flops": 2 * rows * mean * (P * K + N)}
    size, n = (2 if c["dtype"] == "bf16" else 4), c["M"] * (c["q"] + c["k"]) * c["D"]
    return {"bytes": 2 * size * n + 4 * c["M"], "flops": (4 * n if c["kind"] == "norm_rotate" else 0) + 3 * n * c["rot"] / c["D"]}


# ---- the same in 64 bits ------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_adapters(case, s) if case["kind"] == "adapters" else _exact_heads(case, s)


def _exact_adapters(c, s):
    y = s["base"].double()
    rows, ranks = s["rows"].tolist(), _ranks(c)
    for a in sorted(set(rows) - {-1}):
        at = torch.tensor([i for i, r in enumerate(rows) if r == a], device="cuda")
        x, begin = s["x"][at].double(), 0
        for p, n in enumerate(_parts(c)):
            A, B = s["A"][a, p, : ranks[a]].double(), s["B"][a, begin:begin + n, : ranks[a]].double()
            y[at, begin:begin + n] += s["scale"][a].double() * torch.einsum("mr,nr->mn", torch.einsum("mk,rk->mr", x, A), B)
            begin += n
    return y


def _exact_heads(c, s):
    o, d = _scaling(c), c["rot"]
    base = o["base"] * (FACTOR ** (d / (d - 2)) if o["scaling"] == "ntk" else 1.0)
    theta, attention = [], 1.0
    edge = lambda turns: d * math.log(ORIGINAL / (turns * 2 * math.pi)) / (2 * math.log(base))
    for i in range(d // 2):
        f = base ** (-2.0 * i / d)
        if o["scaling"] == "linear":
            f /= FACTOR
        elif o["scaling"] == "yarn":
            lo, hi = max(math.floor(edge(32.0)), 0), min(math.ceil(edge(1.0)), d - 1)
            t = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            f, attention = f * (1 - t) + f * t / FACTOR, 1 + 0.1 * math.log(FACTOR)
        elif o["scaling"] == "bands":
            wave = 2 * math.pi / f
            if wave > ORIGINAL / 1.0:
                f /= FACTOR
            elif wave > ORIGINAL / 4.0:
                t = (ORIGINAL / wave - 1.0) / (4.0 - 1.0)
                f = (1 - t) * f / FACTOR + t * f
        theta.append(f)
    turn = torch.outer(s["positions"].double(), torch.tensor(theta, dtype=torch.float64, device="cuda"))
    turn = torch.polar(torch.full_like(turn, attention), turn)[:, None, :]
    result = []
    for t, w in zip(s["heads"], s["weights"]):
        t = t.double()
        if w is not None:
            t = w.double() * t / (t.pow(2).sum(-1, keepdim=True) / c["D"] + EPS).sqrt()
        head, tail = t[..., :d], t[..., d:]
        shape = head.shape
        pairs = head.reshape(*shape[:-1], 2, d // 2).transpose(-1, -2) if c["layout"] == "half" else head.reshape(*shape[:-1], d // 2, 2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = (z.transpose(-1, -2) if c["layout"] == "half" else z).reshape(shape)
        result.append(torch.cat([z, tail], dim=-1))
    return result
