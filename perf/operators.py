"""Operators over tokens: real calls of them, in plain torch and through the library, and what each cannot do without.

Three operators that a model of K concurrent streams uses one behind the other: the norm of queries and keys with the
position rotation, linear attention with a decay for each head (a recurrent cell over tokens with a state per stream
slot), and cross attention of queries to an encoder's map of another length.  Map sizes, head counts and batches
are those of the benchmark configurations: 60 x 80 tokens of 128 channels (854 x 480 streams), 90 x 160 tokens of 256
channels (1920 x 1080 streams), seven tools, five and eight streams, clips of 60 frames.
"""
import math

import numpy as np
import torch

own = False      # True: run() calls the library's kernels; False: the plain form

EPS = 1e-6


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one tick of eight streams: a single token per stream, where the launch is all there is
        {"name": "rope_tick_b8", "op": "rope", "dtype": "bf16", "B": 8, "T": 1, "H": 4, "KV": 4, "D": 64, "rot": 64,
         "interleaved": False, "factor": 1.0, "ragged": False},
        # the tokens of eight full-HD maps, rotated with frequencies scaled for long contexts; maps cut to different lengths
        {"name": "rope_map_b8", "op": "rope", "dtype": "bf16", "B": 8, "T": 14400, "H": 4, "KV": 4, "D": 64, "rot": 32,
         "interleaved": True, "factor": 4.0, "ragged": True},
        # one tick of five streams
        {"name": "linear_tick_b5", "op": "linear", "dtype": "bf16", "B": 5, "T": 1, "H": 2, "KV": 2, "D": 64, "ragged": False,
         "slots": 8},
        # a server's tick: 256 sessions in slots of any order
        {"name": "linear_tick_b256", "op": "linear", "dtype": "bf16", "B": 256, "T": 1, "H": 8, "KV": 8, "D": 128,
         "ragged": False, "slots": 288},
        # a clip of 60 frames brings five streams' states up to date, some clips shorter
        {"name": "linear_clip_b5", "op": "linear", "dtype": "bf16", "B": 5, "T": 60, "H": 2, "KV": 2, "D": 64, "ragged": True,
         "slots": 8},
        # every token of eight full-HD maps
        {"name": "linear_map_b8", "op": "linear", "dtype": "bf16", "B": 8, "T": 14400, "H": 4, "KV": 4, "D": 64,
         "ragged": False, "slots": 8},
        # the fp32 path: two streams, an odd number of tokens, two heads that share keys and values
        {"name": "linear_fp32_b2", "op": "linear", "dtype": "fp32", "B": 2, "T": 4801, "H": 2, "KV": 1, "D": 64,
         "ragged": False, "slots": 2},
        # seven tools' queries of five streams, each reading the places of its own mask only; one tool sees nothing
        {"name": "cross_tools_b5", "op": "cross", "dtype": "bf16", "B": 5, "Tq": 7, "Tk": 4800, "H": 2, "KV": 2, "D": 64,
         "mask": True, "ragged": False},
        # the same for eight full-HD streams, without masks, maps cut to different lengths
        {"name": "cross_tools_b8", "op": "cross", "dtype": "bf16", "B": 8, "Tq": 7, "Tk": 14400, "H": 4, "KV": 4, "D": 64,
         "mask": False, "ragged": True},
        # every place of a map reads another map of its own size
        {"name": "cross_map_b8", "op": "cross", "dtype": "bf16", "B": 8, "Tq": 4800, "Tk": 4800, "H": 4, "KV": 4, "D": 64,
         "mask": False, "ragged": False},
        # every place of a map reads a full-HD map, wide heads
        {"name": "cross_map_b4", "op": "cross", "dtype": "bf16", "B": 4, "Tq": 4800, "Tk": 14400, "H": 2, "KV": 2, "D": 128,
         "mask": False, "ragged": True},
        # the fp32 path: an odd number of queries on the tiny configuration's 64 x 64 map
        {"name": "cross_fp32_b1", "op": "cross", "dtype": "fp32", "B": 1, "Tq": 1023, "Tk": 4096, "H": 2, "KV": 1, "D": 32,
         "mask": False, "ragged": False},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "linear", "cross"])
    KV = rng.choice([1, 2, 4])
    c = {"op": op, "dtype": rng.choice(["bf16", "bf16", "fp32"]), "B": _spread(rng, 1, 8), "H": KV * rng.choice([1, 1, 2]), "KV": KV,
         "D": rng.choice([32, 64, 64, 128]), "ragged": rng.random() < 0.5}
    if op == "rope":
        c.update(T=_spread(rng, 1, 14400), rot=rng.randrange(0, c["D"] // 8 + 1) * 8, interleaved=rng.random() < 0.5,
                 factor=rng.choice([1.0, 4.0]))
        c["T"] = max(1, min(c["T"], 8 * 14400 * 8 * 64 * 2 // (c["B"] * (c["H"] + KV) * c["D"] * _size(c))))
    elif op == "linear":
        if rng.random() < 0.4:
            c["B"], c["T"] = _spread(rng, 1, 256), 1
        else:
            c["T"] = _spread(rng, 2, 14400)
        c["slots"] = c["B"] + rng.randrange(0, 9)
        most = 8 * 14400 * 4 * 64 if c["dtype"] == "bf16" else 2 * 4801 * 2 * 64
        c["T"] = max(1, min(c["T"], most // (c["B"] * c["H"] * c["D"])))
        c["B"] = max(1, min(c["B"], 256 * 8 * 128 * 128 // (c["H"] * c["D"] * c["D"])))
    else:
        few = rng.random() < 0.5
        c.update(Tq=_spread(rng, 1, 16) if few else _spread(rng, 17, 4800), Tk=_spread(rng, 1, 14400), mask=rng.random() < 0.3)
        most = 4 * 4800 * 14400 * 2 * 128 if c["dtype"] == "bf16" else 1023 * 4096 * 2 * 32 * 4
        c["Tk"] = max(1, min(c["Tk"], most // (c["B"] * c["Tq"] * c["H"] * c["D"])))
    return c


def _size(c):
    return 2 if c["dtype"] == "bf16" else 4


def _lengths(B, T, ragged):
    """Entry b has T tokens, or down to half of them in even steps."""
    return [T - (b * T) // (2 * B) if ragged else T for b in range(B)]


def work(case):
    c, s, D = case, _size(case), case["D"]
    if c["op"] == "rope":
        rows = sum(_lengths(c["B"], c["T"], c["ragged"])) * (c["H"] + c["KV"])
        return {"bytes": 2 * rows * D * s, "flops": rows * (4 * D + 3 * c["rot"])}
    if c["op"] == "linear":
        tokens = sum(_lengths(c["B"], c["T"], c["ragged"]))
        return {"bytes": tokens * (2 * c["H"] + 2 * c["KV"]) * D * s + 2 * 4 * c["B"] * c["H"] * D * D,
                "flops": 4 * tokens * c["H"] * D * D}
    keys = sum(_lengths(c["B"], c["Tk"], c["ragged"]))
    return {"bytes": 2 * c["B"] * c["Tq"] * c["H"] * D * s + 2 * keys * c["KV"] * D * s + (keys * c["Tq"] if c["mask"] else 0),
            "flops": 4 * c["Tq"] * keys * c["H"] * D}


# ------------------------------------------------------------------------------------------------ inputs
def _frequencies(rot, factor):
    """Radians per position of the rot / 2 pairs, base 10000; with a factor over 1, pairs that turn less than once in 4096
    positions are slowed down by it, those that turn over 32 times are not, and a ramp joins the two.  And the gain that goes with it."""
    if rot == 0:
        return np.zeros(0), 1.0
    inv = 10000.0 ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    if factor == 1.0:
        return inv, 1.0
    turns = 4096.0 * inv / (2 * math.pi)
    keep = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
    return inv * (keep + (1.0 - keep) / factor), 0.1 * math.log(factor) + 1.0


def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 11)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    B, H, KV, D = c["B"], c["H"], c["KV"], c["D"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    s = {"case": c}
    if c["op"] == "rope":
        # one projection's output holds a token's queries, keys and values side by side; the operator reads the first two in place
        T = c["T"]
        qkv = (normal(B, T, H + 2 * KV, D) * 1.7 + 0.1).to(dt)
        s["q"], s["k"] = qkv[:, :, :H], qkv[:, :, H:H + KV]
        s["q_weight"], s["k_weight"] = 1 + 0.3 * normal(D), 1 + 0.3 * normal(D)
        first = torch.randint(0, 5_000_000, (B, 1), generator=g, device=dev)       # a day of frames
        s["positions"] = first + torch.arange(T, device=dev)[None]
        inv, s["gain"] = _frequencies(c["rot"], c["factor"])
        s["inv_freq"] = torch.from_numpy(inv).to(dev)
        s["lengths"] = torch.tensor(_lengths(B, T, True), dtype=torch.int32, device=dev) if c["ragged"] else None
        s["out"] = (torch.zeros(B, T, H, D, dtype=dt, device=dev), torch.zeros(B, T, KV, D, dtype=dt, device=dev))
    elif c["op"] == "linear":
        T = c["T"]
        qkv = normal(B, T, H + 2 * KV, D)
        qkv[:, :, H + KV:] += 0.2
        qkv = qkv.to(dt)
        s["q"], s["k"], s["v"] = qkv[:, :, :H], qkv[:, :, H:H + KV], qkv[:, :, H + KV:]
        # memories from two tokens to a few hundred
        s["log_decay"] = -torch.exp(torch.rand(H, generator=g, device=dev) * 5.5 - 6.0)
        s["state"] = normal(c["slots"], H, D, D)
        s["state_out"] = torch.zeros_like(s["state"])
        s["slots"] = torch.randperm(c["slots"], generator=g, device=dev)[:B].to(torch.int32)
        s["lengths"] = torch.tensor(_lengths(B, T, True), dtype=torch.int32, device=dev) if c["ragged"] else None
        s["scale"] = D ** -0.5
        s["out"] = torch.zeros(B, T, H, D, dtype=dt, device=dev)
    else:
        Tq, Tk = c["Tq"], c["Tk"]
        # heads from even to sharp
        sharp = torch.exp(torch.rand(H, 1, generator=g, device=dev) * 1.6 - 0.4)
        s["q"] = (normal(B, Tq, H, D) * sharp).to(dt)
        kv = normal(B, Tk, 2 * KV, D)
        kv[:, :, KV:] += 0.2
        kv = kv.to(dt)
        s["k"], s["v"] = kv[:, :, :KV], kv[:, :, KV:]
        s["lengths"] = torch.tensor(_lengths(B, Tk, True), dtype=torch.int32, device=dev) if c["ragged"] else None
        s["mask"] = None
        if c["mask"]:
            # a tool covers a run of places; the last tool of every entry is out of sight
            place = torch.arange(Tk, device=dev)
            centre = torch.rand(B, Tq, 1, generator=g, device=dev) * Tk
            reach = torch.rand(B, Tq, 1, generator=g, device=dev) * 0.2 * Tk + 1
            s["mask"] = ((place - centre).abs() < reach).to(torch.uint8)
            if Tq > 1:
                s["mask"][:, -1] = 0
        s["scale"] = D ** -0.5
        s["out"] = torch.zeros(B, Tq, H, D, dtype=dt, device=dev)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2402_04466_b200 import binding
        c = s["case"]
        if op == "rope":
            return list(binding.qk_norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], s["q_weight"], s["k_weight"], eps=EPS,
                                             interleaved=c["interleaved"], rot_scale=s["gain"], lengths=s["lengths"], out=s["out"]))
        if op == "linear":
            return list(binding.linear_attention(s["q"], s["k"], s["v"], s["log_decay"], s["state"], scale=s["scale"], slots=s["slots"],
                                                 lengths=s["lengths"], out=s["out"], state_out=s["state_out"]))
        return binding.cross_attention(s["q"], s["k"], s["v"], scale=s["scale"], kv_lengths=s["lengths"], mask=s["mask"], out=s["out"])
    return {"rope": _plain_rope, "linear": _plain_linear, "cross": _plain_cross}[op](s)


def _plain_rope(s):
    c = s["case"]
    rot, T = c["rot"], c["T"]
    angle = s["positions"].double()[:, :, None, None] * s["inv_freq"]
    cos, sin = (angle.cos() * s["gain"]).float(), (angle.sin() * s["gain"]).float()
    res = []
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = x.float()
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w
        if rot:
            a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if c["interleaved"] else (y[..., :rot // 2], y[..., rot // 2:rot])
            ra, rb = a * cos - b * sin, b * cos + a * sin
            r = torch.stack((ra, rb), -1).flatten(-2) if c["interleaved"] else torch.cat((ra, rb), -1)
            y = torch.cat((r, y[..., rot:]), -1)
        if s["lengths"] is not None:
            y = y * (torch.arange(T, device=y.device)[None] < s["lengths"][:, None])[:, :, None, None]
        res.append(y.to(x.dtype))
    return res


def _plain_linear(s):
    c = s["case"]
    B, T, H, KV, D = (c[n] for n in ("B", "T", "H", "KV", "D"))
    n = 64
    head = torch.arange(H, device=s["q"].device) // (H // KV)
    slots = s["slots"].long()
    S = s["state"][slots]
    out = torch.zeros(B, T, H, D, device=S.device)
    for t0 in range(0, T, n):
        q = s["q"][:, t0:t0 + n].float().transpose(1, 2)
        k = s["k"][:, t0:t0 + n].float()[:, :, head].transpose(1, 2)
        v = s["v"][:, t0:t0 + n].float()[:, :, head].transpose(1, 2)
        m = q.shape[2]
        here = torch.ones(B, 1, m, device=S.device)
        if s["lengths"] is not None:
            here = (torch.arange(t0, t0 + m, device=S.device)[None] < s["lengths"][:, None]).float()[:, None]
        # logarithm of the decay up to and including each token; tokens behind an entry's last one neither decay nor add
        L = torch.cumsum(here * s["log_decay"][None, :, None], -1)
        k = k * here[..., None]
        between = torch.where(torch.ones(m, m, device=S.device).tril() > 0, L[..., :, None] - L[..., None, :], -math.inf)
        o = ((q @ k.transpose(-1, -2)) * torch.exp(between)) @ v + (q @ S) * torch.exp(L)[..., None]
        out[:, t0:t0 + n] = (o * here[..., None] * s["scale"]).transpose(1, 2)
        S = S * torch.exp(L[..., -1])[..., None, None] + (k * torch.exp(L[..., -1:] - L)[..., None]).transpose(-1, -2) @ v
    state = torch.zeros_like(s["state"])
    state[slots] = S
    return [out.to(s["q"].dtype), state]


def _plain_cross(s):
    c = s["case"]
    B, Tq, Tk, H, KV, D = (c[n] for n in ("B", "Tq", "Tk", "H", "KV", "D"))
    dev = s["q"].device
    head = torch.arange(H, device=dev) // (H // KV)
    out = torch.empty(B, Tq, H, D, dtype=s["q"].dtype, device=dev)
    for b in range(B):
        q, k, v = s["q"][b].float().transpose(0, 1), s["k"][b].float()[:, head].transpose(0, 1), s["v"][b].float()[:, head].transpose(0, 1)
        z = (q @ k.transpose(-1, -2)) * s["scale"]
        if s["lengths"] is not None:
            z = torch.where(torch.arange(Tk, device=dev) < s["lengths"][b], z, -math.inf)
        if s["mask"] is not None:
            z = torch.where(s["mask"][b] != 0, z, -math.inf)
        top = z.max(-1, keepdim=True).values
        p = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
        total = p.sum(-1, keepdim=True)
        out[b] = ((p @ v) / torch.where(total == 0, 1.0, total)).transpose(0, 1).to(out.dtype)
    return out


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """What run() gives, from the definitions, in 64 bits."""
    s = prepare(case, seed)
    c = s["case"]
    B, H, KV, D = c["B"], c["H"], c["KV"], c["D"]
    if c["op"] == "rope":
        T, half = c["T"], c["rot"] // 2
        res = []
        for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
            y = x.double()
            y = y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / D + EPS) * w.double()
            # each pair is a complex number, turned by its angle
            first = [2 * i if c["interleaved"] else i for i in range(half)]
            second = [2 * i + 1 if c["interleaved"] else i + half for i in range(half)]
            turn = torch.polar(torch.full_like(s["positions"], 1.0, dtype=torch.float64)[..., None] * s["gain"],
                               s["positions"].double()[..., None] * s["inv_freq"])[:, :, None]
            z = torch.complex(y[..., first], y[..., second]) * turn
            y[..., first], y[..., second] = z.real, z.imag
            if s["lengths"] is not None:
                for b, n in enumerate(s["lengths"].tolist()):
                    y[b, n:] = 0
            res.append(y)
        return res
    group = H // KV
    if c["op"] == "linear":
        T = c["T"]
        q = s["q"].double() * s["scale"]
        k, v = s["k"].double().repeat_interleave(group, 2), s["v"].double().repeat_interleave(group, 2)
        decay = torch.exp(s["log_decay"].double())[None, :, None, None]
        slots = s["slots"].long()
        S = s["state"].double()[slots]
        out = torch.zeros(B, T, H, D, dtype=torch.float64, device=S.device)
        lengths = _lengths(B, T, c["ragged"])
        for t in range(T):           # entries are sorted from the longest to the shortest
            n = sum(1 for x in lengths if x > t)
            S[:n] = S[:n] * decay + k[:n, t, :, :, None] * v[:n, t, :, None, :]
            out[:n, t] = (q[:n, t, :, None, :] @ S[:n])[:, :, 0]
        state = torch.zeros_like(s["state"], dtype=torch.float64)
        state[slots] = S
        return [out, state]
    out = torch.zeros(B, c["Tq"], H, D, dtype=torch.float64, device=s["q"].device)
    for b, n in enumerate(_lengths(B, c["Tk"], c["ragged"])):
        for h in range(H):
            z = s["q"][b, :, h].double() @ s["k"][b, :n, h // group].double().T * s["scale"]
            if s["mask"] is not None:
                z[s["mask"][b, :, :n] == 0] = -math.inf
            out[b, :, h] = torch.softmax(z, -1).nan_to_num(0.0) @ s["v"][b, :n, h // group].double()
    return out
