"""More operators over tokens: real calls of them, in plain torch and through the library, and what each cannot do without.

Two operators beside the recurrent cell and the attention that a model of K concurrent streams has already: the gated delta
rule (a cell whose state corrects what it says of a key instead of only adding to it) and differential attention (the
difference of two softmax maps, which takes away the weight that every place of a map gets).  Map sizes, head counts and batches
are those of the benchmark configurations: 60 x 80 tokens of 128 channels (854 x 480 streams), 90 x 160 tokens of 256
channels (1920 x 1080 streams), seven tools, five and eight streams, clips of 60 frames.
"""
import math

import torch

own = False      # True: run() calls the library's kernels; False: the plain form

EPS = 1e-5
LAMBDA_INIT = 0.8 - 0.6 * math.exp(-0.3)      # of a model's second layer


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one tick of five streams: a single token per stream, where the launch is all there is
        {"name": "delta_tick_b5", "op": "delta", "dtype": "bf16", "B": 5, "T": 1, "H": 2, "QK": 2, "D": 64, "ragged": False, "slots": 8},
        # a server's tick: 256 sessions in slots of any order, two value heads to a key head
        {"name": "delta_tick_b256", "op": "delta", "dtype": "bf16", "B": 256, "T": 1, "H": 8, "QK": 4, "D": 128, "ragged": False,
         "slots": 288},
        # a clip of 60 frames brings five streams' states up to date, some clips shorter
        {"name": "delta_clip_b5", "op": "delta", "dtype": "bf16", "B": 5, "T": 60, "H": 2, "QK": 2, "D": 64, "ragged": True, "slots": 8},
        # a server that starts 64 sessions at once, each with an odd number of frames behind it, wide heads
        {"name": "delta_start_b64", "op": "delta", "dtype": "bf16", "B": 64, "T": 497, "H": 4, "QK": 2, "D": 128, "ragged": True,
         "slots": 64},
        # every token of eight full-HD maps
        {"name": "delta_map_b8", "op": "delta", "dtype": "bf16", "B": 8, "T": 14400, "H": 4, "QK": 4, "D": 64, "ragged": False,
         "slots": 8},
        # the fp32 path: two streams, an odd number of tokens, two value heads that share queries and keys
        {"name": "delta_fp32_b2", "op": "delta", "dtype": "fp32", "B": 2, "T": 4801, "H": 2, "QK": 1, "D": 64, "ragged": False,
         "slots": 2},
        # seven tools' queries read the last 60 frames' tokens of five streams: the smallest call
        {"name": "diff_clip_b5", "op": "diff", "dtype": "bf16", "B": 5, "Tq": 7, "Tk": 60, "H": 2, "KV": 2, "D": 64, "mask": False,
         "ragged": True, "norm": True},
        # seven tools' queries of five streams, each reading the places of its own mask only; one tool sees nothing
        {"name": "diff_tools_b5", "op": "diff", "dtype": "bf16", "B": 5, "Tq": 7, "Tk": 4800, "H": 2, "KV": 2, "D": 64, "mask": True,
         "ragged": False, "norm": True},
        # the same for eight full-HD streams, without masks, maps cut to different lengths
        {"name": "diff_tools_b8", "op": "diff", "dtype": "bf16", "B": 8, "Tq": 7, "Tk": 14400, "H": 4, "KV": 4, "D": 64, "mask": False,
         "ragged": True, "norm": True},
        # every place of a map reads another map of its own size
        {"name": "diff_map_b8", "op": "diff", "dtype": "bf16", "B": 8, "Tq": 4800, "Tk": 4800, "H": 4, "KV": 4, "D": 64, "mask": False,
         "ragged": False, "norm": True},
        # every place of a map reads a full-HD map, wide heads
        {"name": "diff_map_b4", "op": "diff", "dtype": "bf16", "B": 4, "Tq": 4800, "Tk": 14400, "H": 2, "KV": 2, "D": 128,
         "mask": False, "ragged": True, "norm": True},
        # the fp32 path: an odd number of queries on the tiny configuration's 64 x 64 map, without the norm
        {"name": "diff_fp32_b1", "op": "diff", "dtype": "fp32", "B": 1, "Tq": 1023, "Tk": 4096, "H": 2, "KV": 1, "D": 32, "mask": False,
         "ragged": False, "norm": False},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    shared = rng.choice([1, 2, 4])
    c = {"op": rng.choice(["delta", "diff"]), "dtype": rng.choice(["bf16", "bf16", "fp32"]), "B": _spread(rng, 1, 8),
         "H": shared * rng.choice([1, 1, 2]), "D": rng.choice([32, 64, 64, 128]), "ragged": rng.random() < 0.5}
    bf16 = c["dtype"] == "bf16"
    if c["op"] == "delta":
        c["QK"] = shared
        kind = rng.random()
        if kind < 0.3:
            c["B"], c["T"] = _spread(rng, 1, 256), 1
        elif kind < 0.6:
            c["B"], c["T"] = _spread(rng, 8, 64), _spread(rng, 2, 600)
        else:
            c["T"] = _spread(rng, 2, 14400)
        most = 8 * 14400 * 4 * 64 if bf16 else 2 * 4801 * 2 * 64
        c["T"] = max(1, min(c["T"], most // (c["B"] * c["H"] * c["D"])))
        c["B"] = max(1, min(c["B"], 256 * 8 * 128 * 128 // (c["H"] * c["D"] * c["D"])))
        c["slots"] = c["B"] + rng.randrange(0, 9)
    else:
        few = rng.random() < 0.5
        c.update(KV=shared, Tq=_spread(rng, 1, 16) if few else _spread(rng, 17, 4800 if bf16 else 1023), Tk=_spread(rng, 1, 14400),
                 mask=rng.random() < 0.3, norm=rng.random() < 0.7)
        most = 4 * 4800 * 14400 * 2 * 128 if bf16 else 1023 * 4096 * 2 * 32 * 4
        c["Tk"] = max(1, min(c["Tk"], most // (c["B"] * c["Tq"] * c["H"] * c["D"])))
    return c


def _size(c):
    return 2 if c["dtype"] == "bf16" else 4


def _lengths(B, T, ragged):
    """Entry b has T tokens, or down to half of them in even steps."""
    return [T - (b * T) // (2 * B) if ragged else T for b in range(B)]


def work(case):
    c, s, D, H = case, _size(case), case["D"], case["H"]
    if c["op"] == "delta":
        tokens = sum(_lengths(c["B"], c["T"], c["ragged"]))
        # S^T k and S^T q, 2 D^2 each, and the state's decay and correction, 3 D^2
        return {"bytes": tokens * ((2 * c["QK"] + 2 * H) * D * s + 2 * 4 * H) + 2 * 4 * c["B"] * H * D * D, "flops": 7 * tokens * H * D * D}
    keys = sum(_lengths(c["B"], c["Tk"], c["ragged"]))
    # the scores of two halves of a head, and two maps' sums of whole values
    return {"bytes": 2 * c["B"] * c["Tq"] * H * D * s + 2 * keys * c["KV"] * D * s + (keys * c["Tq"] if c["mask"] else 0),
            "flops": 6 * c["Tq"] * keys * H * D}


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 13)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    B, H, D = c["B"], c["H"], c["D"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    s = {"case": c, "scale": D ** -0.5}
    if c["op"] == "delta":
        T, QK = c["T"], c["QK"]
        # queries and keys as the norm leaves them, of length 1; tokens of one place in a clip or map resemble each other
        qk = normal(B, T, 2 * QK, D) + 0.7 * normal(B, 1, 2 * QK, D)
        qk = (qk / qk.norm(dim=-1, keepdim=True)).to(dt)
        s["q"], s["k"] = qk[:, :, :QK], qk[:, :, QK:]
        s["v"] = (normal(B, T, H, D) + 0.2).to(dt)
        # gates as a model makes them: a rate per head times a softplus, and a sigmoid; memories from a few tokens to some hundreds
        rate = torch.exp(torch.rand(H, generator=g, device=dev) * 4.5 - 5.0)
        s["log_decay"] = -rate * torch.nn.functional.softplus(normal(B, T, H) + 0.5)
        s["beta"] = torch.sigmoid(normal(B, T, H))
        s["state"] = normal(c["slots"], H, D, D)
        s["state_out"] = torch.zeros_like(s["state"])
        s["slots"] = torch.randperm(c["slots"], generator=g, device=dev)[:B].to(torch.int32)
        s["lengths"] = torch.tensor(_lengths(B, T, True), dtype=torch.int32, device=dev) if c["ragged"] else None
        s["scale"] = 1.0
        s["out"] = torch.zeros(B, T, H, D, dtype=dt, device=dev)
    else:
        Tq, Tk, KV = c["Tq"], c["Tk"], c["KV"]
        # heads from even to sharp
        sharp = torch.exp(torch.rand(H, 1, generator=g, device=dev) * 1.6 - 0.4)
        s["q"] = (normal(B, Tq, H, D) * sharp).to(dt)
        # one projection's output holds keys and values side by side
        kv = normal(B, Tk, 2 * KV, D)
        kv[:, :, KV:] += 0.2
        kv = kv.to(dt)
        s["k"], s["v"] = kv[:, :, :KV], kv[:, :, KV:]
        s["lambda_vectors"] = 0.1 * normal(4, D // 2)
        s["norm_weight"] = 1 + 0.3 * normal(D) if c["norm"] else None
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
        s["scale"] = (D // 2) ** -0.5
        s["out"] = torch.zeros(B, Tq, H, D, dtype=dt, device=dev)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    c = s["case"]
    if own:
        from paper_2402_04466_b200 import binding
        if c["op"] == "delta":
            return list(binding.delta_rule(s["q"], s["k"], s["v"], s["log_decay"], s["beta"], s["state"], scale=s["scale"], slots=s["slots"],
                                           lengths=s["lengths"], out=s["out"], state_out=s["state_out"]))
        return binding.differential_attention(s["q"], s["k"], s["v"], s["lambda_vectors"], LAMBDA_INIT, scale=s["scale"], norm=c["norm"],
                                              norm_weight=s["norm_weight"], eps=EPS, out_scale=1 - LAMBDA_INIT,
                                              kv_lengths=s["lengths"], mask=s["mask"], out=s["out"])
    return _plain_delta(s) if c["op"] == "delta" else _plain_diff(s)


def _plain_delta(s):
    """Chunks of 64 tokens: all of their inverses at once, then the states one chunk behind the other."""
    c = s["case"]
    B, T, H, D = c["B"], c["T"], c["H"], c["D"]
    n = min(64, T)
    N = -(-T // n)
    dev = s["q"].device
    head = torch.arange(H, device=dev) // (H // c["QK"])
    here = torch.ones(B, T, 1, device=dev)
    if s["lengths"] is not None:
        here = (torch.arange(T, device=dev)[None] < s["lengths"][:, None]).float()[..., None]

    def chunks(x):                # [B][T][H][...] -> [B][H][N][n][...], zeros behind the last token
        x = torch.cat((x, torch.zeros(B, N * n - T, *x.shape[2:], device=dev)), 1)
        return x.reshape(B, N, n, *x.shape[2:]).movedim(3, 1)

    q, k = chunks(s["q"].float()[:, :, head]), chunks(s["k"].float()[:, :, head] * here[..., None])
    v, beta = chunks(s["v"].float()), chunks(s["beta"] * here)[..., None]
    # logarithm of the decay within a chunk up to and including each token, in 64 bits: differences of far tokens are taken
    L = torch.cumsum(chunks(s["log_decay"] * here).double(), -1)
    last = L[..., -1:]
    low = torch.ones(n, n, device=dev).tril() > 0
    between = torch.exp(torch.where(low, L[..., :, None] - L[..., None, :], -math.inf)).float()
    up, down, whole = torch.exp(L).float()[..., None], torch.exp(last - L).float()[..., None], torch.exp(last).float()[..., None]
    # (1 + A)^-1 = (1 - A)(1 + A^2)(1 + A^4)..., A strictly lower triangular; in 64 bits: of keys that resemble each other the powers
    # grow far beyond what is left of their sum
    A = ((k @ k.transpose(-1, -2)) * between * beta * (torch.ones(n, n, device=dev).tril(-1) > 0)).double()
    inverse, power, reach = torch.eye(n, dtype=torch.float64, device=dev) - A, A, 1
    while 2 * reach < n:
        power, reach = power @ power, 2 * reach
        inverse = inverse + power @ inverse
    inverse = inverse.float()
    V, K = inverse @ (v * beta), inverse @ (k * beta * up)
    P = (q @ k.transpose(-1, -2)) * between
    slots = s["slots"].long()
    S = s["state"][slots]
    out = torch.empty(B, H, N, n, D, device=dev)
    for i in range(N):
        u = V[:, :, i] - K[:, :, i] @ S
        out[:, :, i] = (q[:, :, i] * up[:, :, i]) @ S + P[:, :, i] @ u
        S = S * whole[:, :, i] + (k[:, :, i] * down[:, :, i]).transpose(-1, -2) @ u
    out = out.movedim(1, 3).reshape(B, N * n, H, D)[:, :T] * here[..., None] * s["scale"]
    state = torch.zeros_like(s["state"])
    state[slots] = S
    return [out.to(s["q"].dtype), state]


def _plain_diff(s):
    c = s["case"]
    B, Tq, Tk, H, KV, D = (c[n] for n in ("B", "Tq", "Tk", "H", "KV", "D"))
    dev = s["q"].device
    head = torch.arange(H, device=dev) // (H // KV)
    a = s["lambda_vectors"]
    lam = torch.exp((a[0] * a[1]).sum()) - torch.exp((a[2] * a[3]).sum()) + LAMBDA_INIT
    out = torch.empty(B, Tq, H, D, dtype=s["q"].dtype, device=dev)
    for b in range(B):
        v = s["v"][b].float()[:, head].transpose(0, 1)
        seen = torch.ones(1, Tk, dtype=torch.bool, device=dev)
        if s["lengths"] is not None:
            seen = seen & (torch.arange(Tk, device=dev) < s["lengths"][b])
        if s["mask"] is not None:
            seen = seen & (s["mask"][b] != 0)
        y = []
        for half in (slice(0, D // 2), slice(D // 2, D)):
            q, k = s["q"][b, :, :, half].float().transpose(0, 1), s["k"][b, :, :, half].float()[:, head].transpose(0, 1)
            z = torch.where(seen, (q @ k.transpose(-1, -2)) * s["scale"], -math.inf)
            top = z.max(-1, keepdim=True).values
            p = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
            total = p.sum(-1, keepdim=True)
            y.append((p @ v) / torch.where(total == 0, 1.0, total))
        y = y[0] - lam * y[1]
        if c["norm"]:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * s["norm_weight"]
        out[b] = (y * (1 - LAMBDA_INIT)).transpose(0, 1).to(out.dtype)
    return out


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """What run() gives, from the definitions, in 64 bits."""
    s = prepare(case, seed)
    c = s["case"]
    B, H, D = c["B"], c["H"], c["D"]
    if c["op"] == "delta":
        T, group = c["T"], H // c["QK"]
        q, k = (s[x].double().repeat_interleave(group, 2)[..., None] for x in ("q", "k"))
        v, beta = s["v"].double()[:, :, :, None], s["beta"].double()[..., None, None]
        decay = torch.exp(s["log_decay"].double())[..., None, None]
        slots = s["slots"].long()
        S = s["state"].double()[slots]
        out = torch.zeros(B, T, H, D, dtype=torch.float64, device=S.device)
        lengths = _lengths(B, T, c["ragged"])
        for t in range(T):           # entries are sorted from the longest to the shortest
            n = sum(1 for x in lengths if x > t)
            old = S[:n] * decay[:n, t]
            said = k[:n, t].transpose(-1, -2) @ old
            S[:n] = old + k[:n, t] @ (beta[:n, t] * (v[:n, t] - said))
            out[:n, t] = (q[:n, t].transpose(-1, -2) @ S[:n])[:, :, 0] * s["scale"]
        state = torch.zeros_like(s["state"], dtype=torch.float64)
        state[slots] = S
        return [out, state]
    half, group = D // 2, H // c["KV"]
    q1, k1, q2, k2 = s["lambda_vectors"].double()
    lam = math.exp(float(q1 @ k1)) - math.exp(float(q2 @ k2)) + LAMBDA_INIT
    out = torch.zeros(B, c["Tq"], H, D, dtype=torch.float64, device=s["q"].device)
    for b, n in enumerate(_lengths(B, c["Tk"], c["ragged"])):
        for h in range(H):
            q, k, v = s["q"][b, :, h].double(), s["k"][b, :n, h // group].double(), s["v"][b, :n, h // group].double()
            weights = []
            for x, y in ((q[:, :half], k[:, :half]), (q[:, half:], k[:, half:])):
                z = x @ y.T * s["scale"]
                if s["mask"] is not None:
                    z[s["mask"][b, :, :n] == 0] = -math.inf
                weights.append(torch.softmax(z, -1).nan_to_num(0.0))
            y = (weights[0] - lam * weights[1]) @ v
            if c["norm"]:
                y = y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / D + EPS) * s["norm_weight"].double()
            out[b, :, h] = y * (1 - LAMBDA_INIT)
    return out
