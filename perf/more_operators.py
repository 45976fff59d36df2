"""Performance cases of the linear attention layer's operators.

Every case is one pass through one operator, as the program that serves such a layer calls it:

* ``prompt``  ``Lin.prompt``: linear attention with a decay for each head over the packed tokens of several prompts, from
              given states (or zero) to the states after them;
* ``step``    ``Lin.step``: the same for one token of each of n sequences;
* ``rot``     ``Rot.apply``: norms of queries and keys for each head and the rotation by their positions;
* ``q8``      ``Q8.matmul``: rows, quantized to 8 bits with a scale each, against 8-bit weights with a scale for each output.

H heads of queries share G states of K x V values (H / G neighbouring heads one), so there are G heads of keys and values.
The states of a ``prompt`` or ``step`` are read from the slots 0 .. n-1 and written to the slots n .. 2n-1, as where a
sequence is continued in a copy, so that a pass can be made again.
"""
from __future__ import annotations

import math

import torch

own = False  # True: the framework's operators; False: the plain forms below
DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CHUNK = 128  # positions a chunk of the plain form
EPS = 1e-5


def listed():
    return [
        # one long prompt of a 4096-channel layer: a single sequence has to fill the card
        dict(name="prompt-long", op="prompt", lens="16384", H=32, G=32, K=128, V=128, dtype="bf16", fresh=True),
        # prompts of a serving batch as they come: ragged, one of a single token, one empty, odd sizes, shared keys
        dict(name="prompt-ragged", op="prompt", lens="731,1,0,1290,64,65,2047", H=15, G=5, K=40, V=72, dtype="f16", fresh=False),
        # values twice as wide as keys in full precision, batch 4, further pieces of prompts begun before
        dict(name="prompt-f32", op="prompt", lens="2048,2048,2048,2048", H=12, G=12, K=64, V=128, dtype="f32", fresh=False),
        # one sequence of a 2048-channel layer, token by token: latency counts
        dict(name="step-one", op="step", n=1, H=16, G=16, K=128, V=128, dtype="bf16"),
        # a decode batch of a 4096-channel layer: the states are everything
        dict(name="step-batch", op="step", n=64, H=32, G=32, K=128, V=128, dtype="bf16"),
        # a token of each of four sequences of a 2048-channel layer: latency counts
        dict(name="rot-token", op="rot", T=4, H=16, G=16, P=128, R=128, norm="rms", pairs="half", dtype="bf16", far=4096),
        # the queries and keys of a long prompt of a 4096-channel layer
        dict(name="rot-prompt", op="rot", T=16384, H=32, G=32, P=128, R=128, norm="rms", pairs="half", dtype="bf16", far=16384),
        # odd sizes in full precision: part of a head turned, neighbours as pairs, far positions
        dict(name="rot-odd", op="rot", T=333, H=7, G=3, P=50, R=18, norm="layer", pairs="adjacent", dtype="f32", far=1 << 20),
        # the input projection of a 2048-channel layer (queries, keys, values and gate in one) for one token
        dict(name="q8-token", op="q8", R=1, N=8192, C=2048, dtype="bf16", bias=False),
        # its output projection for a decode batch
        dict(name="q8-batch", op="q8", R=64, N=2048, C=2048, dtype="f16", bias=False),
        # the input projection for a long prompt
        dict(name="q8-prompt", op="q8", R=16384, N=8192, C=2048, dtype="bf16", bias=False),
        # odd sizes in full precision
        dict(name="q8-odd", op="q8", R=67, N=1543, C=773, dtype="f32", bias=True),
    ]


def _log_int(rng, lo, hi, step=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))
    return max(lo, min(hi, v // step * step))


def _draw_heads(rng, most):
    """(H, G): neighbouring heads share a state, often just one."""
    H = rng.choice([_log_int(rng, 1, most), _log_int(rng, 8, most, 8)])
    return H, H // rng.choice([r for r in range(1, 9) if H % r == 0] + [1, 1, 1])


def draw(rng):
    op = rng.choice(["prompt", "prompt", "step", "rot", "q8", "q8"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("prompt", "step"):
        while True:
            H, G = _draw_heads(rng, 64)
            K, V = (rng.choice([32, 64, 128, 128, 256, _log_int(rng, 8, 256)]) for _ in "KV")
            c = dict(op=op, H=H, G=G, K=K, V=V, dtype=dtype)
            if op == "step":
                c["n"] = _log_int(rng, 1, 256)
                if H * max(K, V) <= 8192 and c["n"] * G * K * V <= 64 * 32 * 128 * 128:
                    return c
                continue
            n = rng.choice([1, 1, 2, 4, _log_int(rng, 2, 16)])
            longest = _log_int(rng, 2, 16384)
            lens = [longest if rng.random() < 0.4 else rng.choice([rng.randint(0, longest), _log_int(rng, 1, longest)])
                    for _ in range(n)]
            lens[rng.randrange(n)] = longest
            c.update(lens=",".join(str(v) for v in lens), fresh=rng.random() < 0.5)
            # the plain form's rows are all as long as the longest one
            if H * max(K, V) <= 8192 and n * longest * H * (K + V) <= 16384 * 32 * 256 and n * longest * G * K * V <= 1 << 33:
                return c
    if op == "rot":
        while True:
            H, G = _draw_heads(rng, 64)
            P, T = rng.choice([64, 128, 128, _log_int(rng, 2, 256)]), _log_int(rng, 1, 16384)
            if T * (H + G) * P <= 16384 * 64 * 128:
                break
        R = rng.choice([P // 2 * 2, P // 2 * 2, 2 * rng.randint(0, P // 2)])
        return dict(op=op, T=T, H=H, G=G, P=P, R=R, norm=rng.choice(["rms", "rms", "layer", "none"]),
                    pairs=rng.choice(["half", "half", "adjacent"]), dtype=dtype, far=_log_int(rng, 16, 1 << 20))
    while True:
        R, N, C = _log_int(rng, 1, 16384), _log_int(rng, 64, 16384, rng.choice([1, 16])), _log_int(rng, 64, 16384, rng.choice([1, 32]))
        if R * N * C <= 16384 * 8192 * 2048 and N * C <= 1 << 26 and R * max(N, C) <= 1 << 27:
            return dict(op=op, R=R, N=N, C=C, dtype=dtype, bias=rng.random() < 0.5)


# ---------------------------------------------------------------- inputs

def _gen(seed, stream):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) * 32 + stream)
    return g


def _randn(seed, stream, shape):
    return torch.randn(shape, generator=_gen(seed, stream), device=DEVICE)


def _rand(seed, stream, shape):
    return torch.rand(shape, generator=_gen(seed, stream), device=DEVICE)


def _lens(case):
    return [int(v) for v in case["lens"].split(",")] if case["op"] == "prompt" else [1] * case["n"]


def _lin_data(case, seed):
    """Normed queries and keys, values, and heads whose memory reaches from a few tokens to some hundreds back."""
    H, G, K, V = (case[k] for k in "HGKV")
    lens, dt = _lens(case), TYPES[case["dtype"]]
    n, T = len(lens), sum(lens)
    s = dict(case=case, n=n, T=T, scale=K ** -0.5, decay=-torch.exp2(-1 - 8 * _rand(seed, 0, (1, G))),
             q=_randn(seed, 1, (T, H * K)).to(dt), k=_randn(seed, 2, (T, G * K)).to(dt), v=_randn(seed, 3, (T, G * V)).to(dt),
             state=None if case.get("fresh") else 3 * _randn(seed, 4, (n, G, K, V)))
    offs = [0]
    for m in lens:
        offs.append(offs[-1] + m)
    s["offsets"] = torch.tensor(offs, dtype=torch.int32, device=DEVICE)
    s["src"] = torch.full((n,), -1, dtype=torch.int32, device=DEVICE) if s["state"] is None else torch.arange(
        n, dtype=torch.int32, device=DEVICE)
    s["dst"] = torch.arange(n, 2 * n, dtype=torch.int32, device=DEVICE)
    return s


def _rot_data(case, seed):
    T, H, G, P, R, dt = case["T"], case["H"], case["G"], case["P"], case["R"], TYPES[case["dtype"]]
    weight = lambda k: 1 + 0.1 * _randn(seed, k, (1, P)) if case["norm"] != "none" else None  # noqa: E731
    start = torch.randint(0, max(case["far"] - T, 1), (1,), generator=_gen(seed, 4), device=DEVICE)
    return dict(case=case, q=(3 * _randn(seed, 0, (T, H * P))).to(dt), k=(3 * _randn(seed, 1, (T, G * P))).to(dt),
                q_w=weight(2), k_w=weight(3),
                positions=(start + torch.arange(T, device=DEVICE)).to(torch.int32),
                freqs=10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device=DEVICE) / max(R, 1)))


def _q8_data(case, seed):
    R, N, C = case["R"], case["N"], case["C"]
    codes = torch.randint(-127, 128, (1, N, C), generator=_gen(seed, 0), device=DEVICE, dtype=torch.int8)
    scales = (0.5 + _rand(seed, 1, (1, N))) / (73 * math.sqrt(C))
    # rows of a residual stream: a few channels are far larger than the others
    x = _randn(seed, 2, (R, C)) * torch.exp(0.5 * _randn(seed, 3, (1, C)))
    return dict(case=case, codes=codes, scales=scales, bias=0.1 * _randn(seed, 4, (1, N)) if case["bias"] else None,
                x=x.to(TYPES[case["dtype"]]))


def _data(case, seed):
    return {"rot": _rot_data, "q8": _q8_data}.get(case["op"], _lin_data)(case, seed)


# ----------------------------------------------------------- prepare, run

def prepare(case, seed):
    s = _data(case, seed)
    if own:
        import paper_2410_12982_amd.lcsm as lcsm
        if case["op"] == "rot":
            s["ctx"] = lcsm.Rot(case["P"], case["H"], case["G"], freqs=s["freqs"], pairs=case["pairs"], norm=case["norm"], eps=EPS,
                                q_weight=s["q_w"], k_weight=s["k_w"], dtype=TYPES[case["dtype"]], device=DEVICE)
        elif case["op"] == "q8":
            s["ctx"] = lcsm.Q8(s["codes"], s["scales"], bias=s["bias"], max_rows=case["R"])
        else:
            s["ctx"] = ctx = lcsm.Lin(s["decay"], slots=2 * s["n"], heads=case["H"], keys=case["K"], values=case["V"],
                                      scale=s["scale"], dtype=TYPES[case["dtype"]],
                                      max_tokens=s["T"] if case["op"] == "prompt" else 0)
            if s["state"] is not None:
                ctx.state(0)[:s["n"]].copy_(s["state"])
    return s


def run(state):
    op = state["case"]["op"]
    if own:
        ctx = state["ctx"]
        if op == "rot":
            q, k = ctx.apply(0, state["q"], state["k"], state["positions"])
            return {"q": q, "k": k}
        if op == "q8":
            return {"y": ctx.matmul(0, state["x"])}
        if op == "prompt":
            y = ctx.prompt(0, state["q"], state["k"], state["v"], offsets=state["offsets"], src=state["src"], dst=state["dst"])
        else:
            y = ctx.step(0, state["q"], state["k"], state["v"], src=state["src"], dst=state["dst"])
        return {"y": y, "state": ctx.state(0)[state["n"]:]}
    return {"rot": _plain_rot, "q8": _plain_q8, "step": _plain_step, "prompt": _plain_prompt}[op](state)


# ------------------------------------------------------------ plain forms

def _powers(g, k):
    """exp(g (i - j)) for j <= i < k, 0 above: [G, k, k]."""
    i = torch.arange(k, device=DEVICE)
    far = i[:, None] - i
    return torch.where(far >= 0, torch.exp(g[:, None, None] * far.clamp(min=0)), torch.zeros((), device=DEVICE))


def _plain_prompt(s):
    """Chunks: inside a chunk a masked product of queries and keys, from chunk to chunk the states as another one.  A
    sequence's rows end at the end of its last chunk, so that what pads it comes first."""
    c = s["case"]
    H, G, K, V = (c[k] for k in "HGKV")
    n, lens, per = s["n"], _lens(c), H // G
    nc = -(-max(max(lens), 1) // CHUNK)
    Tm = nc * CHUNK
    offs = s["offsets"].long()
    at = offs[1:, None] - Tm + torch.arange(Tm, device=DEVICE)
    inside = at >= offs[:-1, None]
    rows = lambda x: torch.cat([x, x.new_zeros((1, x.shape[1]))])[torch.where(inside, at, s["T"])].float()  # noqa: E731
    q = rows(s["q"]).view(n, nc, CHUNK, G, per, K).permute(0, 1, 3, 4, 2, 5)  # [n, nc, G, per, Q, K]
    k = rows(s["k"]).view(n, nc, CHUNK, G, K).permute(0, 1, 3, 2, 4)
    v = rows(s["v"]).view(n, nc, CHUNK, G, V).permute(0, 1, 3, 2, 4)
    g = s["decay"][0]
    i = torch.arange(CHUNK, device=DEVICE)
    y = ((q @ k.transpose(-1, -2).unsqueeze(3)) * _powers(g, CHUNK)[:, None]) @ v.unsqueeze(3)
    # what a chunk adds to the state at its end
    local = (k * torch.exp(g[:, None] * (CHUNK - 1 - i))[..., None]).transpose(-1, -2) @ v  # [n, nc, G, K, V]
    between = _powers(g * CHUNK, nc)  # [G, to, from]
    after = (between @ local.permute(0, 2, 1, 3, 4).reshape(n, G, nc, K * V)).view(n, G, nc, K, V)
    into = torch.cat([after.new_zeros((n, G, 1, K, V)), after[:, :, :-1]], 2)
    start = torch.zeros((n, G, K, V), device=DEVICE) if s["state"] is None else s["state"]
    count = (offs[1:] - offs[:-1]).view(n, 1, 1, 1)
    final = after[:, :, -1] + start * torch.exp(g[:, None, None] * count)
    reach = torch.exp(g[:, None] * (i + 1))  # [G, Q]
    y = y + (q * reach[:, None, :, None]) @ into.permute(0, 2, 1, 3, 4).unsqueeze(3)
    y = y.permute(0, 1, 4, 2, 3, 5).reshape(n, Tm, G, per, V)
    if s["state"] is not None:
        # tokens since the sequence's first one; its own state has decayed that often
        t = (at - offs[:-1, None] + 1).clamp(min=0)
        whole = q.permute(0, 1, 4, 2, 3, 5).reshape(n, Tm, G, per, K) * torch.exp(g * t[..., None])[..., None, None]
        y = y + (whole.permute(0, 2, 3, 1, 4) @ start.unsqueeze(2)).permute(0, 3, 1, 2, 4)
    y = y.reshape(n, Tm, H * V)[inside] * s["scale"]
    return {"y": y.to(s["q"].dtype), "state": final}


def _plain_step(s):
    c = s["case"]
    H, G, K, V = (c[k] for k in "HGKV")
    n = s["n"]
    q, k, v = s["q"].float().view(n, G, H // G, K), s["k"].float().view(n, G, K, 1), s["v"].float().view(n, G, 1, V)
    state = s["state"] * torch.exp(s["decay"][0])[:, None, None] + k * v
    return {"y": ((q @ state) * s["scale"]).view(n, H * V).to(s["q"].dtype), "state": state}


def _plain_rot(s):
    c = s["case"]
    P, R = c["P"], c["R"]
    angle = s["positions"].double()[:, None] * s["freqs"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def one(x, heads, weight):
        v = x.float().view(-1, heads, P)
        if c["norm"] == "layer":
            v = v - v.mean(-1, keepdim=True)
        if c["norm"] != "none":
            v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * weight[0]
        if c["pairs"] == "half":
            a, b = v[..., :R // 2], v[..., R // 2:R]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        else:
            a, b = v[..., 0:R:2], v[..., 1:R:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        return torch.cat([turned, v[..., R:]], -1).reshape(-1, heads * P).to(x.dtype)

    return {"q": one(s["q"], c["H"], s["q_w"]), "k": one(s["k"], c["G"], s["k_w"])}


def _plain_q8(s):
    x = s["x"].float()
    # (64 bits round the scale, and decide between two codes that are almost equally near)
    scale = (x.abs().amax(-1, keepdim=True).double() / 127).float()
    codes = torch.where(scale > 0, torch.round(x.double() / scale.double()), torch.zeros((), dtype=torch.float64, device=DEVICE))
    y = (codes.clamp(-127, 127).float() @ s["codes"][0].float().T) * scale * s["scales"][0]
    return {"y": (y if s["bias"] is None else y + s["bias"][0]).to(s["x"].dtype)}


# ------------------------------------------------------------ work, exact

def work(case):
    """Inputs, weights and states read once, outputs and states written once; for linear attention the operations of its
    recurrence (a position adds to every state once, and each of its heads reads one)."""
    e = TYPES[case["dtype"]].itemsize
    if case["op"] == "rot":
        cells = case["T"] * (case["H"] + case["G"]) * case["P"]
        return {"bytes": 2.0 * e * cells + 4 * case["T"], "flops": 8.0 * cells}
    if case["op"] == "q8":
        R, N, C = case["R"], case["N"], case["C"]
        return {"bytes": N * C + N * (8.0 if case["bias"] else 4.0) + e * R * (N + C), "flops": 2.0 * R * N * C}
    H, G, K, V = (case[k] for k in "HGKV")
    n, T = len(_lens(case)), sum(_lens(case))
    return {"bytes": e * T * (H + G) * (K + V) + 4.0 * n * G * K * V * (1 if case.get("fresh") else 2),
            "flops": 2.0 * T * (H + G) * K * V}


def exact(case, seed):
    """The definitions in 64 bits: the recurrence position by position, the rotation as a complex product."""
    s = _data(case, seed)
    if case["op"] == "rot":
        T, P, R = case["T"], case["P"], case["R"]
        turn = torch.polar(torch.ones((T, 1, R // 2), dtype=torch.float64, device=DEVICE),
                           (s["positions"].double()[:, None] * s["freqs"])[:, None])
        first = torch.arange(R // 2, device=DEVICE) * (1 if case["pairs"] == "half" else 2)
        second = first + (R // 2 if case["pairs"] == "half" else 1)
        out = {}
        for name, heads in (("q", case["H"]), ("k", case["G"])):
            v = s[name].double().reshape(T, heads, P)
            if case["norm"] != "none":
                var, mean = torch.var_mean(v, -1, correction=0, keepdim=True)
                v = (v - mean) / (var + EPS).sqrt() if case["norm"] == "layer" else v / (var + mean * mean + EPS).sqrt()
                v = v * s[name + "_w"].double()
            z = torch.complex(v[..., first], v[..., second]) * turn
            v = v.clone()
            v[..., first], v[..., second] = z.real, z.imag
            out[name] = v.reshape(T, heads * P)
        return out
    if case["op"] == "q8":
        x = s["x"].double()
        scale = (x.abs().amax(-1, keepdim=True) / 127).float().double()  # a scale is a number of 32 bits
        q = torch.round(x / scale.clamp(min=1e-300)).clamp(-127, 127)
        y = torch.nn.functional.linear(q, s["codes"][0].double()) * (scale * s["scales"].double())
        return {"y": y if s["bias"] is None else y + s["bias"].double()}
    H, G, K, V = (case[k] for k in "HGKV")
    n, lens, per = s["n"], _lens(case), H // G
    longest = max(lens)
    padded = {}
    for name, width in (("q", (G, per, K)), ("k", (G, K, 1)), ("v", (G, 1, V))):
        padded[name] = torch.zeros((longest, n) + width, dtype=torch.float64, device=DEVICE)
    at, keep = 0, torch.zeros((longest, n, 1, 1, 1), dtype=torch.bool, device=DEVICE)
    for i, m in enumerate(lens):
        for name in "qkv":
            padded[name][:m, i] = s[name][at:at + m].double().reshape((m,) + tuple(padded[name].shape[2:]))
        keep[:m, i] = True
        at += m
    lam = torch.exp(s["decay"][0].double())[:, None, None]
    h = torch.zeros((n, G, K, V), dtype=torch.float64, device=DEVICE) if s["state"] is None else s["state"].double()
    y = torch.zeros((longest, n, G, per, V), dtype=torch.float64, device=DEVICE)
    for t in range(longest):
        h = torch.where(keep[t], h * lam + padded["k"][t] * padded["v"][t], h)
        torch.matmul(padded["q"][t], h, out=y[t])
    y = torch.cat([y[:m, i] for i, m in enumerate(lens)]).reshape(s["T"], H * V) * s["scale"]
    return {"y": y, "state": h}
