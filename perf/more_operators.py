"""The operators of a served attention layer between its projections and its cache, as cases to measure: causal attention over
packed prompts, the norms and position rotation of queries and keys, and low-rank adapters beside a shared projection.

`listed()` names the cases, `draw(rng)` gives more of the same ranges, `prepare(case, seed)` makes what a program has
in hand before the call, and `run(state)` is one pass: with `own` false in elementary torch operations in 32 bits (angles
in 64), with `own` true through the calls of `paper_2410_07505_b200.cq`.  `exact(case, seed)` is the same pass in 64 bits
and `work(case)` what a pass cannot do without.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


# --------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # A short prompt of a small layer (8 heads of 64 over 2): the smallest call, latency.
        dict(name="prompt_1x70", kind="prompt", B=1, longest=70, context=0, Hq=8, H=2, D=64, dtype="f16"),
        # One prompt of 1000 tokens through a 4096-wide layer with grouped heads: the demo's own size.
        dict(name="prompt_1x1000", kind="prompt", B=1, longest=1000, context=0, Hq=32, H=8, D=128, dtype="bf16"),
        # Prompts of 12 requests packed into one batch, ragged, one of them empty.
        dict(name="prompt_12x2060", kind="prompt", B=12, longest=2060, context=0, Hq=64, H=8, D=128, dtype="f16"),
        # A chunk of a long prompt: 1000 tokens behind a context of 19011 that was read back from the cache, every head with keys of its own.
        dict(name="prompt_1000_of_20011", kind="prompt", B=1, longest=1000, context=19011, Hq=32, H=32, D=64, dtype="f16"),
        # A long prompt of an 8192-wide layer: the largest product.
        dict(name="prompt_1x8192", kind="prompt", B=1, longest=8192, context=0, Hq=64, H=8, D=128, dtype="bf16"),
        # One decode step of one sequence.
        dict(name="rotate_1", kind="rotate", T=1, Hq=32, H=8, D=128, R=128, norm=True, neighbours=False, first=513, dtype="bf16"),
        # A ragged prompt without norms, neighbouring channels paired, half of each head rotated.
        dict(name="rotate_777", kind="rotate", T=777, Hq=40, H=40, D=64, R=32, norm=False, neighbours=True, first=0, dtype="f16"),
        # A chunk of a very long prompt: the angles of far positions.
        dict(name="rotate_8192", kind="rotate", T=8192, Hq=64, H=8, D=128, R=128, norm=True, neighbours=False, first=1000003, dtype="bf16"),
        # One decode step of one request: the smallest call, latency.
        dict(name="adapt_1x4096x6144", kind="adapt", T=1, K=4096, N=6144, R=16, n=8, requests=1, dtype="bf16"),
        # A decode batch of 64 requests, nearly every one with an adapter of its own: the read of the adapters.
        dict(name="adapt_64x8192x8192", kind="adapt", T=64, K=8192, N=8192, R=16, n=64, requests=64, dtype="bf16"),
        # A ragged prompt of three requests through a layer whose widths are no multiples of anything.
        dict(name="adapt_777x2060x1003", kind="adapt", T=777, K=2060, N=1003, R=8, n=3, requests=3, dtype="f16"),
        # A 4096-token batch of prompts through the 8192 -> 28672 MLP projection: the largest product.
        dict(name="adapt_4096x8192x28672", kind="adapt", T=4096, K=8192, N=28672, R=64, n=4, requests=5, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(("prompt", "prompt", "rotate", "adapt", "adapt"))
    dtype = rng.choice(("bf16", "f16"))
    if kind == "prompt":
        H, G = rng.choice((1, 2, 4, 8, 12)), rng.choice((1, 2, 3, 4, 5, 8))
        case = dict(kind=kind, B=_log(rng, 1, 24), longest=_log(rng, 1, 8192), context=rng.choice((0, 0, _log(rng, 1, 20000))), Hq=H * G, H=H,
                    D=rng.choice((64, 128)), dtype=dtype)
        while work(case)["flops"] > 1.0e12:
            case["longest"], case["context"] = max(1, case["longest"] * 2 // 3), case["context"] * 2 // 3
        return case
    if kind == "rotate":
        H, D = rng.choice((1, 2, 4, 8, 12)), rng.choice((64, 128))
        return dict(kind=kind, T=_log(rng, 1, 8192), Hq=H * rng.choice((1, 2, 3, 5)), H=H, D=D, R=rng.choice((D, D, D // 2, D // 4)),
                    norm=rng.random() < 0.6, neighbours=rng.random() < 0.4, first=rng.choice((0, _log(rng, 1, 2000000))), dtype=dtype)
    T = _log(rng, 1, 4096)
    return dict(kind=kind, T=T, K=_log(rng, 100, 8192), N=_log(rng, 100, 28672), R=rng.choice((8, 16, 32, 64)), n=_log(rng, 1, 64),
                requests=_log(rng, 1, T), dtype=dtype)


def _lens(case):
    """(queries, keys) of each sequence, by the case alone: the longest first, one sequence empty in batches of 4 or more."""
    B, longest = case["B"], case["longest"]
    lens = [max(1, longest * (B - b) // B - 13 * (b % 3)) for b in range(B)]
    lens[0] = longest
    if B >= 4:
        lens[B // 2] = 0
    return [(n, n + case["context"] * (B - b) // B if n else 0) for b, n in enumerate(lens)]


def _requests(case):
    """(tokens, adapter) of each request, by the case alone; an adapter of -1 is none (every ninth request, never the first)."""
    T, R = case["T"], min(case["requests"], case["T"])
    cuts = [T * r // R for r in range(R + 1)]
    return [(cuts[r + 1] - cuts[r], -1 if r % 9 == 8 else (7 * r + 3) % case["n"]) for r in range(R)]


def work(case):
    kind = case["kind"]
    if kind == "prompt":
        lens, Hq, H, D = _lens(case), case["Hq"], case["H"], case["D"]
        pairs = sum(n * (m - n) + n * (n + 1) // 2 for n, m in lens)
        queries, keys = sum(n for n, _ in lens), sum(m for _, m in lens)
        return {"bytes": 4 * D * (queries * Hq + keys * H) + 4 * queries * Hq + 8 * (len(lens) + 1), "flops": 4 * D * Hq * pairs}
    if kind == "rotate":
        T, rows, D = case["T"], case["Hq"] + case["H"], case["D"]
        return {"bytes": 4 * T * rows * D + 8 * T + 4 * case["R"], "flops": T * rows * (3 * case["R"] + (4 * D if case["norm"] else 0))}
    T, K, N, R = case["T"], case["K"], case["N"], case["R"]
    adapted = sum(t for t, a in _requests(case) if a >= 0)
    used = len({a for _, a in _requests(case) if a >= 0})
    return {"bytes": 2 * adapted * K + 4 * T * N + 2 * used * R * (K + N) + 4 * used + 4 * T, "flops": 2 * adapted * R * (K + N)}


# --------------------------------------------------------------------------------------------------- inputs
def _projection(gen, T, heads, D, dtype):
    """Queries, keys and values as a fused projection leaves them: slices of one row per token, a few channels x6."""
    qkv = torch.randn(T, sum(heads), D, device="cuda", generator=gen)
    qkv[:, :, 3::29] *= 6
    return qkv.to(dtype).split(heads, dim=1)


def _starts(lens):
    total, starts = 0, [0]
    for n in lens:
        total += n
        starts.append(total)
    return torch.tensor(starts, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    state = {"case": case, "dtype": dtype}
    if kind == "prompt":
        lens, Hq, H, D = _lens(case), case["Hq"], case["H"], case["D"]
        queries, keys = sum(n for n, _ in lens), sum(m for _, m in lens)
        q, k, v = _projection(gen, queries, (Hq, H, H), D, dtype)
        state["q_starts"] = state["k_starts"] = _starts([n for n, _ in lens])
        if case["context"]:                                             # keys and values read back from the cache
            k, v = (torch.randn(keys, H, D, device="cuda", generator=gen).to(dtype) for _ in range(2))
            state["k_starts"] = _starts([m for _, m in lens])
        # the norms before leave queries and keys of one length per head
        state["q"] = q / q.float().square().mean(-1, keepdim=True).sqrt().to(dtype)
        state["k"], state["v"] = k / k.float().square().mean(-1, keepdim=True).sqrt().to(dtype), v
    elif kind == "rotate":
        state["q"], state["k"], _ = _projection(gen, case["T"], (case["Hq"], case["H"], case["H"]), case["D"], dtype)
        state["positions"] = torch.arange(case["T"], device="cuda") + case["first"]
        state["freq"] = 500000.0 ** (-torch.arange(0, case["R"], 2, dtype=torch.float64, device="cuda") / case["R"])
        for name in ("q_weight", "k_weight"):
            state[name] = torch.exp(0.3 * torch.randn(case["D"], device="cuda", generator=gen)).to(dtype) if case["norm"] else None
    else:
        T, K, N, R, n = (case[x] for x in ("T", "K", "N", "R", "n"))
        x = torch.randn(T, K, device="cuda", generator=gen)
        x[:, torch.randint(0, K, (max(1, K // 512),), device="cuda", generator=gen)] *= 30
        state["x"], state["y"] = x.to(dtype), torch.randn(T, N, device="cuda", generator=gen).to(dtype)
        state["A"] = (torch.randn(n, R, K, device="cuda", generator=gen) / math.sqrt(K)).to(dtype)
        state["B"] = (torch.randn(n, N, R, device="cuda", generator=gen) / math.sqrt(R)).to(dtype)
        state["scale"] = 0.25 + torch.rand(n, device="cuda", generator=gen)
        # which request has which adapter: another rotation of the adapters for another seed
        turn = seed % n
        state["index"] = torch.tensor([(a + turn) % n if a >= 0 else -1 for t, a in _requests(case) for _ in range(t)], dtype=torch.int32, device="cuda")
    return state


# --------------------------------------------------------------------------------------------------- plain forms
def _plain_prompt(s):
    q, k, v, case = s["q"].float(), s["k"].float(), s["v"].float(), s["case"]
    Hq, H, D = case["Hq"], case["H"], case["D"]
    G = Hq // H
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    q0 = k0 = 0
    for n, m in _lens(case):
        keys, values = k[k0:k0 + m].transpose(0, 1), v[k0:k0 + m].transpose(0, 1)                # [H, m, D]
        step = max(1, (1 << 27) // max(1, Hq * m))                                              # rows whose logits fit well
        for i0 in range(0, n, step):
            rows = min(step, n - i0)
            part = q[q0 + i0:q0 + i0 + rows].view(rows, H, G, D).permute(1, 2, 0, 3).reshape(H, G * rows, D)
            logits = ((part @ keys.transpose(1, 2)) / math.sqrt(D)).view(H, G, rows, m)
            last = m - n + i0 + torch.arange(rows, device=q.device)                              # last key that each query sees
            logits = torch.where(torch.arange(m, device=q.device) <= last[:, None], logits, torch.full_like(logits, -math.inf))
            top = logits.amax(dim=-1, keepdim=True)
            p = torch.exp(logits - top)
            total = p.sum(dim=-1, keepdim=True)
            got = (p.view(H, G * rows, m) @ values).view(H, G, rows, D) / total
            out[q0 + i0:q0 + i0 + rows] = got.permute(2, 0, 1, 3).reshape(rows, Hq, D)
            lse[q0 + i0:q0 + i0 + rows] = (top + torch.log(total)).squeeze(-1).permute(2, 0, 1).reshape(rows, Hq)
        q0, k0 = q0 + n, k0 + m
    return out.to(s["dtype"]), lse


def _plain_rotate(s):
    case, outs = s["case"], []
    R = case["R"]
    angle = s["positions"].double()[:, None] * s["freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]              # [T, 1, R / 2]
    for name in ("q", "k"):
        x = s[name].float()
        if case["norm"]:
            x = x / torch.sqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * s[name + "_weight"].float()
        y = x.clone()
        a, b = (slice(0, R, 2), slice(1, R, 2)) if case["neighbours"] else (slice(0, R // 2), slice(R // 2, R))
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., a] * sin + x[..., b] * cos
        outs.append(y.to(s["dtype"]))
    return tuple(outs)


def _plain_adapt(s):
    x, y = s["x"].float(), s["y"].float()
    for a in range(s["case"]["n"]):
        mine = (s["index"] == a)[:, None]
        inner = torch.where(mine, x @ s["A"][a].float().t(), torch.zeros((), device=x.device))
        y = y + (inner @ s["B"][a].float().t()) * s["scale"][a]
    return y.to(s["dtype"])


# --------------------------------------------------------------------------------------------------- the framework's operators
def _run_own(s):
    from paper_2410_07505_b200 import cq
    kind = s["case"]["kind"]
    if kind == "prompt":
        lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=s["q"].device)
        return cq.prompt_attention(s["q"], s["k"], s["v"], s["q_starts"], s["k_starts"], lse=lse), lse
    if kind == "rotate":
        return cq.norm_rotate(s["q"], s["k"], s["positions"], s["freq"], s["q_weight"], s["k_weight"], eps=EPS if s["case"]["norm"] else None,
                              neighbours=s["case"]["neighbours"])
    return cq.adapter_add(s["y"], s["x"], cq.Adapters(s["A"], s["B"], s["scale"]), s["index"])


def run(state):
    if own:
        return _run_own(state)
    return {"prompt": _plain_prompt, "rotate": _plain_rotate, "adapt": _plain_adapt}[state["case"]["kind"]](state)


# --------------------------------------------------------------------------------------------------- in 64 bits
def _exact_prompt(s):
    case = s["case"]
    Hq, H, D = case["Hq"], case["H"], case["D"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    q0 = k0 = 0
    for n, m in _lens(case):
        for h in range(Hq if n else 0):
            k, v = s["k"][k0:k0 + m, h * H // Hq].double(), s["v"][k0:k0 + m, h * H // Hq].double()
            for i0 in range(0, n, 4096):
                rows = slice(q0 + i0, q0 + min(n, i0 + 4096))
                logits = s["q"][rows, h].double() @ k.t() / math.sqrt(D)
                logits += torch.full_like(logits, -math.inf).triu(m - n + i0 + 1)
                lse[rows, h] = torch.logsumexp(logits, dim=-1)
                out[rows, h] = torch.softmax(logits, dim=-1) @ v
        q0, k0 = q0 + n, k0 + m
    return out, lse


def _exact_rotate(s):
    case, outs = s["case"], []
    R = case["R"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["freq"][None])[:, None]
    for name in ("q", "k"):
        x = s[name].double()
        if case["norm"]:
            x = s[name + "_weight"].double() * x * (x.pow(2).sum(-1, keepdim=True) / case["D"] + EPS).rsqrt()
        first, rest = x[..., :R], x[..., R:]
        pairs = first.unflatten(-1, (-1, 2)) if case["neighbours"] else first.unflatten(-1, (2, -1)).transpose(-1, -2)
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        first = pairs.flatten(-2) if case["neighbours"] else pairs.transpose(-1, -2).flatten(-2)
        outs.append(torch.cat((first, rest), dim=-1))
    return tuple(outs)


def _exact_adapt(s):
    out, t0 = s["y"].double(), 0
    index = s["index"].tolist()
    while t0 < len(index):
        t1, a = t0, index[t0]
        while t1 < len(index) and index[t1] == a:
            t1 += 1
        if a >= 0:
            out[t0:t1] += s["scale"][a].double() * ((s["x"][t0:t1].double() @ s["A"][a].double().t()) @ s["B"][a].double().t())
        t0 = t1
    return out


def exact(case, seed):
    return {"prompt": _exact_prompt, "rotate": _exact_rotate, "adapt": _exact_adapt}[case["kind"]](prepare(case, seed))
