"""Timed cases of the operators around the mixer: the linear layer with its
epilogue (feed-forward halves of the blocks, input and output projections),
the token embedding and its gradient, and the AdamW step that consumes the
gradients.

Where ``own`` is false the operators run in their plain form, elementary torch
operations in 32 bits (64 for long sums); where it is true, through the
library's entry points.
"""

from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BETAS = (0.9, 0.999)
EPS = 1e-8
LR = 1e-3
BLOCK = 256        # elements that share a scale in the 8-bit optimiser state
E4M3_MAX = 448.0
SCALE_FLOOR = 1e-30  # a block whose largest value is below this is stored as zeros


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _linear(op, dtype, T, K, N, act, bias=True, residual=False, keep=False, name=None):
    c = dict(op=op, dtype=dtype, T=T, K=K, N=N, act=act, bias=bias, residual=residual, keep=keep)
    if name:
        c["name"] = name
    return c


def _embed(op, dtype, T, V, C, scale, ids, name=None):
    c = dict(op=op, dtype=dtype, T=T, V=V, C=C, scale=scale, ids=ids)
    if name:
        c["name"] = name
    return c


def _adamw(state, blocks, C, extra, low, step, name=None):
    c = dict(op="adamw", state=state, blocks=blocks, C=C, extra=extra, low=low, step=step)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # serving: the feed-forward half's first product for a single token
        _linear("linear", "bf16", 1, 128, 256, "gelu", name="linear one token"),
        # training, long-sequence classification (32 x 4096 tokens): first product of the feed-forward half,
        # the pre-activation kept for the backward
        _linear("linear", "bf16", 131072, 128, 256, "gelu", keep=True, name="linear ffn up lra"),
        # inference, irregular meshes (2 x 50000 points): second product of the feed-forward half with its residual
        _linear("linear", "bf16", 100000, 512, 256, "none", residual=True, name="linear ffn down mesh"),
        # a generic wide layer, bound by the matrix cores
        _linear("linear", "bf16", 8192, 2048, 2048, "silu", name="linear wide"),
        # point coordinates to channels: odd narrow rows in single precision
        _linear("linear", "f32", 50021, 3, 64, "gelu", keep=True, name="linear coordinates f32"),
        # training: backward of the feed-forward half's first product
        _linear("linear_backward", "bf16", 131072, 128, 256, "gelu", keep=True, name="linear backward ffn up lra"),
        # training in single precision on a ragged small cloud
        _linear("linear_backward", "f32", 4099, 64, 128, "silu", keep=True, name="linear backward f32"),
        # symbols of the long sequences to vectors
        _embed("embedding", "bf16", 131072, 256, 128, 1.0, "uniform", name="embedding lra"),
        # gradient of that table from the block's fp32 input gradient, padded batch
        _embed("embedding_backward", "f32", 131072, 256, 128, 1.0, "padded", name="embedding backward lra"),
        # a word vocabulary with skewed counts, scaled rows, bf16 gradients
        _embed("embedding_backward", "bf16", 65536, 32000, 256, 16.0, "zipf", name="embedding backward words"),
        # optimiser step of a small model: latency
        _adamw("f32", 1, 64, 1003, True, 1, name="adamw small"),
        # optimiser step with 8-bit state of wide layers and a word table
        _adamw("q8", 2, 1024, 32000 * 1024 + 7, True, 100, name="adamw 8-bit wide"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, hi):
    w = _log(rng, 1, hi)
    kind = rng.random()
    if kind < 0.6 and w >= 8:  # most widths are multiples of 8 or 32
        w = w // 8 * 8 if kind < 0.3 or w < 32 else w // 32 * 32
    return w


MOST_FLOPS = 2 * 8192 * 2048 * 2048
MOST_BYTES = 400e6


def draw(rng):
    while True:
        op = rng.choice(["linear", "linear", "linear_backward", "linear_backward", "embedding", "embedding_backward",
                         "embedding_backward", "adamw"])
        dt = rng.choice(["bf16", "bf16", "f32"])
        if op.startswith("linear"):
            c = _linear(op, dt, _log(rng, 1, 1 << 19), _width(rng, 2048), _width(rng, 2048),
                        rng.choice(["none", "relu", "gelu", "silu"]), rng.random() < 0.7,
                        op == "linear" and rng.random() < 0.4, rng.random() < 0.5)
            if op == "linear_backward":
                c["keep"] = c["act"] != "none"
        elif op.startswith("embedding"):
            c = _embed(op, dt, _log(rng, 1, 1 << 19), _log(rng, 2, 1 << 17), _width(rng, 1024), rng.choice([1.0, 11.3, 32.0]),
                       rng.choice(["uniform", "zipf", "padded", "one"]))
        else:
            c = _adamw(rng.choice(["f32", "q8"]), rng.randint(1, 2), rng.choice([64, 128, 192, 256, 512, 1024]),
                       _log(rng, 1, 1 << 24), rng.random() < 0.5, _log(rng, 1, 100000))
        w = work(c)
        # single-precision products of the widest layers would cost more than the largest listed case
        if w["flops"] * (10 if c.get("dtype") == "f32" else 1) <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _sizes(c):
    """Element counts of the optimiser's tensors: per block four square weights, the feed-forward pair and the
    vectors; then a table or head of any size."""
    C = c["C"]
    per = [4 * C * C, 4 * C * C, 3 * C]
    return per * c["blocks"] + [c["extra"]]


def _ids(c, g, dev):
    T, V = c["T"], c["V"]
    u = torch.rand(T, generator=g, device=dev)
    if c["ids"] == "one":  # one symbol makes up the whole batch
        return torch.full((T,), V // 2, dtype=torch.int64, device=dev)
    if c["ids"] == "zipf":
        ids = torch.exp(u.double() * math.log(V)).long() - 1
    else:
        ids = (u.double() * V).long()
    ids = ids.clamp_(0, V - 1)
    if c["ids"] == "padded":  # the end of every row of 64 positions is padding
        pos = torch.arange(T, device=dev)
        ids[(pos % 64) >= 40 + (pos // 64) % 24] = -1
    return ids


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 13)
    rn = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    ru = lambda *s: torch.rand(*s, generator=g, device=dev) * 2 - 1  # noqa: E731
    st = {"case": c}
    if c["op"].startswith("linear"):
        dt, T, K, N = DTYPES[c["dtype"]], c["T"], c["K"], c["N"]
        st["X"] = rn(T, K).to(dt)
        st["W"] = (ru(K, N) * math.sqrt(6.0 / (K + N))).to(dt)
        st["bias"] = (rn(N) * 0.1).to(dt) if c["bias"] else None
        if c["op"] == "linear":
            st["residual"] = rn(T, N).to(dt) if c["residual"] else None
        else:
            st["dOut"] = rn(T, N).to(dt)
            st["pre"] = None
            if c["act"] != "none":  # what the forward kept
                y = st["X"].float() @ st["W"].float()
                st["pre"] = (y if st["bias"] is None else y + st["bias"].float()).to(dt)
    elif c["op"].startswith("embedding"):
        dt = DTYPES[c["dtype"]]
        st["ids"] = _ids(c, g, dev)
        if c["op"] == "embedding":
            st["table"] = rn(c["V"], c["C"]).to(dt)
        else:
            st["dOut"] = rn(c["T"], c["C"]).to(dt)
    else:
        st["tensors"] = []
        for k, n in enumerate(_sizes(c)):
            t = {"p": ru(n) * 0.05, "g": rn(n) * 1e-3, "weight_decay": 0.0 if k % 3 == 2 else 0.01}
            m, r = rn(n) * 3e-4, rn(n).abs() * 1e-3 + 1e-5  # first moment, root of the second
            if c["state"] == "f32":
                t["m"], t["v"] = m, r * r
            else:
                for key, x in (("m", m), ("v", r)):
                    scale = _blocks(x).abs().amax(1) / E4M3_MAX
                    t[key] = (_blocks(x) / scale[:, None]).reshape(-1)[:n].to(torch.float8_e4m3fn)
                    t[key + "_scale"] = scale
            t["p_low"] = torch.empty(n, dtype=torch.bfloat16, device=dev) if c["low"] else None
            st["tensors"].append(t)
        if own:  # the handle that a program keeps beside its parameters
            from paper_2608_11519_amd import flarepp as fp
            st["plan"] = fp.flarepp_adamw_plan(st["tensors"])
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------

def _act(y, act):
    if act == "relu":
        return torch.where(y < 0, torch.zeros_like(y), y)
    if act == "gelu":
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    if act == "silu":
        return y / (1 + torch.exp(-y))
    return y


def _slope(y, act):
    if act == "relu":
        return (y > 0).to(y.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(y * math.sqrt(0.5))) + y * torch.exp(-0.5 * y * y) / math.sqrt(2 * math.pi)
    s = 1 / (1 + torch.exp(-y))
    return s * (1 + y * (1 - s))


def _plain_linear(st):
    c, dt = st["case"], st["X"].dtype
    y = st["X"].float() @ st["W"].float()
    if st["bias"] is not None:
        y = y + st["bias"].float()
    out = _act(y, c["act"])
    if st["residual"] is not None:
        out = st["residual"].float() + out
    return {"out": out.to(dt), "pre": y.to(dt)} if c["keep"] else {"out": out.to(dt)}


def _plain_linear_backward(st):
    c, dt = st["case"], st["X"].dtype
    d = st["dOut"].float()
    if c["act"] != "none":
        d = d * _slope(st["pre"].float(), c["act"])
    r = {"dX": (d @ st["W"].float().t()).to(dt), "dW": st["X"].float().t() @ d}
    if c["bias"]:
        r["dbias"] = d.sum(0, dtype=torch.float64).float()
    return r


def _plain_embedding(st):
    c, ids = st["case"], st["ids"]
    rows = st["table"].float()[ids.clamp(min=0)] * c["scale"]
    return {"out": torch.where((ids >= 0)[:, None], rows, torch.zeros_like(rows)).to(st["table"].dtype)}


def _plain_embedding_backward(st):
    # sums over the runs of the sorted symbols, as differences of running sums
    c = st["case"]
    V, dev = c["V"], st["ids"].device
    ids, order = torch.sort(torch.where(st["ids"] < 0, V, st["ids"]))
    total = torch.zeros(c["T"] + 1, c["C"], dtype=torch.float64, device=dev)
    torch.cumsum(st["dOut"][order].double(), 0, out=total[1:])
    ends = torch.searchsorted(ids, torch.arange(V + 1, device=dev))
    return {"dTable": ((total[ends[1:]] - total[ends[:-1]]) * c["scale"]).float()}


def _blocks(x):
    n = x.numel()
    return torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)


def _noise(n, step, dev):
    """16 + 16 random bits of every element of a step: a hash of the step and the element's index."""
    i = torch.arange(n, dtype=torch.int64, device=dev)
    lo32 = 0xFFFFFFFF
    h = ((i & lo32) * 0x9E3779B1 + (i >> 32) * 0x6A09E667 + step * 0xBB67AE85) & lo32
    h = h ^ (h >> 16)
    h = (h * 0x6A09E667) & lo32
    h = h ^ (h >> 15)
    h = (h * 0xBB67AE85) & lo32
    h = h ^ (h >> 16)
    return h & 0xFFFF, h >> 16


def _to_e4m3(x, u, at_least_one):
    """x as e4m3 times a scale per block, rounded up or down at random: up with the probability of the part cut off."""
    n = x.numel()
    b = _blocks(x)
    big = b.abs().amax(1)
    zero = big < SCALE_FLOOR
    scale = torch.where(zero, torch.zeros_like(big), big * (1 / E4M3_MAX))
    inv = torch.where(zero, torch.zeros_like(big), torch.reciprocal(scale))
    y = (b * inv[:, None]).reshape(-1)[:n]
    a = torch.clamp(y.abs(), max=E4M3_MAX)
    normal = ((a.view(torch.int32) + (u.to(torch.int32) << 4)) & ~0xFFFFF).view(torch.float32)
    fixed = torch.floor(a * 512.0 + u.float() * (1.0 / 65536)) * (1.0 / 512)
    q = torch.where(a < 1.0 / 64, fixed, normal)
    if at_least_one:
        q = torch.where(y > 0, torch.clamp(q, min=1.0 / 512), q)
    return torch.where(y < 0, -q, q).to(torch.float8_e4m3fn), scale


def _plain_adamw(st):
    c, outs = st["case"], []
    t = c["step"]
    f32 = lambda x: torch.tensor(x, dtype=torch.float32).item()  # noqa: E731
    size, root = f32(LR / (1 - BETAS[0] ** t)), f32(1 / math.sqrt(1 - BETAS[1] ** t))
    b1, a1, b2, a2 = f32(BETAS[0]), f32(1 - BETAS[0]), f32(BETAS[1]), f32(1 - BETAS[1])
    for x in st["tensors"]:
        p, g, n = x["p"], x["g"], x["p"].numel()
        keep = f32(1 - LR * x["weight_decay"])
        if c["state"] == "f32":
            m, v = x["m"], x["v"]
        else:
            m = (_blocks(x["m"].float()) * x["m_scale"][:, None]).reshape(-1)[:n]
            r = (_blocks(x["v"].float()) * x["v_scale"][:, None]).reshape(-1)[:n]
            v = r * r
        m = m * b1 + g * a1
        v = v * b2 + (g * g) * a2
        r = torch.sqrt(v)
        p.copy_(p * keep - (m / (r * root + EPS)) * size)
        o = {"p": p}
        if c["state"] == "f32":
            o["m"], o["v"] = x["m"].copy_(m), x["v"].copy_(v)
        else:
            um, uv = _noise(n, t, p.device)
            for key, y, u in (("m", m, um), ("v", r, uv)):
                q, scale = _to_e4m3(y, u, key == "v")
                o[key], o[key + "_scale"] = x[key].copy_(q), x[key + "_scale"].copy_(scale)
        if x["p_low"] is not None:
            o["p_low"] = x["p_low"].copy_(p)
        outs.append(o)
    return outs


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    st, c = state, state["case"]
    if not own:
        return {"linear": _plain_linear, "linear_backward": _plain_linear_backward, "embedding": _plain_embedding,
                "embedding_backward": _plain_embedding_backward, "adamw": _plain_adamw}[c["op"]](st)
    from paper_2608_11519_amd import flarepp as fp
    if c["op"].startswith("linear"):
        act = {"none": fp.ACT_NONE, "relu": fp.ACT_RELU, "gelu": fp.ACT_GELU, "silu": fp.ACT_SILU}[c["act"]]
        if c["op"] == "linear":
            r = fp.flarepp_linear_forward(st["X"], st["W"], st["bias"], act=act, residual=st["residual"], keep_pre=c["keep"])
            return {"out": r[0], "pre": r[1]} if c["keep"] else {"out": r}
        return fp.flarepp_linear_backward(st["X"], st["W"], st["dOut"], pre=st["pre"], act=act, want_dbias=c["bias"])
    if c["op"] == "embedding":
        return {"out": fp.flarepp_embedding_forward(st["ids"], st["table"], scale=c["scale"])}
    if c["op"] == "embedding_backward":
        return {"dTable": fp.flarepp_embedding_backward(st["ids"], st["dOut"], V=c["V"], scale=c["scale"])}
    fp.flarepp_adamw_step(st["plan"], lr=LR, step=c["step"], betas=BETAS, eps=EPS)
    return [{k: x[k] for k in ("p", "m", "m_scale", "v", "v_scale", "p_low") if x.get(k) is not None} for x in st["tensors"]]


def work(case):
    c = case
    if c["op"].startswith("linear"):
        b, T, K, N = 4 if c["dtype"] == "f32" else 2, c["T"], c["K"], c["N"]
        if c["op"] == "linear":
            outs = 1 + c["residual"] + c["keep"]
            return {"bytes": b * (T * K + K * N + outs * T * N + c["bias"] * N), "flops": 2 * T * K * N}
        ins = 2 if c["act"] != "none" else 1
        return {"bytes": b * (2 * T * K + K * N + ins * T * N) + 4 * (K * N + c["bias"] * N), "flops": 4 * T * K * N}
    if c["op"].startswith("embedding"):
        b, T, V, C = 4 if c["dtype"] == "f32" else 2, c["T"], c["V"], c["C"]
        if c["op"] == "embedding":
            return {"bytes": 8 * T + b * C * (T + min(V, T)), "flops": T * C}
        return {"bytes": 8 * T + b * T * C + 4 * V * C, "flops": T * C}
    n = sum(_sizes(c))
    per = 28 if c["state"] == "f32" else 16 + 16 / BLOCK
    return {"bytes": int(n * (per + 2 * c["low"])), "flops": 16 * n}


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    c = case
    st = prepare(case, seed)
    if c["op"].startswith("linear"):
        X, W, f = st["X"].double(), st["W"].double(), c["act"]
        if c["op"] == "linear":
            y = torch.mm(X, W)
            if st["bias"] is not None:
                y += st["bias"].double()
            a = {"none": lambda: y, "relu": lambda: y.clamp(min=0), "gelu": lambda: y * torch.special.ndtr(y),
                 "silu": lambda: y * torch.special.expit(y)}[f]()
            if st["residual"] is not None:
                a = a + st["residual"].double()
            return {"out": a, "pre": y} if c["keep"] else {"out": a}
        d = st["dOut"].double()
        if f == "relu":
            d = d.masked_fill(st["pre"] <= 0, 0.0)
        elif f != "none":
            y = st["pre"].double()
            if f == "gelu":
                d *= torch.special.ndtr(y) + y * torch.exp(-y * y / 2) * 0.3989422804014327
            else:
                s = torch.special.expit(y)
                d *= s + y * s * torch.special.expit(-y)
        r = {"dX": torch.mm(d, W.t()), "dW": torch.mm(X.t(), d)}
        if c["bias"]:
            r["dbias"] = torch.mv(d.t(), torch.ones(c["T"], dtype=torch.float64, device=d.device))
        return r
    if c["op"] == "embedding":
        E = torch.cat([st["table"].double() * c["scale"], torch.zeros(1, c["C"], dtype=torch.float64, device="cuda")])
        return {"out": E.index_select(0, torch.where(st["ids"] < 0, c["V"], st["ids"]))}
    if c["op"] == "embedding_backward":
        E = torch.zeros(c["V"] + 1, c["C"], dtype=torch.float64, device="cuda")  # the last row takes the padding
        E.index_add_(0, torch.where(st["ids"] < 0, c["V"], st["ids"]), st["dOut"].double())
        return {"dTable": c["scale"] * E[:-1]}
    outs, t = [], c["step"]
    for x in st["tensors"]:
        g, q8 = x["g"].double(), c["state"] == "q8"
        m, v = x["m"].double(), x["v"].double()
        if q8:
            n = g.numel()
            m *= x["m_scale"].double().repeat_interleave(BLOCK)[:n]
            v = (v * x["v_scale"].double().repeat_interleave(BLOCK)[:n]) ** 2
        m = BETAS[0] * m + (1 - BETAS[0]) * g
        v = BETAS[1] * v + (1 - BETAS[1]) * g ** 2
        p = x["p"].double() * (1 - LR * x["weight_decay"])
        p -= LR * (m / (1 - BETAS[0] ** t)) / ((v / (1 - BETAS[1] ** t)).sqrt() + EPS)
        o = {"p": p, "m": m, "v": v}
        if q8:  # which of two codes a moment takes depends on its last bits: no value in 64 bits
            o = {"p": p, "m": None, "v": None}
            for key, y in (("m_scale", m), ("v_scale", v.sqrt())):
                pad = torch.cat([y, y.new_zeros(-n % BLOCK)])
                o[key] = pad.reshape(-1, BLOCK).abs().max(dim=1).values / E4M3_MAX
        if x["p_low"] is not None:
            o["p_low"] = p
        outs.append(o)
    return outs
