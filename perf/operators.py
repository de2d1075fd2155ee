"""Performance cases of the operators around a token transformer's layers:
activation checkpoints in 8 bits with the linear backward that reads them,
rotary positions with several axes, and per-token log probabilities with
entropy, top alternatives and their gradient.

``listed()`` names the cases, ``draw(rng)`` gives another of the same ranges,
``prepare`` makes the inputs, ``run`` is one pass (``own`` false: elementary
torch operations in 32 bits; true: the calls of
``paper_2507_03312_amd.binding``), ``work`` the bytes and operations it cannot
do without, ``exact`` the same results in 64 bits, written apart.
"""
from __future__ import annotations

import math

import torch

own = False

HALF = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
DT = {"f32": 0, "f16": 1, "bf16": 2}  # the library's type codes
GROUP = 32                            # rows of a column that share a checkpoint's scale
# exponents of a checkpoint's scales: at the largest one a code of 256 would be
# infinite in the half type and is held as 240
EXPONENTS = {"f16": (-15, 8), "bf16": (-117, 120)}
LOSS_SCALE = 2.0 ** 12


def listed():
    return [
        # the hidden layer of a small two-layer MLP step: one launch's latency
        {"name": "pack_mlp", "kind": "pack", "half": "f16", "m": 64, "k": 1024},
        # the inputs of a 768-wide block's projections: 64 images of 197 tokens
        {"name": "pack_tokens", "kind": "pack", "half": "bf16", "m": 12608, "k": 768},
        # the small MLP's second layer, backward through GELU'
        {"name": "linear8_mlp", "kind": "linear8", "half": "f16", "m": 64, "n": 512, "k": 1024,
         "gelu": True},
        # the QKV projection of that 768-wide block
        {"name": "linear8_qkv", "kind": "linear8", "half": "bf16", "m": 12608, "n": 2304, "k": 768,
         "gelu": False},
        # the down projection of a 384-wide block on 256 small images: the packed
        # hidden activations and, for GELU', the packed pre-activations
        {"name": "linear8_down", "kind": "linear8", "half": "f16", "m": 16640, "n": 384, "k": 1536,
         "gelu": True},
        # a patch embedding of 14 x 14 x 3 patches: ragged rows, rows of 588
        {"name": "linear8_odd", "kind": "linear8", "half": "bf16", "m": 8415, "n": 768, "k": 588,
         "gelu": False},
        # single tokens of 16 sequences, grouped heads, time x height x width
        {"name": "rope_tokens", "kind": "rope", "half": "bf16", "rows": 16, "grid": 16, "rot": 40,
         "copy": 8, "hd": 128, "pairs": "16,24,24", "interleaved": False, "back": False,
         "far": 1000000},
        # the benchmark's block: 64 images of 197 tokens, 12 heads, height x width
        {"name": "rope_image", "kind": "rope", "half": "bf16", "rows": 12608, "grid": 197, "rot": 24,
         "copy": 12, "hd": 64, "pairs": "16,16", "interleaved": False, "back": False, "far": 14},
        # the cotangents of a batch of video clips, interleaved pairs, grouped heads
        {"name": "rope_video", "kind": "rope", "half": "f16", "rows": 29997, "grid": 29997, "rot": 40,
         "copy": 8, "hd": 128, "pairs": "16,24,24", "interleaved": True, "back": True, "far": 256},
        # a few answers scored against a large vocabulary, no gradient
        {"name": "logprob_few", "kind": "logprob", "half": "bf16", "rows": 8, "v": 131072, "k": 8,
         "train": False},
        # a 1000-class head's rows, with the gradient
        {"name": "logprob_classes", "kind": "logprob", "half": "f16", "rows": 256, "v": 1000, "k": 5,
         "train": True},
        # a training batch's tokens over an odd vocabulary, with the gradient
        {"name": "logprob_train", "kind": "logprob", "half": "bf16", "rows": 4096, "v": 65537, "k": 4,
         "train": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["pack", "linear8", "linear8", "rope", "rope", "logprob", "logprob"])
    half = rng.choice(["f16", "bf16"])
    if kind in ("pack", "linear8"):
        m = _log(rng, 33, 16640)
        if rng.random() < 0.35:  # any widths, as a head or an odd patch size has
            n, k = _log(rng, 40, 2304), _log(rng, 40, 2304)
        else:
            n, k = 64 * _log(rng, 2, 36), 64 * _log(rng, 2, 36)
        if kind == "pack":
            return {"kind": "pack", "half": half, "m": m, "k": k}
        while m * n * k > 12608 * 2304 * 768:
            m = m * 2 // 3 + 1
        return {"kind": "linear8", "half": half, "m": m, "n": n, "k": k, "gelu": rng.random() < 0.5}
    if kind == "rope":
        axes = rng.randint(1, 4)
        hd = rng.choice([32, 64, 64, 80, 96, 128, 128, 256])
        unit = rng.choice([1, 2, 4, 8])
        left = hd // 2 // unit
        pairs = []
        for a in range(axes):
            most = left - (axes - 1 - a)
            pairs.append(rng.randint(1, max(1, most)) if a + 1 < axes else most)
            left -= pairs[-1]
        rot, copy = rng.randint(1, 48), rng.choice([0, 1, 8, 12])
        grid = _log(rng, 1, 4096)
        rows = grid * _log(rng, 1, max(1, 100_000_000 // (grid * (rot + copy) * hd)))
        return {"kind": "rope", "half": rng.choice([half, half, "f32"]), "rows": rows, "grid": grid,
                "rot": rot, "copy": copy, "hd": hd, "pairs": ",".join(str(unit * p) for p in pairs),
                "interleaved": rng.random() < 0.5, "back": rng.random() < 0.5,
                "far": _log(rng, 2, 2_000_000)}
    v = _log(rng, 10, 262144)
    k = rng.randint(0, min(16, v))
    rows = _log(rng, 1, max(2, min(16384, 2_500_000_000 // (v * (6 + k)))))
    return {"kind": "logprob", "half": rng.choice([half, half, "f32"]), "rows": rows, "v": v, "k": k,
            "train": rng.random() < 0.6}


# ------------------------------------------------------------------ inputs --

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g)


def _uniform(g, shape):
    return torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(generator=g)


def _activations(g, m, k, dtype):
    """Layer inputs as a normalised residual stream has them: unit variance, a
    few columns far larger."""
    wide = torch.where(_uniform(g, (1, k)) < 0.01, 30.0, 1.0)
    return (_normal(g, (m, k)) * wide).to(dtype)


def prepare(case, seed):
    g, c, t = _gen(seed), dict(case), HALF[case["half"]]
    s = {"case": c}
    if c["kind"] == "pack":
        s["x"] = _activations(g, c["m"], c["k"], t)
    elif c["kind"] == "linear8":
        m, n, k = c["m"], c["n"], c["k"]
        pre = _activations(g, m, k, t)
        x = torch.nn.functional.gelu(pre.float(), approximate="tanh").to(t) if c["gelu"] else pre
        # the checkpoints that the forward pass left
        s["xc"], s["xs"] = _pack(x, c["half"])
        if c["gelu"]:
            s["pc"], s["ps"] = _pack(pre, c["half"])
        s["w"] = _normal(g, (n, k), 0.02).to(t)
        s["dy"] = (_normal(g, (m, n), 1e-4) * LOSS_SCALE).to(t)
    elif c["kind"] == "rope":
        width = (c["rot"] + c["copy"]) * c["hd"]
        s["x"] = _normal(g, (c["rows"], width)).to(t)
        axes = len(c["pairs"].split(","))
        s["pos"] = torch.floor(_uniform(g, (c["grid"], axes)) * c["far"])
    else:
        rows, v, k = c["rows"], c["v"], c["k"]
        # rows of a logits buffer whose stride is a whole number of 16-byte vectors
        z = torch.zeros(rows, -(-v // 8) * 8, dtype=t, device="cuda")
        z[:, :v] = _normal(g, (rows, v), 2.5)
        s["z"] = z[:, :v]
        s["target"] = (_uniform(g, (rows,)) * v).long().clamp_(max=v - 1).int()
        if c["train"]:
            s["g_logp"] = -(0.5 + _uniform(g, (rows,))) / rows
            s["g_entropy"] = _normal(g, (rows,), 0.01) / rows
            s["g_top"] = _normal(g, (rows, k), 0.1) / rows
            # scale, counter, period, factor, least and largest scale
            s["state"] = torch.tensor([LOSS_SCALE, 0.0, 0.0, 2.0, 1.0, 2.0 ** 100], device="cuda")
    return s


# ------------------------------------------------------------- plain forms --

def _exponents(a):
    """floor(log2(a)) of positive float32 values."""
    return torch.frexp(a)[1] - 1


def _pack(x, half):
    """Codes (e4m3 bytes) and scale exponents (biased by 127) of a half matrix."""
    lo, hi = EXPONENTS[half]
    m, k = x.shape
    groups = -(-m // GROUP)
    f = x.float()
    fin = torch.isfinite(f)
    a = torch.where(fin, f, 0.0).abs()
    padded = torch.zeros(groups * GROUP, k, device=x.device)
    padded[:m] = a
    amax = padded.view(groups, GROUP, k).amax(1)
    p = _exponents(torch.where(amax > 0, amax, 2.0 ** -126))
    p = torch.where(amax > 0, p, -126)
    e = p - 8 + (amax > torch.ldexp(torch.full_like(amax, 1.75), p)).int()
    e = e.clamp(lo, hi)
    row_e = e.repeat_interleave(GROUP, 0)[:m]
    y = torch.ldexp(torch.ldexp(f, -(row_e // 2)), -(row_e - row_e // 2))
    y = torch.where(fin, y, float("nan"))
    codes = y.to(torch.float8_e4m3fn)
    top = (row_e == hi) & (codes.float().abs() == 256.0)
    codes = torch.where(top, torch.copysign(torch.full_like(y, 240.0), y), codes.float())
    return codes.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _widen(codes, scales):
    e = scales.int() - 127
    row_e = e.repeat_interleave(GROUP, 0)[:codes.shape[0]]
    return torch.ldexp(torch.ldexp(codes.float(), row_e // 2), row_e - row_e // 2)


def _gelu_grad(x):
    c, a = math.sqrt(2.0 / math.pi), 0.044715
    s = torch.sigmoid(2.0 * c * (x + a * x * x * x))
    return s + x * s * (1.0 - s) * 2.0 * c * (1.0 + 3.0 * a * x * x)


def _pairs(c):
    return [int(p) for p in c["pairs"].split(",")]


def _columns(c, device):
    """The first and second dimension of every pair within a head."""
    first, second, o = [], [], 0
    for n in _pairs(c):
        i = torch.arange(n, device=device)
        first.append(o + (2 * i if c["interleaved"] else i))
        second.append(o + (2 * i + 1 if c["interleaved"] else n + i))
        o += 2 * n
    return torch.cat(first), torch.cat(second)


def _angles(c, pos):
    return torch.cat([pos[:, a:a + 1].double() * 10000.0 ** (-torch.arange(
        n, device=pos.device, dtype=torch.float64) / n) for a, n in enumerate(_pairs(c))], 1)


def _rope(c, x, pos):
    rows, hd = c["rows"], c["hd"]
    angle = _angles(c, pos).repeat(rows // c["grid"], 1)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if c["back"]:
        sin = -sin
    f, s = _columns(c, x.device)
    h = x.view(rows, -1, hd)[:, :c["rot"]].float()
    y = h.clone()
    y[..., f] = h[..., f] * cos - h[..., s] * sin
    y[..., s] = h[..., s] * cos + h[..., f] * sin
    return torch.cat([y.to(x.dtype).reshape(rows, -1), x[:, c["rot"] * hd:]], 1)


def _logprob(c, s):
    z = s["z"].float()
    rows, v, k = c["rows"], c["v"], c["k"]
    m = z.amax(1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    ln = torch.log(total)
    out = {"stats": torch.cat([m, ln], 1),
           "logp": (z.gather(1, s["target"].long()[:, None]) - m - ln)[:, 0],
           "entropy": (ln - (e * d).sum(1, keepdim=True) / total)[:, 0]}
    if k:
        left, at = z.clone(), torch.arange(v, device=z.device)
        top, index = [], []
        for _ in range(k):
            best = left.amax(1, keepdim=True)
            i = torch.where(left == best, at, v).amin(1, keepdim=True)
            left.scatter_(1, i, float("-inf"))
            top.append(best - m - ln)
            index.append(i)
        out["top_logp"], out["top_index"] = torch.cat(top, 1), torch.cat(index, 1).int()
    if c["train"]:
        lp = d - ln
        p = torch.exp(lp)
        g = s["g_logp"][:, None]
        grad = -p * (g + s["g_top"].sum(1, keepdim=True))
        grad -= s["g_entropy"][:, None] * p * (lp + out["entropy"][:, None])
        grad.scatter_add_(1, s["target"].long()[:, None], g)
        if k:
            grad.scatter_add_(1, out["top_index"].long(), s["g_top"])
        out["dz"] = (grad * s["state"][0]).to(s["z"].dtype)
    return out


def _plain(s):
    c = s["case"]
    if c["kind"] == "pack":
        codes, scales = _pack(s["x"], c["half"])
        return {"codes": codes, "scales": scales}
    if c["kind"] == "linear8":
        dy, w = s["dy"].float(), s["w"].float()
        dx = dy @ w
        if c["gelu"]:
            dx *= _gelu_grad(_widen(s["pc"], s["ps"]))
        t = s["w"].dtype
        return {"dx": dx.to(t), "dw": (dy.t() @ _widen(s["xc"], s["xs"])).to(t),
                "db": dy.sum(0).to(t)}
    if c["kind"] == "rope":
        return {"y": _rope(c, s["x"], s["pos"])}
    return _logprob(c, s)


# --------------------------------------------------- the framework's calls --

def _buffers(s, make):
    """The pass's outputs and workspace, made at the state's first pass as a
    training program makes its own at set-up."""
    if "buffers" not in s:
        s["buffers"] = make()
    return s["buffers"]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _calls(s):
    from paper_2507_03312_amd import binding as mx

    c, dt = s["case"], DT[s["case"]["half"]]
    stream = torch.cuda.current_stream().cuda_stream
    if c["kind"] == "pack":
        x = s["x"]
        m, k = x.shape
        codes, scales = _buffers(s, lambda: (
            torch.empty(m, k, dtype=torch.uint8, device="cuda"),
            torch.empty(-(-m // GROUP), k, dtype=torch.uint8, device="cuda")))
        mx.mpx_act8_pack(x.data_ptr(), k, codes.data_ptr(), scales.data_ptr(), m, k, dt, stream)
        return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales}
    if c["kind"] == "linear8":
        m, n, k, t = c["m"], c["n"], c["k"], s["w"].dtype
        dx, dw, db, ws = _buffers(s, lambda: (
            torch.empty(m, k, dtype=t, device="cuda"), torch.empty(n, k, dtype=t, device="cuda"),
            torch.empty(n, dtype=t, device="cuda"),
            torch.empty(mx.mpx_linear_bwd_act8_workspace(m, n, k), dtype=torch.uint8,
                        device="cuda")))
        mx.mpx_linear_bwd_act8(s["xc"].data_ptr(), s["xs"].data_ptr(), s["w"].data_ptr(),
                               s["dy"].data_ptr(), _ptr(s.get("pc")), _ptr(s.get("ps")),
                               mx.MPX_ACT_GELU_TANH if c["gelu"] else mx.MPX_ACT_NONE, dx.data_ptr(),
                               dw.data_ptr(), db.data_ptr(), m, n, k, dt, ws.data_ptr(), ws.numel(),
                               None, stream)
        return {"dx": dx, "dw": dw, "db": db}
    if c["kind"] == "rope":
        x = s["x"]
        y, plan = _buffers(s, lambda: (torch.empty_like(x), mx.RopePlan(
            _pairs(c), interleaved=c["interleaved"])))
        call = mx.mpx_rope_bwd if c["back"] else mx.mpx_rope_fwd
        call(x.data_ptr(), x.shape[1], y.data_ptr(), x.shape[1], s["pos"].data_ptr(), c["grid"],
             c["rows"], c["rot"], c["copy"], c["hd"], plan, dt, stream)
        return {"y": y}
    z, rows, v, k = s["z"], c["rows"], c["v"], c["k"]
    ld = z.stride(0)
    f, dz, index, ws = _buffers(s, lambda: (
        torch.empty(4 * rows + rows * k, device="cuda"),
        torch.empty(rows, ld, dtype=z.dtype, device="cuda") if c["train"] else None,
        torch.empty(rows, k, dtype=torch.int32, device="cuda"),
        torch.empty(mx.mpx_logprob_workspace(rows, v, k), dtype=torch.uint8, device="cuda")))
    logp, entropy, stats, top = f[:rows], f[rows:2 * rows], f[2 * rows:4 * rows], f[4 * rows:]
    mx.mpx_logprob_fwd(z.data_ptr(), ld, s["target"].data_ptr(), rows, v, k, logp.data_ptr(),
                       entropy.data_ptr(), stats.data_ptr(), top.data_ptr() if k else None,
                       index.data_ptr() if k else None, dt, ws.data_ptr(), ws.numel(), stream)
    out = {"stats": stats.view(rows, 2), "logp": logp, "entropy": entropy}
    if k:
        out["top_logp"], out["top_index"] = top.view(rows, k), index
    if c["train"]:
        mx.mpx_logprob_bwd(z.data_ptr(), ld, s["target"].data_ptr(), rows, v, k, stats.data_ptr(),
                           entropy.data_ptr(), index.data_ptr() if k else None,
                           s["g_logp"].data_ptr(), s["g_entropy"].data_ptr(),
                           s["g_top"].data_ptr() if k else None, s["state"].data_ptr(),
                           dz.data_ptr(), ld, dt, stream)
        out["dz"] = dz[:, :v]
    return out


def run(state):
    return _calls(state) if own else _plain(state)


# -------------------------------------------------------------------- work --

def work(case):
    c = case
    b = 4 if c["half"] == "f32" else 2
    if c["kind"] == "pack":
        m, k = c["m"], c["k"]
        return {"bytes": b * m * k + m * k + -(-m // GROUP) * k, "flops": 4 * m * k}
    if c["kind"] == "linear8":
        m, n, k = c["m"], c["n"], c["k"]
        packed = (m * k + -(-m // GROUP) * k) * (2 if c["gelu"] else 1)
        return {"bytes": packed + b * (m * n + 2 * n * k + n + m * k), "flops": 4 * m * n * k + m * n}
    if c["kind"] == "rope":
        width = (c["rot"] + c["copy"]) * c["hd"]
        return {"bytes": 2 * b * c["rows"] * width + 4 * c["grid"] * len(_pairs(c)),
                "flops": 3 * c["rows"] * c["rot"] * c["hd"]}
    rows, v, k = c["rows"], c["v"], c["k"]
    passes = 3 if c["train"] else 1  # the gradient reads the logits again and writes as much
    return {"bytes": passes * b * rows * v + rows * (20 + 8 * k), "flops": (14 if c["train"] else 6) * rows * v}


# ------------------------------------------------------------ in 64 bits --

def _exact_pack(x, half):
    lo, hi = EXPONENTS[half]
    m, k = x.shape
    values, exponents = torch.empty(m, k, dtype=torch.float64, device=x.device), []
    for r in range(0, m, GROUP):
        block = x[r:r + GROUP].double()
        a = torch.where(torch.isfinite(block), block.abs(), 0.0).amax(0)
        # the least power of two that brings the largest magnitude to 448 or less
        e = torch.ceil(torch.log2(torch.clamp(a, min=2.0 ** -200) / 448.0))
        e = torch.where(a > 448.0 * torch.exp2(e), e + 1, e)
        e = torch.where(a <= 448.0 * torch.exp2(e - 1), e - 1, e).clamp(lo, hi)
        y = block / torch.exp2(e)
        step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(y.abs(), min=2.0 ** -20))),
                                      min=-6.0) - 3.0)
        q = torch.round(y / step) * step
        values[r:r + GROUP] = torch.where((e == hi) & (q.abs() > 240.0), torch.sign(q) * 240.0, q)
        exponents.append(e)
    return values, torch.stack(exponents)


def _exact_values(codes, scales):
    rows = torch.arange(codes.shape[0], device=codes.device) // GROUP
    return codes.float().double() * torch.exp2(scales.double() - 127.0)[rows]


def _exact_rope(c, x, pos):
    rows, hd = c["rows"], c["hd"]
    sign = -1.0 if c["back"] else 1.0
    h = x.double().view(rows, c["rot"] + c["copy"], hd)
    out, o = h.clone(), 0
    at = torch.arange(rows, device=x.device) % c["grid"]
    for a, n in enumerate(_pairs(c)):
        for i in range(n):
            j, k = (o + 2 * i, o + 2 * i + 1) if c["interleaved"] else (o + i, o + n + i)
            turn = sign * pos[at, a].double() * math.exp(-math.log(10000.0) * i / n)
            w = torch.polar(torch.ones_like(turn), turn)[:, None]
            z = torch.complex(h[:, :c["rot"], j], h[:, :c["rot"], k]) * w
            out[:, :c["rot"], j], out[:, :c["rot"], k] = z.real, z.imag
        o += 2 * n
    return out.view(rows, -1)


def _exact_logprob(c, s):
    rows, k = c["rows"], c["k"]
    keys = ["entropy", "logp", "stats"] + (["top_logp"] if k else []) + (["dz"] if c["train"] else [])
    parts = {key: [] for key in keys}
    for r in range(0, rows, 256):
        z = s["z"][r:r + 256].double()
        lp = torch.log_softmax(z, 1)
        p, t = lp.exp(), s["target"][r:r + 256].long()
        at = torch.arange(z.shape[0], device=z.device)
        h = -torch.xlogy(p, p).sum(1)
        big = z.max(dim=1).values
        parts["stats"].append(torch.stack([big, torch.log(torch.exp(z - big[:, None]).sum(1))], 1))
        parts["logp"].append(lp[at, t])
        parts["entropy"].append(h)
        if k:
            order = torch.sort(z, dim=1, descending=True, stable=True)[1][:, :k]
            parts["top_logp"].append(lp.gather(1, order))
        if c["train"]:
            gl, ge = s["g_logp"][r:r + 256].double(), s["g_entropy"][r:r + 256].double()
            up = torch.zeros_like(lp)  # the cotangent of every log probability
            up[at, t] += gl
            if k:
                for i in range(k):
                    up[at, order[:, i]] += s["g_top"][r:r + 256, i].double()
            d = up - p * up.sum(1, keepdim=True) - ge[:, None] * p * (lp + h[:, None])
            parts["dz"].append(d * LOSS_SCALE)
    out = {key: torch.cat(v) for key, v in parts.items()}
    if k:
        out["top_index"] = None
    return out


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["kind"] == "pack":
        return {"codes": _exact_pack(s["x"], c["half"])[0], "scales": None}
    if c["kind"] == "linear8":
        dy = s["dy"].double()
        dx = dy @ s["w"].double()
        if c["gelu"]:
            x = _exact_values(s["pc"], s["ps"])
            u = math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)
            dx = dx * (0.5 * (1.0 + torch.tanh(u)) + 0.5 * x / torch.cosh(u.clamp(-300, 300)) ** 2
                       * math.sqrt(2.0 / math.pi) * (1.0 + 3.0 * 0.044715 * x ** 2))
        return {"dx": dx, "dw": dy.t() @ _exact_values(s["xc"], s["xs"]), "db": dy.sum(0)}
    if c["kind"] == "rope":
        return {"y": _exact_rope(c, s["x"], s["pos"])}
    return _exact_logprob(c, s)
