"""What is measured of the language-model operators: the RMS norm with 8-bit output and its gradient, 8-bit activation
checkpoints and the weight gradient taken from them, and the log probabilities of given tokens with their gradient.

listed() and draw() give cases, prepare() their inputs, run() one pass: the plain form in elementary torch operations in
32 bits, or, with `own` set, the calls of the library.  work() is what a pass cannot do without, exact() the definition
in 64 bits.

Checkpoint format (both forms): blocks of 32 values along a row share one exponent E = max(floor(log2(largest
magnitude)), -120), kept as the byte E + 127; a value's code is a * 2^(6-E) rounded to the nearest integer (ties to even)
within [-127, 127], and stands for code * 2^(E-6)."""
import math

import torch

own = False

BLOCK = 32
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one token of a decoding step: latency
        {"name": "norm_token", "op": "norm", "rows": 1, "cols": 4096, "type": "bf16", "residual": True, "weight": True, "pad": 0},
        # a training micro-batch through a block's norm
        {"name": "norm_batch", "op": "norm", "rows": 8192, "cols": 4096, "type": "bf16", "residual": True, "weight": True, "pad": 0},
        # its backward pass: eight workers' tokens in one call
        {"name": "norm_grad_batch", "op": "norm_grad", "rows": 8192, "cols": 4096, "type": "bf16", "residual": True, "weight": True,
         "workers": 8, "pad": 0},
        # odd width and row stride, half precision, shards of uneven length
        {"name": "norm_grad_odd", "op": "norm_grad", "rows": 1537, "cols": 5003, "type": "f16", "residual": True, "weight": True,
         "workers": 3, "pad": 5},
        # the wide inner activation of a feed-forward layer, saved and restored
        {"name": "checkpoint_wide", "op": "checkpoint", "rows": 8192, "cols": 16384, "type": "bf16", "pad": 0},
        # weight gradient of a small layer and a short batch: launch and latency
        {"name": "wgrad_small", "op": "wgrad", "rows": 256, "out": 512, "cols": 512, "type": "bf16", "workers": 1, "weight": True, "pad": 0},
        # a full-width layer over a training micro-batch: matrix arithmetic
        {"name": "wgrad_batch", "op": "wgrad", "rows": 8192, "out": 4096, "cols": 4096, "type": "bf16", "workers": 1, "weight": True, "pad": 0},
        # eight workers with uneven shards, odd sizes, half-precision output gradients
        {"name": "wgrad_workers", "op": "wgrad", "rows": 3001, "out": 1000, "cols": 2050, "type": "f16", "workers": 8, "weight": False, "pad": 0},
        # one row of logits: decoding with log probabilities and alternatives
        {"name": "logprob_token", "op": "logprob", "rows": 1, "vocab": 131072, "type": "bf16", "top": 20, "masked": 0.0, "padded": 0.0, "pad": 0},
        # scoring a training batch over a large vocabulary
        {"name": "logprob_batch", "op": "logprob", "rows": 2048, "vocab": 131072, "type": "bf16", "top": 8, "masked": 0.0, "padded": 0.05, "pad": 0},
        # odd vocabulary, 32-bit logits, a third of the vocabulary masked out
        {"name": "logprob_odd", "op": "logprob", "rows": 701, "vocab": 50021, "type": "f32", "top": 5, "masked": 0.33, "padded": 0.1, "pad": 3},
        # the loss's backward pass over the same batch
        {"name": "logprob_grad_batch", "op": "logprob_grad", "rows": 2048, "vocab": 131072, "type": "bf16", "masked": 0.0, "padded": 0.05, "pad": 0},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "checkpoint", "wgrad", "logprob", "logprob_grad"])
    case = {"op": op, "type": rng.choice(["bf16", "bf16", "f16", "f32"])}
    pad = rng.choice([0, 0, 8, rng.randint(1, 40)])
    if op in ("norm", "norm_grad", "checkpoint"):
        rows, cols = _log_uniform(rng, 1, 8192), _log_uniform(rng, 64, 16384)
        if rng.random() < 0.5:
            cols = (cols + 63) // 64 * 64
        rows = max(1, min(rows, (8192 * 4096 * 2) // (cols * SIZE[case["type"]])))
        case |= {"rows": rows, "cols": cols, "pad": pad}
        if op != "checkpoint":
            case |= {"residual": rng.random() < 0.7, "weight": rng.random() < 0.8}
        if op == "norm_grad":
            case["workers"] = rng.randint(1, 16)
    elif op == "wgrad":
        rows, out, cols = _log_uniform(rng, 16, 8192), _log_uniform(rng, 64, 4096), _log_uniform(rng, 64, 4096)
        if rng.random() < 0.5:
            out, cols = (out + 63) // 64 * 64, (cols + 63) // 64 * 64
        case |= {"rows": rows, "out": out, "cols": cols, "workers": rng.randint(1, 8), "weight": rng.random() < 0.5, "pad": pad}
    else:
        rows, vocab = _log_uniform(rng, 1, 2048), _log_uniform(rng, 1000, 131072)
        rows = max(1, min(rows, (2048 * 131072 * 2) // (vocab * SIZE[case["type"]])))
        case |= {"rows": rows, "vocab": vocab, "masked": rng.choice([0.0, 0.0, round(rng.random(), 2)]),
                 "padded": rng.choice([0.0, 0.1]), "pad": pad}
        if op == "logprob":
            case["top"] = rng.choice([0, 1, 5, 20, 32])
    return case


# ------------------------------------------------------------------ inputs
def _shards(rows, workers, seed):
    """Row ranges of the workers: uneven and, with more workers than rows, some of them empty."""
    g = torch.Generator().manual_seed(seed)
    cuts = torch.sort(torch.randint(0, rows + 1, (workers - 1,), generator=g)).values.tolist() if workers > 1 else []
    even = [rows * (m + 1) // workers for m in range(workers - 1)]
    inner = [(a + 3 * b) // 4 for a, b in zip(cuts, even)]
    return [0] + inner + [rows]


def _strided(rows, cols, pad, dtype):
    return torch.zeros((rows, cols + pad), dtype=dtype, device="cuda")[:, :cols]


def _normal(rows, cols, pad, dtype, gen, scale=1.0):
    t = _strided(rows, cols, pad, dtype)
    t.copy_(torch.randn((rows, cols), generator=gen, device="cuda") * scale)
    return t


def _activations(rows, cols, gen):
    """Normal values times a scale of each column's own, a few columns far above the rest, as in hidden states."""
    col = torch.exp(0.5 * torch.randn((cols,), generator=gen, device="cuda"))
    col[torch.randint(0, cols, (max(1, cols // 512),), generator=gen, device="cuda")] *= 20.0
    return torch.randn((rows, cols), generator=gen, device="cuda") * col


def _pow2(e):
    """2^e as fp32 for whole e in [-126, 127]."""
    return ((e + 127) << 23).view(torch.float32)


def _pack(x):
    """Codes (int8) and exponent bytes of fp32 rows."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    full = torch.zeros((rows, blocks * BLOCK), dtype=torch.float32, device=x.device)
    full[:, :cols] = x
    full = full.view(rows, blocks, BLOCK)
    e = (torch.frexp(full.abs().amax(-1)).exponent - 1).clamp(min=-120).to(torch.int32)
    codes = torch.round(full * _pow2(6 - e)[..., None]).clamp(-127, 127)
    return codes.view(rows, blocks * BLOCK).to(torch.int8), (e + 127).to(torch.uint8)


def _values(codes, exps, cols):
    """What the codes stand for, in fp32."""
    rows, blocks = exps.shape
    v = codes[:, : blocks * BLOCK].float().view(rows, blocks, BLOCK) * _pow2(exps.to(torch.int32) - 133)[..., None]
    return v.view(rows, blocks * BLOCK)[:, :cols]


def _checkpoint(x):
    """A kept checkpoint as a program holds it: rows of codes in whole blocks, exponent rows of whole 16 bytes."""
    codes, exps = _pack(x)
    kept = torch.zeros((exps.shape[0], (exps.shape[1] + 15) // 16 * 16), dtype=torch.uint8, device=x.device)
    kept[:, : exps.shape[1]] = exps
    return codes.contiguous(), kept


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, dtype, pad, rows = case["op"], TYPES[case["type"]], case["pad"], case["rows"]
    s = {"op": op, "case": case, "dtype": dtype}
    empty = lambda *shape, dtype=dtype: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if op in ("norm", "norm_grad", "checkpoint", "wgrad"):
        cols = case["cols"]
        blocks = -(-cols // BLOCK)
        if case.get("weight"):
            s["weight"] = 1.0 + 0.2 * torch.randn((cols,), generator=gen, device="cuda")
    if op in ("norm_grad", "wgrad"):
        s["shards"] = _shards(rows, case["workers"], seed)
    if op in ("norm", "checkpoint"):
        s["x"] = _strided(rows, cols, pad, dtype)
        s["x"].copy_(_activations(rows, cols, gen))
        s["codes"], s["exps"] = empty(rows, blocks * BLOCK, dtype=torch.int8), empty(rows, (blocks + 15) // 16 * 16, dtype=torch.uint8)
        s["values"] = empty(rows, cols, dtype=torch.bfloat16)
    if op == "norm":
        s["residual"] = _normal(rows, cols, pad, dtype, gen, 2.0) if case["residual"] else None
        s["h"] = empty(rows, cols) if case["residual"] else None
        s["y"], s["rstd"] = empty(rows, cols), empty(rows, dtype=torch.float32)
    elif op == "norm_grad":
        h = _activations(rows, cols, gen)
        s["rstd"] = torch.rsqrt((h * h).mean(-1) + EPS)
        s["codes"], s["exps"] = _checkpoint(h * s["rstd"][:, None])
        s["dy"] = _normal(rows, cols, pad, dtype, gen, 0.02)
        s["dres"] = _normal(rows, cols, pad, dtype, gen, 0.02) if case["residual"] else None
        s["dx"], s["dw"] = empty(rows, cols), empty(case["workers"], cols + (-cols) % 4, dtype=torch.float32)
    elif op == "wgrad":
        s["codes"], s["exps"] = _checkpoint(_activations(rows, cols, gen))
        s["dy"] = _normal(rows, case["out"], pad, dtype, gen, 0.02)
        d = case["out"] * cols
        s["g"] = empty(case["workers"], d + (-d) % 4, dtype=torch.float32)
    elif op in ("logprob", "logprob_grad"):
        vocab = case["vocab"]
        x = torch.randn((rows, vocab), generator=gen, device="cuda") * 2.5
        tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
        x.scatter_add_(1, tokens[:, None], 10.0 * torch.rand((rows, 1), generator=gen, device="cuda"))
        if case["masked"]:
            out = torch.rand((vocab,), generator=gen, device="cuda") < case["masked"]
            out[int(seed) % vocab] = False
            x[:, out] = -math.inf
        if case["padded"]:
            tokens[torch.randperm(rows, generator=gen, device="cuda")[: int(rows * case["padded"])]] = -1
        s["logits"], s["tokens"] = _strided(rows, vocab, pad, dtype), tokens
        s["logits"].copy_(x)
        del x
        if op == "logprob":
            k = case["top"]
            s["logprob"], s["entropy"], s["lse"] = (empty(rows, dtype=torch.float32) for _ in range(3))
            s["top_ids"], s["top_logprob"] = empty(rows, k, dtype=torch.int64), empty(rows, k, dtype=torch.float32)
        else:
            _, _, s["entropy"], s["lse"] = _plain_logprob(s["logits"].float(), tokens)
            s["g_logprob"] = -(0.5 + torch.rand((rows,), generator=gen, device="cuda")) / rows
            s["g_entropy"] = 0.1 * torch.randn((rows,), generator=gen, device="cuda") / rows
            s["g_lse"] = 0.1 * torch.randn((rows,), generator=gen, device="cuda") / rows
            s["dlogits"] = empty(rows, vocab)
    return s


# ------------------------------------------------------------------ plain forms
def _plain_logprob(x, tokens):
    """(log probabilities of all tokens, of the given ones, entropy, log-sum-exp); rows with a negative token give 0."""
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    z = x - m
    log_s = torch.log(torch.exp(z).sum(-1, keepdim=True))
    logp = z - log_s
    p = torch.exp(logp)
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(-1)
    given = logp.gather(1, tokens.clamp(min=0)[:, None])[:, 0]
    keep = tokens >= 0
    zero = torch.zeros_like(given)
    return logp, torch.where(keep, given, zero), torch.where(keep, entropy, zero), torch.where(keep, (m + log_s)[:, 0], zero)


def _top(x, k):
    """Columns of the k largest values of each row; of equal values the lowest column first."""
    bits = (x + 0.0).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).to(torch.int64)
    column = torch.arange(x.shape[1], device=x.device)
    key = (order << 32) | (0x7FFFFFFF - column)
    return 0x7FFFFFFF - (torch.topk(key, k, dim=1).values & 0x7FFFFFFF)


def _run_plain(s):
    op, case, dtype = s["op"], s["case"], s["dtype"]
    w = s.get("weight")
    if op == "norm":
        h = s["x"].float() + (s["residual"].float() if case["residual"] else 0.0)
        rstd = 1.0 / torch.sqrt((h * h).mean(-1) + EPS)
        values = _values(*_pack(h * rstd[:, None]), case["cols"])
        out = {"y": (values * w if w is not None else values).to(dtype), "rstd": rstd, "values": values.to(torch.bfloat16)}
        if case["residual"]:
            out["h"] = h.to(dtype)
        return out
    if op == "checkpoint":
        return {"values": _values(*_pack(s["x"].float()), case["cols"]).to(torch.bfloat16)}
    if op == "norm_grad":
        n = _values(s["codes"], s["exps"][:, : -(-case["cols"] // BLOCK)], case["cols"])
        dy = s["dy"].float()
        u = dy * w if w is not None else dy
        dx = s["rstd"][:, None] * (u - n * (u * n).mean(-1, keepdim=True))
        if case["residual"]:
            dx = dx + s["dres"].float()
        dw = dy * n
        return {"dx": dx.to(dtype), "dw": torch.stack([dw[a:b].sum(0) for a, b in zip(s["shards"], s["shards"][1:])])}
    if op == "wgrad":
        a = _values(s["codes"], s["exps"][:, : -(-case["cols"] // BLOCK)], case["cols"])
        dy = s["dy"].float()
        g = torch.stack([dy[i:j].t() @ a[i:j] for i, j in zip(s["shards"], s["shards"][1:])])
        return {"g": g * w if w is not None else g}
    x, tokens = s["logits"].float(), s["tokens"]
    keep = (tokens >= 0)[:, None]
    if op == "logprob":
        logp, given, entropy, lse = _plain_logprob(x, tokens)
        ids = _top(x, case["top"])
        return {"logprob": given, "entropy": entropy, "lse": lse, "top_ids": torch.where(keep, ids, -1),
                "top_logprob": torch.where(keep, logp.gather(1, ids), 0.0)}
    logp = x - s["lse"][:, None]
    p = torch.exp(logp)
    inner = torch.where(p > 0, logp + s["entropy"][:, None], 0.0)
    dx = p * ((s["g_lse"] - s["g_logprob"])[:, None] - s["g_entropy"][:, None] * inner)
    dx.scatter_add_(1, tokens.clamp(min=0)[:, None], s["g_logprob"][:, None])
    return {"dlogits": torch.where(keep, dx, 0.0).to(dtype)}


# ------------------------------------------------------------------ the library's calls
_context = None


def _library():
    """The program's one context and the binding."""
    global _context
    from paper_2208_05631_b200 import libqasg
    if _context is None:
        _context = libqasg.Context(1 << 16, 64, device=torch.cuda.current_device())
    return libqasg, _context


def _kept(s, key, make):
    """What a program makes once and keeps with its buffers: a handle, a workspace."""
    if key not in s:
        s[key] = make()
    return s[key]


def _run_own(s):
    lib, ctx = _library()
    op, case = s["op"], s["case"]
    kind = {"bf16": lib.BF16, "f16": lib.F16, "f32": lib.F32}[case["type"]]
    rows, w = case["rows"], s.get("weight")
    if op in ("norm", "norm_grad", "checkpoint", "wgrad"):
        cols = case["cols"]
        act = _kept(s, "act", lambda: lib.Act(s["codes"], s["exps"], rows, cols))
    if op == "norm":
        x, r, h, y = s["x"], s["residual"], s["h"], s["y"]
        ctx.rmsnorm_pack(kind, x, x.stride(0), r, r.stride(0) if r is not None else 0, w, EPS, h, cols if h is not None else 0,
                         y, cols, act, s["rstd"])
        ctx.act_unpack(act, lib.BF16, s["values"], cols)
        return {"y": y, "rstd": s["rstd"], "values": s["values"]} | ({"h": h} if h is not None else {})
    if op == "checkpoint":
        ctx.act_pack(kind, s["x"], s["x"].stride(0), act)
        ctx.act_unpack(act, lib.BF16, s["values"], cols)
        return {"values": s["values"]}
    if op == "norm_grad":
        dy, r, dw = s["dy"], s["dres"], s["dw"]
        scratch = _kept(s, "scratch", lambda: lib.new_scratch(lib.rmsnorm_grad_scratch_bytes(cols, case["workers"])))
        ctx.rmsnorm_grad(kind, dy, dy.stride(0), r, r.stride(0) if r is not None else 0, act, s["rstd"], w, case["workers"],
                         s["shards"], s["dx"], cols, dw, dw.stride(0), False, scratch)
        return {"dx": s["dx"], "dw": dw[:, :cols]}
    if op == "wgrad":
        dy, g, out = s["dy"], s["g"], case["out"]
        scratch = _kept(s, "scratch", lambda: lib.new_scratch(lib.act_wgrad_scratch_bytes(out, cols, case["workers"])))
        ctx.act_wgrad(kind, dy, dy.stride(0), out, act, w, case["workers"], s["shards"], g, g.stride(0), cols, False, scratch)
        return {"g": g[:, : out * cols].unflatten(1, (out, cols))}
    x, vocab = s["logits"], case["vocab"]
    if op == "logprob":
        ctx.token_logprob(kind, x, x.stride(0), rows, vocab, s["tokens"], s["logprob"], s["entropy"], s["lse"], case["top"],
                          s["top_ids"], s["top_logprob"])
        return {k: s[k] for k in ("logprob", "entropy", "lse", "top_ids", "top_logprob")}
    ctx.token_logprob_grad(kind, x, x.stride(0), rows, vocab, s["tokens"], s["lse"], s["entropy"], s["g_logprob"], s["g_entropy"],
                           s["g_lse"], s["dlogits"], vocab)
    return {"dlogits": s["dlogits"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------ work and exact values
def work(case):
    op, rows, size = case["op"], case["rows"], SIZE[case["type"]]
    if op in ("norm", "norm_grad", "checkpoint"):
        cols = case["cols"]
        n, code = rows * cols, 1.0 + 1.0 / BLOCK
        res, w = int(case.get("residual", False)), 4 * cols * int(case.get("weight", False))
        if op == "norm":  # x, residual -> h, y, codes, rstd; codes -> their values
            return {"bytes": n * (size * (2 + 2 * res) + code + 2) + w + 4 * rows, "flops": 8 * n}
        if op == "checkpoint":
            return {"bytes": n * (size + code + 2), "flops": 4 * n}
        return {"bytes": n * (size * (2 + res) + code) + w + 4 * rows + 4 * cols * case["workers"], "flops": 10 * n}
    if op == "wgrad":
        cols, out = case["cols"], case["out"]
        return {"bytes": rows * (out * size + cols * (1.0 + 1.0 / BLOCK)) + 4 * out * cols * case["workers"],
                "flops": 2 * rows * out * cols}
    n = (rows - int(rows * case["padded"])) * case["vocab"]
    if op == "logprob":
        return {"bytes": n * size + rows * (20 + 12 * case["top"]), "flops": 6 * n}
    return {"bytes": n * size + rows * case["vocab"] * size + 28 * rows, "flops": 6 * n}


def _exact_values(codes, exps, cols):
    e = exps.double().repeat_interleave(BLOCK, dim=1)[:, :cols]
    return codes[:, :cols].double() * torch.exp2(e - 133.0)


def _exact_round(a):
    """The values that the 8-bit form of fp64 rows stands for."""
    rows, cols = a.shape
    full = torch.nn.functional.pad(a, (0, (-cols) % BLOCK)).unflatten(1, (-1, BLOCK))
    top = full.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -120)))
    e = e + (torch.exp2(e + 1) <= top).double() - (torch.exp2(e) > top.clamp(min=2.0 ** -120)).double()
    unit = torch.exp2(e - 6)
    return ((full / unit).round().clamp(-127, 127) * unit).flatten(1)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    w = s["weight"].double() if "weight" in s else 1.0
    if op == "norm":
        h = s["x"].double()
        if case["residual"]:
            h = h + s["residual"].double()
        rstd = (h.square().sum(1) / case["cols"] + EPS) ** -0.5
        n = _exact_round(h * rstd[:, None])
        return {"y": n * w, "rstd": rstd, "values": n} | ({"h": h} if case["residual"] else {})
    if op == "checkpoint":
        return {"values": _exact_round(s["x"].double())}
    if op in ("norm_grad", "wgrad"):
        n = _exact_values(s["codes"], s["exps"], case["cols"])
        dy = s["dy"].double()
        owner = torch.zeros(case["rows"], dtype=torch.int64)
        for m, (a, b) in enumerate(zip(s["shards"], s["shards"][1:])):
            owner[a:b] = m
        owner = owner.cuda()
    if op == "norm_grad":
        u = dy * w
        dx = (u - n * ((u * n).sum(1) / case["cols"])[:, None]) * s["rstd"].double()[:, None]
        if case["residual"]:
            dx = dx + s["dres"].double()
        dw = torch.zeros((case["workers"], case["cols"]), dtype=torch.float64, device="cuda").index_add_(0, owner, dy * n)
        return {"dx": dx, "dw": dw}
    if op == "wgrad":
        return {"g": torch.stack([(dy * (owner == m)[:, None]).t() @ (n * w) for m in range(case["workers"])])}
    x, tokens = s["logits"].double(), s["tokens"]
    keep = (tokens >= 0).double()
    lse = torch.logsumexp(x, 1)
    if op == "logprob":
        given = x.gather(1, tokens.clamp(min=0)[:, None])[:, 0] - lse
        p = torch.softmax(x, 1)
        mean = (p * x.clamp(min=-1e30)).sum(1)
        top = torch.sort(x, dim=1, descending=True).values[:, : case["top"]] - lse[:, None]
        return {"logprob": torch.where(keep > 0, given, 0.0), "entropy": (lse - mean) * keep, "lse": lse * keep, "top_ids": None,
                "top_logprob": torch.where(keep[:, None] > 0, top, 0.0)}
    logp = x - s["lse"].double()[:, None]
    p = logp.exp()
    dx = p * (s["g_lse"] - s["g_logprob"]).double()[:, None]
    dx -= s["g_entropy"].double()[:, None] * p * (logp.clamp(min=-1e30) + s["entropy"].double()[:, None])
    dx[torch.arange(case["rows"], device="cuda"), tokens.clamp(min=0)] += s["g_logprob"].double()
    return {"dlogits": dx * keep[:, None]}
