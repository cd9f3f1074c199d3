"""The language-model operators in numpy fp64, from their definitions: the 8-bit block format, the RMS norm with its
gradient, the weight gradient from a checkpoint, log probabilities with entropy and alternatives, and their gradient.
Slow and plain: test infrastructure only."""
import numpy as np

BLOCK = 32


def _blocks(a):
    a = np.asarray(a, dtype=np.float64)
    rows, cols = a.shape
    full = np.zeros((rows, -(-cols // BLOCK) * BLOCK))
    full[:, :cols] = a
    return full.reshape(rows, -1, BLOCK)


def pack(a):
    """(codes int8 [rows][whole blocks], exponent bytes uint8 [rows][blocks])."""
    full = _blocks(a)
    bad = ~np.isfinite(full).all(-1)
    full = np.where(bad[..., None], 0.0, full)
    top = np.abs(full).max(-1)
    e = np.maximum(np.where(top > 0, np.frexp(top)[1] - 1, -120), -120)
    codes = np.clip(np.rint(np.ldexp(full, (6 - e)[..., None])), -127, 127).astype(np.int8)
    return codes.reshape(len(codes), -1), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, exps, cols):
    """What codes and exponent bytes stand for."""
    blocks = -(-cols // BLOCK)
    c = np.asarray(codes)[:, : blocks * BLOCK].astype(np.float64).reshape(len(codes), blocks, BLOCK)
    b = np.asarray(exps)[:, :blocks].astype(np.int64)
    v = np.ldexp(c, (b - 133)[..., None])
    v = np.where((b == 255)[..., None], np.nan, v)
    return v.reshape(len(codes), -1)[:, :cols]


def rmsnorm(h, eps):
    """(n, rstd) of fp64 rows, before any rounding to 8 bits."""
    h = np.asarray(h, dtype=np.float64)
    rstd = 1.0 / np.sqrt((h * h).mean(-1) + eps)
    return h * rstd[:, None], rstd


def rmsnorm_grad(dy, n, rstd, weight=None, dres=None):
    """(dx, dy * n) from the normalised values that the checkpoint stands for."""
    dy = np.asarray(dy, dtype=np.float64)
    u = dy if weight is None else dy * weight
    dx = rstd[:, None] * (u - n * (u * n).mean(-1, keepdims=True))
    return dx if dres is None else dx + dres, dy * n


def wgrad(dy, a, shards, weight=None):
    """[M][out][cols]: dy^T a over each worker's rows, columns scaled by weight."""
    dy = np.asarray(dy, dtype=np.float64)
    g = np.stack([dy[i:j].T @ a[i:j] for i, j in zip(shards, shards[1:])])
    return g if weight is None else g * weight


def token_logprob(x, tokens=None):
    """dict of lse, entropy, logp (all tokens) and logprob (the given ones; padding rows 0 throughout)."""
    x = np.asarray(x, dtype=np.float64)
    m = x.max(-1, keepdims=True)
    empty = m == -np.inf
    z = x - np.where(empty, 0.0, m)
    e = np.exp(z)
    s = e.sum(-1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        logp = np.where(empty, -np.inf, z - np.log(s))
        entropy = np.where(empty[:, 0], 0.0, -np.where(e > 0, e / s * logp, 0.0).sum(-1))
        lse = np.where(empty, -np.inf, m + np.log(s))[:, 0]
    out = {"lse": lse, "entropy": entropy, "logp": logp}
    if tokens is not None:
        tokens = np.asarray(tokens)
        keep = (tokens >= 0) & (tokens < x.shape[1])
        given = logp[np.arange(len(x)), np.where(keep, tokens, 0)]
        out["logprob"] = np.where(keep, given, 0.0)
        out["lse"], out["entropy"], out["keep"] = np.where(keep, lse, 0.0), np.where(keep, entropy, 0.0), keep
    return out


def top(x, k):
    """Columns of the k largest of each row, NaN largest, ties to the lowest column."""
    x = np.asarray(x, dtype=np.float64)
    key = np.where(np.isnan(x), np.inf, x)
    rank = np.isnan(x).astype(np.int64)  # a NaN goes before an infinity
    return np.stack([np.lexsort((np.arange(len(r)), -r, -q))[:k] for r, q in zip(key, rank)])


def token_logprob_grad(x, tokens, g_logprob=None, g_entropy=None, g_lse=None):
    """Gradient of sum(g_logprob * logprob + g_entropy * entropy + g_lse * lse) for the logits."""
    r = token_logprob(x, tokens)
    x = np.asarray(x, dtype=np.float64)
    zero = np.zeros(len(x))
    gp, gh, gl = (zero if v is None else np.asarray(v, dtype=np.float64) for v in (g_logprob, g_entropy, g_lse))
    if tokens is None:
        gp = zero
    p = np.exp(r["logp"])
    logp = np.where(p > 0, r["logp"], 0.0)
    full = token_logprob(x)
    dx = p * ((gl - gp)[:, None] - gh[:, None] * (logp + full["entropy"][:, None]))
    if tokens is not None:
        dx[np.arange(len(x)), np.where(r["keep"], tokens, 0)] += gp
        dx[~r["keep"]] = 0.0
    dx[full["lse"] == -np.inf] = 0.0
    return dx
