"""GPU parity of the language-model operators against the fp64 oracle: 8-bit checkpoints, the RMS norm with 8-bit output
and its gradient, the weight gradient from a checkpoint, token log probabilities and their gradient.

Bounds: EPS = 2^-24 is half a unit in the last place of fp32.  A sum of n terms taken in any order is within n * EPS of
the sum of magnitudes; results are rounded once to their type (HALF ulp)."""
import math

import numpy as np
import pytest
import torch

from oracle import lm_oracle as O
from paper_2208_05631_b200 import libqasg
from tests import _gpu_util as U

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
TYPES = {"f32": (libqasg.F32, torch.float32), "bf16": (libqasg.BF16, torch.bfloat16), "f16": (libqasg.F16, torch.float16)}
HALF = {kind: torch.finfo(dtype).eps / 2 for kind, (_, dtype) in TYPES.items()}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -24}  # below: spacing of f16 subnormals


@pytest.fixture(scope="module")
def ctx():
    c = libqasg.Context(1 << 12, 64, device=0)
    yield c
    c.close()


def _f64(t):
    return t.detach().cpu().double().numpy()


def _rows(a, dtype, pad=0, offset=0, fill=float("nan")):
    """A [rows][cols] tensor of `dtype` with `pad` extra columns and a base `offset` elements into its storage, `fill`
    everywhere else; values rounded to the type."""
    rows, cols = a.shape
    flat = torch.full((offset + rows * (cols + pad) + 64,), fill, dtype=torch.float32, device=U.dev()).to(dtype)
    t = flat[offset: offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float64)).to(U.dev()).to(dtype))
    return t


def _untouched(t, fill):
    """The storage behind a _rows tensor outside of its rows still holds `fill`."""
    rows, cols = t.shape
    full = torch.as_strided(t, (t.untyped_storage().nbytes() // t.element_size(),), (1,), 0).clone()
    at = t.storage_offset() + torch.arange(rows, device=t.device)[:, None] * t.stride(0) + torch.arange(cols, device=t.device)
    full[at.reshape(-1)] = fill
    return bool((full == fill).all())


def _act(rows, cols):
    """An Act whose memory is poisoned and guarded by extra columns and a row."""
    blocks = -(-cols // 32)
    codes = torch.full((rows + 1, blocks * 32 + 32), 77, dtype=torch.int8, device=U.dev())
    exps = torch.full((rows + 1, (blocks + 15) // 16 * 16 + 16), 99, dtype=torch.uint8, device=U.dev())
    return libqasg.Act(codes, exps, rows, cols)


def _act_of(a):
    """A guarded Act that holds the 8-bit form of a (fp64 rows), its values, its unused bytes hostile."""
    act = _act(*a.shape)
    codes, exps = O.pack(a)
    act.codes[: len(a), : codes.shape[1]] = U.to_dev(codes)
    act.exps[:] = 255
    act.exps[: len(a), : exps.shape[1]] = U.to_dev(exps)
    return act, O.values(codes, exps, a.shape[1])


def _act_guards(act):
    blocks = -(-act.cols // 32)
    assert (act.codes[act.rows:] == 77).all() and (act.codes[:, blocks * 32:] == 77).all()
    assert (act.exps[act.rows:] == 99).all() and (act.exps[:, blocks:] == 99).all()
    return act.codes[: act.rows, : blocks * 32].cpu().numpy(), act.exps[: act.rows, :blocks].cpu().numpy()


def _normal(rng, *shape, scale=1.0):
    return rng.standard_normal(shape) * scale * np.exp(rng.standard_normal(shape[-1]) * 0.7)


def _shards(rng, rows, M):
    """Uneven row ranges, some empty."""
    cuts = np.sort(rng.integers(0, rows + 1, M - 1)) if M > 1 else []
    s = [0, *[int(c) for c in cuts], rows]
    if M > 2:
        s[2] = s[1]
    return s


# ------------------------------------------------------------------ checkpoints
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols,pad,offset", [(1, 1, 0, 0), (3, 31, 1, 0), (2, 33, 0, 3), (5, 64, 8, 0), (130, 1000, 24, 8),
                                                  (7, 1025, 0, 1), (9, 5003, 3, 5), (1, 20000, 0, 0), (70, 32, 0, 0)])
def test_pack_and_unpack(ctx, kind, rows, cols, pad, offset):
    code, dtype = TYPES[kind]
    rng = np.random.default_rng(rows + cols)
    a = _normal(rng, rows, cols)
    a[rng.random(a.shape) < 0.02] *= 1e3
    a[0, : min(cols, 32)] = 0.0
    x = _rows(a, dtype, pad, offset)
    act = _act(rows, cols)
    ctx.act_pack(code, x, x.stride(0), act)
    codes, exps = _act_guards(act)
    want = O.pack(_f64(x))
    assert np.array_equal(codes, want[0]) and np.array_equal(exps, want[1])
    v = O.values(*want, cols)
    for other, (ocode, odtype) in TYPES.items():
        out = _rows(np.zeros((rows, cols)), odtype, pad, offset, fill=5.0)
        ctx.act_unpack(act, ocode, out, out.stride(0))
        with np.errstate(over="ignore"):
            expect = torch.from_numpy(v).to(torch.float32).to(odtype)
        assert torch.equal(out.cpu(), expect), other
        assert _untouched(out, 5.0)
    assert ctx.last_async_status() == libqasg.OK


def test_pack_edges(ctx):
    a = np.zeros((8, 40))
    a[1] = 2.0 ** -140                  # fp32 subnormals: far below the smallest exponent
    a[2, 7], a[2, 39] = 2.0 ** -126, 3.0e38
    a[3, :2] = 1.0, -1.9999             # 128 is kept at 127
    a[4, 5] = np.inf
    a[5, 33] = np.nan
    a[6, :4] = 64.0, 0.5, 1.5, 2.5      # ties to even
    a[7] = -0.0
    x = _rows(a, torch.float32)
    act = _act(8, 40)
    ctx.act_pack(libqasg.F32, x, x.stride(0), act)
    codes, exps = _act_guards(act)
    want = O.pack(_f64(x))
    assert np.array_equal(codes, want[0]) and np.array_equal(exps, want[1])
    assert codes[6, :4].tolist() == [64, 0, 2, 2] and exps[4, 0] == 255 and exps[4, 1] == 7 and exps[5].tolist() == [7, 255]
    out = torch.empty((8, 40), device=U.dev())
    ctx.act_unpack(act, libqasg.F32, out, 40)
    assert np.array_equal(_f64(out), O.values(*want, 40), equal_nan=True)
    assert ctx.last_async_status() == libqasg.ERR_NONFINITE
    assert ctx.last_async_status() == libqasg.OK


# ------------------------------------------------------------------ norm
NORM_SHAPES = [(1, 1, 0, 0), (1, 4096, 0, 0), (5, 33, 3, 1), (19, 256, 0, 0), (37, 257, 0, 0), (9, 1000, 8, 0), (3, 1024, 0, 8), (6, 2047, 1, 0),
               (5, 4096, 8, 0), (4, 5003, 5, 3), (3, 8192, 0, 0), (2, 16384, 0, 0), (300, 64, 0, 0)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols,pad,offset", NORM_SHAPES)
def test_rmsnorm_pack(ctx, kind, rows, cols, pad, offset):
    code, dtype = TYPES[kind]
    rng = np.random.default_rng(cols + rows)
    residual, weighted, in_place = cols % 2 == 1 or cols == 4096, rows != 3, rows == 5
    eps = 1e-5
    x = _rows(_normal(rng, rows, cols), dtype, pad, offset)
    r = _rows(_normal(rng, rows, cols), dtype, pad, offset) if residual else None
    w = torch.from_numpy(rng.standard_normal(cols).astype(np.float32)).to(U.dev()) if weighted else None
    h32 = x.float() + (r.float() if residual else 0.0)
    h64 = _f64(h32)
    h = x if in_place else _rows(np.zeros((rows, cols)), dtype, pad, offset, fill=5.0)
    y = _rows(np.zeros((rows, cols)), dtype, 0, offset, fill=5.0)
    rstd = torch.full((rows + 1,), -1.0, device=U.dev())
    act = _act(rows, cols)
    ctx.rmsnorm_pack(code, x, x.stride(0), r, r.stride(0) if residual else 0, w, eps, h, h.stride(0), y, y.stride(0), act, rstd)
    codes, exps = _act_guards(act)
    assert ctx.last_async_status() == libqasg.OK
    assert torch.equal(h, h32.to(dtype))
    assert _untouched(y, 5.0) and (in_place or _untouched(h, 5.0)) and rstd[rows] == -1.0
    n, want_rstd = O.rmsnorm(h64, eps)
    rel = (32 + 16 + 4) * EPS   # 32 squares a thread, the tree, the division and the root
    assert (np.abs(_f64(rstd)[:rows] - want_rstd) <= rel * want_rstd).all()
    unit = np.ldexp(1.0, exps.astype(int) - 133).repeat(32, axis=1)[:, :cols]
    v = O.values(codes, exps, cols)
    # half a unit, a whole one where the code is held at 127; 128 units times the error of n on top
    assert (np.abs(v - n) <= np.where(np.abs(n) > 127 * unit, 1.0, 0.5) * unit + 2 * rel * np.abs(n)).all()
    top = np.abs(O._blocks(n)).max(-1)
    assert (np.ldexp(1.0, exps.astype(int) - 127) <= top * (1 + 2 * rel)).all()
    assert ((np.ldexp(1.0, exps.astype(int) - 126) >= top * (1 - 2 * rel))).all()
    want_y = v * (_f64(w) if weighted else 1.0)
    assert (np.abs(_f64(y) - want_y) <= (HALF[kind] + EPS) * np.abs(want_y) + TINY[kind]).all()


@pytest.mark.parametrize("rows,cols", [(64, 64), (64, 1000), (32, 4096), (8, 9001)])
def test_rmsnorm_pack_fp32_rounds_like_exact_rows(ctx, rows, cols):
    # Sums of squares of small whole numbers are exact in fp32, 1 / sqrt is two floats: what is left is one rounding of n.
    x = torch.from_numpy(np.random.default_rng(cols).integers(-40, 41, (rows, cols)).astype(np.float32)).to(U.dev())
    rstd = torch.empty(rows, device=U.dev())
    act = _act(rows, cols)
    ctx.rmsnorm_pack(TYPES["f32"][0], x, cols, None, 0, None, 0.0, None, 0, None, 0, act, rstd)
    codes, exps = _act_guards(act)
    n, _ = O.rmsnorm(_f64(x), 0.0)
    unit = np.ldexp(1.0, exps.astype(int) - 133).repeat(32, axis=1)[:, :cols]
    away = np.abs(O.values(codes, exps, cols) - n) - np.where(np.abs(n) > 127 * unit, 1.0, 0.5) * unit
    assert (away <= 2.0 ** -24 * (1 + 2.0 ** -20) * np.abs(n)).all()


def test_rmsnorm_pack_without_outputs_and_nonfinite(ctx):
    rows, cols = 4, 96
    a = np.ones((rows, cols))
    a[1] = 0.0
    a[2, 40] = np.nan
    a[3, 70] = np.inf
    x = _rows(a, torch.bfloat16)
    act = _act(rows, cols)
    rstd = torch.empty(rows, device=U.dev())
    ctx.rmsnorm_pack(libqasg.BF16, x, x.stride(0), None, 0, None, 1e-6, None, 0, None, 0, act, rstd)
    codes, exps = _act_guards(act)
    assert (codes[0] == 64).all() or (codes[0] == 127).all()   # 1 or the number just below it
    assert not codes[1].any() and (exps[1] == 7).all()
    assert (exps[2] == 255).all()                              # the whole row's norm is NaN
    assert exps[3, 2] == 255 and not codes[3].any()            # 1/inf = 0, inf * 0 = NaN
    assert ctx.last_async_status() == libqasg.ERR_NONFINITE


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,cols,pad,offset", NORM_SHAPES + [(700, 300, 0, 0), (1500, 2048, 0, 0), (160, 5120, 0, 0), (3, 6144, 0, 0), (2, 6145, 0, 0), (300, 9000, 0, 0), (150, 16381, 3, 1)])
def test_rmsnorm_grad(ctx, kind, rows, cols, pad, offset):
    code, dtype = TYPES[kind]
    rng = np.random.default_rng(3 * cols + rows)
    residual, weighted, in_place, M = cols % 2 == 0, rows != 3, rows == 5, 1 + rows % 7
    act, n = _act_of(O.rmsnorm(_normal(rng, rows, cols), 1e-5)[0])
    dy = _rows(_normal(rng, rows, cols, scale=0.1), dtype, pad, offset)
    dres = _rows(_normal(rng, rows, cols, scale=0.1), dtype, pad, offset) if residual else None
    rstd = torch.from_numpy(np.exp(rng.standard_normal(rows)).astype(np.float32)).to(U.dev())
    w = torch.from_numpy(rng.standard_normal(cols).astype(np.float32)).to(U.dev()) if weighted else None
    shards = _shards(rng, rows, M)
    gw = torch.full((M, cols + 3), 7.0, device=U.dev())
    scratch = libqasg.new_scratch(libqasg.rmsnorm_grad_scratch_bytes(cols, M))
    dy64, dres64 = _f64(dy), _f64(dres) if residual else None
    dx = dy if in_place else _rows(np.zeros((rows, cols)), dtype, pad, offset, fill=5.0)
    args = (act, rstd, w, M, shards)
    ctx.rmsnorm_grad(code, dy, dy.stride(0), dres, dres.stride(0) if residual else 0, *args, dx, dx.stride(0), gw, cols + 3, False,
                     scratch)
    w64, r64 = _f64(w) if weighted else 1.0, _f64(rstd)
    want, dwt = O.rmsnorm_grad(dy64, n, r64, w64, dres64)
    u = np.abs(dy64 * w64)
    terms = 32 + 16
    mean_abs = (u * np.abs(n)).mean(-1, keepdims=True)
    bound = r64[:, None] * (np.abs(n) * mean_abs * (terms + 4) * EPS + 4 * EPS * (u + np.abs(n) * mean_abs)) \
        + (HALF[kind] + 2 * EPS) * np.abs(want) + TINY[kind] + (2 * EPS * np.abs(dres64) if residual else 0.0)
    assert (np.abs(_f64(dx) - want) <= bound).all()
    assert in_place or _untouched(dx, 5.0)
    assert (gw[:, cols:] == 7.0).all()
    for m, (a, b) in enumerate(zip(shards, shards[1:])):
        assert (np.abs(_f64(gw[m, :cols]) - dwt[a:b].sum(0)) <= (b - a + 2) * EPS * np.abs(dwt[a:b]).sum(0)).all()
    if not in_place:   # added to what is there, and the same bits again without the weight gradient
        first, dx1 = gw.clone(), dx.clone()
        ctx.rmsnorm_grad(code, dy, dy.stride(0), dres, dres.stride(0) if residual else 0, *args, dx, dx.stride(0), gw, cols + 3, True,
                         scratch)
        assert torch.equal(gw[:, :cols], (first + first)[:, :cols]) and torch.equal(dx, dx1)
        ctx.rmsnorm_grad(code, dy, dy.stride(0), dres, dres.stride(0) if residual else 0, *args, dx, dx.stride(0), None, 0, False, None)
        assert torch.equal(dx, dx1)
    assert ctx.last_async_status() == libqasg.OK


def test_rmsnorm_gradient_against_differences(ctx):
    """The gradient of sum(dy * weight * h / rms(h)) + sum(dres * h) by central differences of the fp64 function, in 32
    directions.  The kernel works from n^, within 2^-6 of its block's largest value of n."""
    rng = np.random.default_rng(5)
    rows, cols, eps = 6, 384, 1e-4
    h, dy, dres = (rng.standard_normal((rows, cols)).astype(np.float32).astype(np.float64) for _ in range(3))
    w = rng.standard_normal(cols).astype(np.float32).astype(np.float64)
    x = _rows(h, torch.float32)
    act, rstd = libqasg.new_act(rows, cols), torch.empty(rows, device=U.dev())
    wd = U.to_dev(w.astype(np.float32))
    ctx.rmsnorm_pack(libqasg.F32, x, x.stride(0), None, 0, wd, eps, None, 0, None, 0, act, rstd)
    dx = torch.empty((rows, cols), device=U.dev())
    ctx.rmsnorm_grad(libqasg.F32, U.to_dev(dy.astype(np.float32)), cols, U.to_dev(dres.astype(np.float32)), cols, act, rstd, wd, 1,
                     [0, rows], dx, cols, None, 0, False, None)
    dx = _f64(dx)
    n, r = O.rmsnorm(h, eps)
    top = np.abs(O._blocks(n)).max(-1).repeat(32, axis=1)[:, :cols]
    err = top * 2.0 ** -6                       # |n^ - n|: a unit, and a unit is at most 2^-6 of the block's largest
    u = np.abs(dy * w)
    worst = r[:, None] * (err * (u * np.abs(n)).mean(-1, keepdims=True) + (np.abs(n) + err) * (u * err).mean(-1, keepdims=True))
    f = lambda v: (dy * w * O.rmsnorm(v, eps)[0]).sum() + (dres * v).sum()  # noqa: E731
    for _ in range(32):
        d = rng.standard_normal((rows, cols))
        want = (f(h + 1e-5 * d) - f(h - 1e-5 * d)) / 2e-5
        assert abs((dx * d).sum() - want) <= (worst * np.abs(d)).sum() + 1e-5 * np.abs(dx * d).sum()


# ------------------------------------------------------------------ weight gradient
WGRAD_SHAPES = [(1, 1, 1, 1, 0, 0), (0, 5, 40, 2, 0, 0), (1, 130, 257, 1, 0, 0), (5, 64, 64, 3, 8, 0), (63, 128, 256, 1, 0, 0),
                (64, 256, 512, 1, 0, 8), (65, 300, 33, 4, 1, 3), (200, 72, 1000, 7, 0, 0), (513, 512, 256, 2, 0, 0),
                (1000, 257, 514, 5, 7, 1), (2100, 128, 96, 1, 0, 0), (3000, 40, 2050, 16, 0, 0), (300, 1160, 700, 3, 0, 0),
                (25000, 20, 33, 4, 1, 0),   # longer than the scratch holds of dy in another form: in parts
                (200, 1500, 3000, 3, 0, 0), (1100, 1500, 3400, 1, 4, 0)]   # several rounds of tiles; the last ones cut in pieces


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,out,cols,M,pad,offset", WGRAD_SHAPES)
def test_wgrad_is_exact_on_small_integers(ctx, kind, rows, out, cols, M, pad, offset):
    """Codes and output gradients that are small integers: every partial sum is an integer below 2^24, so the fp32
    result is exact whatever the order."""
    code, dtype = TYPES[kind]
    rng = np.random.default_rng(rows + out)
    act, a = _act_of(rng.integers(-31, 32, (rows, cols)).astype(float)) if rows else (libqasg.new_act(1, cols), None)
    if not rows:
        act = libqasg.Act(act.codes, act.exps, 0, cols)
        a = np.zeros((0, cols))
    dy64 = rng.integers(-8, 9, (rows, out)).astype(float)
    dy = _rows(dy64, dtype, pad, offset)
    w64 = 2.0 ** rng.integers(-2, 3, cols)
    w = U.to_dev(w64.astype(np.float32)) if out % 2 else None
    shards = _shards(rng, rows, M)
    want = O.wgrad(dy64, a, shards, w64 if out % 2 else None)
    ld_w, ld_g = cols + 3 * (out % 3), out * (cols + 3 * (out % 3)) + 5
    g = torch.full((M, ld_g), 7.0, device=U.dev())
    scratch = libqasg.new_scratch(libqasg.act_wgrad_scratch_bytes(out, cols, M))
    ctx.act_wgrad(code, dy, max(dy.stride(0), out), out, act, w, M, shards, g, ld_g, ld_w, False, scratch)
    inner = g[:, : out * ld_w].reshape(M, out, ld_w)
    assert np.array_equal(_f64(inner[:, :, :cols]), want)
    guard = g.clone()
    guard[:, : out * ld_w].view(M, out, ld_w)[:, :, :cols] = 7.0
    assert (guard == 7.0).all()
    ctx.act_wgrad(code, dy, max(dy.stride(0), out), out, act, w, M, shards, g, ld_g, ld_w, True, scratch)
    assert np.array_equal(_f64(inner[:, :, :cols]), 2 * want)
    assert ctx.last_async_status() == libqasg.OK


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,out,cols,M", [(700, 200, 300, 3), (3000, 128, 256, 1), (257, 520, 130, 2), (8192, 64, 96, 1)])
def test_wgrad_of_real_values(ctx, kind, rows, out, cols, M):
    code, dtype = TYPES[kind]
    rng = np.random.default_rng(rows)
    act, a = _act_of(_normal(rng, rows, cols, scale=3.0))
    dy = _rows(_normal(rng, rows, out, scale=0.01), dtype)
    w64 = rng.standard_normal(cols).astype(np.float32).astype(np.float64)
    shards = _shards(rng, rows, M)
    g = torch.empty((M, out * cols), device=U.dev())
    scratch = libqasg.new_scratch(libqasg.act_wgrad_scratch_bytes(out, cols, M))
    ctx.act_wgrad(code, dy, dy.stride(0), out, act, U.to_dev(w64.astype(np.float32)), M, shards, g, out * cols, cols, False, scratch)
    dy64 = _f64(dy)
    want = O.wgrad(dy64, a, shards, w64)
    size = np.stack([np.abs(dy64[i:j]).T @ np.abs(a[i:j]) for i, j in zip(shards, shards[1:])]) * np.abs(w64)
    got = _f64(g).reshape(M, out, cols)
    # products are exact; every addition is within 2 EPS (rounding or truncation) of the magnitudes summed so far
    assert (np.abs(got - want) <= (2 * rows + 4) * EPS * size).all()
    # and far nearer on the whole: as a chain of fp32 additions of independent errors
    assert np.linalg.norm(got - want) <= 4 * EPS * math.sqrt(rows) * np.linalg.norm(want) + EPS * np.linalg.norm(want)
    again = torch.empty_like(g)
    ctx.act_wgrad(code, dy, dy.stride(0), out, act, U.to_dev(w64.astype(np.float32)), M, shards, again, out * cols, cols, False, scratch)
    assert torch.equal(g, again)


def test_wgrad_keeps_other_rows_out(ctx):
    """NaNs of one worker's rows, of columns past the layer and of a NaN block stay where they belong."""
    rng = np.random.default_rng(9)
    rows, out, cols = 150, 136, 160
    a = rng.standard_normal((rows, cols))
    a[70, 40] = np.nan                                    # block 1 of row 70: worker 1
    act, _ = _act_of(a)
    dy = _rows(rng.standard_normal((rows, out)), torch.bfloat16, pad=8)   # padding is NaN
    dy[100, 5] = float("nan")
    dy[149, 7] = float("inf")
    shards = [0, 50, 90, 150]
    g = torch.empty((3, out * cols), device=U.dev())
    scratch = libqasg.new_scratch(libqasg.act_wgrad_scratch_bytes(out, cols, 3))
    ctx.act_wgrad(libqasg.BF16, dy, dy.stride(0), out, act, None, 3, shards, g, out * cols, cols, False, scratch)
    g = _f64(g).reshape(3, out, cols)
    assert np.isfinite(g[0]).all()
    assert np.isnan(g[1][:, 32:64]).all() and np.isfinite(np.delete(g[1], range(32, 64), axis=1)).all()
    assert np.isnan(g[2][5]).all() and not np.isfinite(g[2][7]).any()
    assert np.isfinite(np.delete(g[2], [5, 7], axis=0)).all()


# ------------------------------------------------------------------ token log probabilities
LOGPROB_SHAPES = [(1, 1, 0, 0, 1), (3, 2, 1, 0, 2), (5, 37, 0, 3, 32), (4, 1000, 24, 0, 5), (2, 4096, 0, 0, 20), (3, 4097, 0, 1, 8),
                  (1, 131072, 0, 0, 20), (2, 50021, 3, 5, 32), (300, 17000, 0, 0, 1), (150, 33000, 1, 0, 0), (6, 70001, 0, 7, 3)]


def _check_logprob(out, x, tokens, k, V):
    r = O.token_logprob(x, tokens)
    keep = np.ones(len(x), bool) if tokens is None else r["keep"]
    big = np.abs(np.where(np.isfinite(x), x, 0.0)).max(-1)
    # an exponent's argument is within 2 EPS of the largest |x| log2 e, a power within 2^-22, a thread adds V / 128 of them
    tol = EPS * (V / 128 + 64 + 6 * big + 8)
    for name, width in (("lse", 1.0), ("logprob", 1.0), ("entropy", None)):
        if out[name] is None:
            continue
        got, want = _f64(out[name]), r[name] if name in r else None
        wide = (2 + np.abs(np.where(np.isfinite(want), want, 0.0))) * 2 if width is None else 1.0
        fine = np.isfinite(want)
        assert np.array_equal(got[~fine], want[~fine]), name
        bound = tol * wide + 4 * EPS * np.abs(np.where(fine, want, 0.0)) + 2 * EPS * big
        assert (np.abs(got[fine] - want[fine]) <= bound[fine]).all(), name
    if k:
        ids = O.top(x, k)
        assert np.array_equal(out["top_ids"].cpu().numpy(), np.where(keep[:, None], ids, -1))
        want = np.where(keep[:, None], np.take_along_axis(r["logp"], ids, 1), 0.0)
        got, fine = _f64(out["top_logprob"]), np.isfinite(want)
        assert np.array_equal(got[~fine], want[~fine])
        bound = tol[:, None] + 4 * EPS * np.abs(np.where(fine, want, 0.0)) + 2 * EPS * big[:, None]
        assert (np.abs(got[fine] - want[fine]) <= bound[fine]).all()


def _logprob(ctx, kind, t, tokens, k):
    rows, V = t.shape
    out = {n: torch.full((rows,), -3.0, device=U.dev()) for n in ("lse", "entropy")}
    out["logprob"] = torch.full((rows,), -3.0, device=U.dev()) if tokens is not None else None
    out["top_ids"] = torch.full((rows, k), -3, dtype=torch.int64, device=U.dev())
    out["top_logprob"] = torch.full((rows, k), -3.0, device=U.dev())
    ctx.token_logprob(TYPES[kind][0], t, t.stride(0), rows, V, tokens, out["logprob"], out["entropy"], out["lse"], k, out["top_ids"],
                      out["top_logprob"])
    return out


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,V,pad,offset,k", LOGPROB_SHAPES)
def test_token_logprob_and_gradient(ctx, kind, rows, V, pad, offset, k):
    code, dtype = TYPES[kind]
    rng = np.random.default_rng(V + rows)
    a = rng.standard_normal((rows, V)) * 3
    if rows > 2:
        a[1, rng.random(V) < 0.6] = -np.inf
        a[2, rng.random(V) < 0.9] = float(torch.finfo(dtype).min)
    tokens = rng.integers(0, V, rows)
    if rows > 4:
        tokens[3] = -1
    x = _rows(a, dtype, pad, offset)
    x64, tok = _f64(x), U.to_dev(tokens)
    out = _logprob(ctx, kind, x, tok, k)
    _check_logprob(out, x64, tokens, k, V)
    # gradient from these very outputs
    gp, gh, gl = (rng.standard_normal(rows).astype(np.float32) for _ in range(3))
    for gs in ((gp, gh, gl), (gp, None, None), (None, gh, None)):
        dx = _rows(np.zeros((rows, V)), dtype, 0, offset, fill=5.0)
        ctx.token_logprob_grad(code, x, x.stride(0), rows, V, tok, out["lse"], out["entropy"],
                               *(None if g is None else U.to_dev(g) for g in gs), dx, dx.stride(0))
        _check_grad(dx, x64, tokens, gs, out, kind)
        assert _untouched(dx, 5.0)
    dx = dx.clone()
    ctx.token_logprob_grad(code, x, x.stride(0), rows, V, tok, out["lse"], out["entropy"], None, U.to_dev(gh), None, x, x.stride(0))
    assert torch.equal(x, dx)                         # in place
    assert ctx.last_async_status() == libqasg.OK


def _check_grad(dx, x, tokens, gs, out, kind):
    want = O.token_logprob_grad(x, tokens, *gs)
    r = O.token_logprob(x)
    p = np.exp(r["logp"])
    logp = np.where(p > 0, r["logp"], 0.0)
    gp, gh, gl = (np.zeros(len(x)) if g is None else np.abs(g.astype(np.float64)) for g in gs)
    V = x.shape[1]
    big = np.abs(np.where(np.isfinite(x), x, 0.0)).max(-1)
    off = EPS * (V / 128 + 64 + 6 * big + 8) + 8 * EPS * np.abs(np.where(np.isfinite(r["lse"]), r["lse"], 0.0))  # of lse; entropy 2 (2 + H) times
    H = np.abs(r["entropy"])
    size = (gp + gl)[:, None] + gh[:, None] * (np.abs(logp) + H[:, None])
    rel = off[:, None] + (np.abs(logp) + 8) * 4 * EPS
    bound = p * (size * rel + gh[:, None] * (off * (1 + 2 * (2 + H)))[:, None] + 4 * EPS * size) + (HALF[kind] + 4 * EPS) * np.abs(want)
    bound += np.where(np.abs(want) > 0, 4 * EPS, 0) * gp[:, None] + TINY[kind]
    assert (np.abs(_f64(dx) - want) <= bound).all()


@pytest.mark.parametrize("V", [40, 5000, 40000])
def test_token_logprob_special_rows(ctx, V):
    """Rows of ties, of masks, of NaN and infinity; rising and falling rows, the worst order for the candidates."""
    rng = np.random.default_rng(V)
    a = np.zeros((12, V))
    a[1] = -np.inf
    a[2, :] = -np.inf
    a[2, V // 2] = -7.0
    a[3] = np.arange(V) * 0.01
    a[4] = -np.arange(V) * 0.01
    a[5] = rng.integers(0, 3, V)
    a[6] = np.float32(np.finfo(np.float32).min)
    a[7] = rng.standard_normal(V)
    a[7, V - 1] = np.nan
    a[8] = rng.standard_normal(V)
    a[8, 1] = np.inf
    a[9] = np.where(rng.random(V) < 0.5, -0.0, 0.0)
    a[10] = 1e4
    a[10, 3] = -1e4
    a[11] = np.nan
    a[11, ::3] = 1.0
    tokens = np.array([5, 5, V // 2, 0, 0, 1, 2, 3, 4, 5, 3, 0])
    x = _rows(a, torch.float32)
    out = _logprob(ctx, "f32", x, U.to_dev(tokens), 32)
    assert ctx.last_async_status() == libqasg.ERR_NONFINITE
    x64 = _f64(x)
    assert np.array_equal(out["top_ids"].cpu().numpy(), O.top(x64, 32))
    bad = [7, 8, 11]
    good = [i for i in range(12) if i not in bad]
    sub = {n: t[good] for n, t in out.items()}
    _check_logprob(sub, x64[good], tokens[good], 32, V)
    for n in ("lse", "entropy", "logprob"):
        assert out[n][bad].isnan().all()
    assert out["entropy"][1] == 0 and out["logprob"][1] == -math.inf and (out["top_logprob"][1] == -math.inf).all()
    ones = torch.ones(12, device=U.dev())
    dx = torch.full((12, V), 5.0, device=U.dev())
    ctx.token_logprob_grad(libqasg.F32, x, x.stride(0), 12, V, U.to_dev(tokens), out["lse"], out["entropy"], ones, ones, ones, dx, V)
    assert dx[bad].isnan().all() and (dx[1] == 0).all() and dx[good].isfinite().all()


def test_token_logprob_without_tokens_and_bad_tokens(ctx):
    rng = np.random.default_rng(11)
    x = _rows(rng.standard_normal((6, 500)), torch.bfloat16)
    out = _logprob(ctx, "bf16", x, None, 4)
    _check_logprob(out, _f64(x), None, 4, 500)
    dx = torch.empty((6, 500), dtype=torch.bfloat16, device=U.dev())
    gh = rng.standard_normal(6).astype(np.float32)
    ctx.token_logprob_grad(libqasg.BF16, x, x.stride(0), 6, 500, None, out["lse"], out["entropy"], U.to_dev(gh), U.to_dev(gh), None, dx, 500)
    _check_grad(dx, _f64(x), None, (None, gh, None), out, "bf16")
    assert ctx.last_async_status() == libqasg.OK
    tokens = np.array([499, 500, -5, 0, 1 << 40, 7])
    out = _logprob(ctx, "bf16", x, U.to_dev(tokens), 4)
    _check_logprob(out, _f64(x), tokens, 4, 500)
    assert ctx.last_async_status() == libqasg.ERR_BAD_INDEX


def test_token_logprob_gradient_against_differences(ctx):
    rng = np.random.default_rng(12)
    rows, V = 5, 900
    x64 = rng.standard_normal((rows, V)).astype(np.float32).astype(np.float64) * 2
    tokens = rng.integers(0, V, rows)
    x, tok = _rows(x64, torch.float32), U.to_dev(tokens)
    gs = [rng.standard_normal(rows).astype(np.float32) for _ in range(3)]
    out = _logprob(ctx, "f32", x, tok, 0)
    dx = torch.empty((rows, V), device=U.dev())
    ctx.token_logprob_grad(libqasg.F32, x, x.stride(0), rows, V, tok, out["lse"], out["entropy"], *(U.to_dev(g) for g in gs), dx, V)

    def f(v):
        r = O.token_logprob(v, tokens)
        return (gs[0] * r["logprob"] + gs[1] * r["entropy"] + gs[2] * r["lse"]).sum()

    for _ in range(16):
        d = rng.standard_normal((rows, V))
        want = (f(x64 + 1e-5 * d) - f(x64 - 1e-5 * d)) / 2e-5
        assert abs((_f64(dx) * d).sum() - want) <= 2e-5 * (np.abs(_f64(dx)) * np.abs(d)).sum() + 1e-7


# ------------------------------------------------------------------ boundary
def test_refusals_enqueue_nothing(ctx):
    Q = libqasg
    act = Q.new_act(8, 64)
    x = torch.zeros((8, 64), dtype=torch.bfloat16, device=U.dev())
    f = torch.zeros(64 * 64, device=U.dev())
    ids = torch.zeros(8, dtype=torch.int64, device=U.dev())
    big = Q.new_scratch(max(Q.act_wgrad_scratch_bytes(64, 64, 2), Q.rmsnorm_grad_scratch_bytes(64, 2)))
    odd = x.view(torch.uint8).reshape(-1)[1:]
    codes, exps = act.codes, act.exps
    sh = [0, 3, 8]

    def bad_act(**kw):
        a = Q.Act(codes, exps, 8, 64)
        for k, v in kw.items():
            setattr(a.struct, k, v)
        return a

    cases = [
        (Q.ERR_INVALID_ARG, lambda: ctx.act_pack(3, x, 64, act)),
        (Q.ERR_INVALID_ARG, lambda: ctx.act_pack(Q.BF16, x, 63, act)),
        (Q.ERR_INVALID_ARG, lambda: ctx.act_pack(Q.BF16, None, 64, act)),
        (Q.ERR_ALIGNMENT, lambda: ctx.act_pack(Q.BF16, odd, 64, act)),
        (Q.ERR_INVALID_ARG, lambda: ctx.act_pack(Q.BF16, x, 64, bad_act(struct_size=8))),
        (Q.ERR_INVALID_ARG, lambda: ctx.act_pack(Q.BF16, x, 64, bad_act(cols=0))),
        (Q.ERR_INVALID_ARG, lambda: ctx.act_pack(Q.BF16, x, 64, bad_act(codes=0))),
        (Q.ERR_INVALID_ARG, lambda: ctx.act_pack(Q.BF16, x, 64, bad_act(ld_codes=32))),
        (Q.ERR_ALIGNMENT, lambda: ctx.act_pack(Q.BF16, x, 64, bad_act(ld_codes=72))),
        (Q.ERR_ALIGNMENT, lambda: ctx.act_pack(Q.BF16, x, 64, bad_act(ld_exps=8))),
        (Q.ERR_ALIGNMENT, lambda: ctx.act_unpack(bad_act(exps=exps.data_ptr() + 1), Q.BF16, x, 64)),
        (Q.ERR_INVALID_ARG, lambda: ctx.rmsnorm_pack(Q.BF16, x, 64, None, 0, None, -1.0, None, 0, x, 64, act, f)),
        (Q.ERR_INVALID_ARG, lambda: ctx.rmsnorm_pack(Q.BF16, x, 64, None, 0, None, float("nan"), None, 0, x, 64, act, f)),
        (Q.ERR_INVALID_ARG, lambda: ctx.rmsnorm_pack(Q.BF16, x, 64, None, 0, None, 1e-5, None, 0, x, 64, act, None)),
        (Q.ERR_INVALID_ARG, lambda: ctx.rmsnorm_pack(Q.BF16, x, 64, x, 10, None, 1e-5, None, 0, x, 64, act, f)),
        (Q.ERR_ALIGNMENT, lambda: ctx.rmsnorm_pack(Q.BF16, x, 64, None, 0, f.data_ptr() + 2, 1e-5, None, 0, x, 64, act, f)),
        (Q.ERR_INVALID_ARG, lambda: ctx.rmsnorm_grad(Q.BF16, x, 64, None, 0, act, f, None, 2, [0, 3, 7], x, 64, f, 64, False, big)),
        (Q.ERR_INVALID_ARG, lambda: ctx.rmsnorm_grad(Q.BF16, x, 64, None, 0, act, f, None, 2, [0, 9, 8], x, 64, f, 64, False, big)),
        (Q.ERR_INVALID_ARG, lambda: ctx.rmsnorm_grad(Q.BF16, x, 64, None, 0, act, f, None, 2, sh, x, 64, f, 60, False, big)),
        (Q.ERR_WORKSPACE, lambda: ctx.rmsnorm_grad(Q.BF16, x, 64, None, 0, act, f, None, 2, sh, x, 64, f, 64, False, big[:64])),
        (Q.ERR_INVALID_ARG, lambda: ctx.act_wgrad(Q.BF16, x, 64, 0, act, None, 2, sh, f, 64 * 64, 64, False, big)),
        (Q.ERR_INVALID_ARG, lambda: ctx.act_wgrad(Q.BF16, x, 64, 65, act, None, 2, sh, f, 65 * 64, 64, False, big)),
        (Q.ERR_INVALID_ARG, lambda: ctx.act_wgrad(Q.BF16, x, 64, 64, act, None, 2, sh, f, 64 * 63, 64, False, big)),
        (Q.ERR_INVALID_ARG, lambda: ctx.act_wgrad(Q.BF16, x, 64, 64, act, None, 2, sh, f, 64 * 64, 63, False, big)),
        (Q.ERR_INVALID_ARG, lambda: ctx.act_wgrad(Q.BF16, x, 64, 64, act, None, 0, [0], f, 64 * 64, 64, False, big)),
        (Q.ERR_ALIGNMENT, lambda: ctx.act_wgrad(Q.BF16, x, 64, 64, act, None, 2, sh, f, 64 * 64, 64, False, big[8:])),
        (Q.ERR_INVALID_ARG, lambda: ctx.token_logprob(Q.BF16, x, 64, 8, 0, ids, f, f, f)),
        (Q.ERR_INVALID_ARG, lambda: ctx.token_logprob(Q.BF16, x, 63, 8, 64, ids, f, f, f)),
        (Q.ERR_INVALID_ARG, lambda: ctx.token_logprob(Q.BF16, x, 64, 8, 64, None, f, f, f)),
        (Q.ERR_INVALID_ARG, lambda: ctx.token_logprob(Q.BF16, x, 64, 8, 64, ids, f, f, f, 33, ids, f)),
        (Q.ERR_INVALID_ARG, lambda: ctx.token_logprob(Q.BF16, x, 64, 8, 5, ids, f, f, f, 6, ids, f)),
        (Q.ERR_ALIGNMENT, lambda: ctx.token_logprob(Q.BF16, x, 64, 8, 64, ids.data_ptr() + 4, f, f, f)),
        (Q.ERR_INVALID_ARG, lambda: ctx.token_logprob_grad(Q.BF16, x, 64, 8, 64, ids, None, f, f, f, f, x, 64)),
        (Q.ERR_INVALID_ARG, lambda: ctx.token_logprob_grad(Q.BF16, x, 64, 8, 64, ids, f, None, f, f, f, x, 64)),
        (Q.ERR_INVALID_ARG, lambda: ctx.token_logprob_grad(Q.BF16, x, 64, 8, 64, ids, f, f, f, f, f, None, 64)),
    ]
    before = ctx.launch_count()
    for want, call in cases:
        with pytest.raises(Q.QasgError) as e:
            call()
        assert e.value.status == want
    # sizes the norm and a struct cannot take
    wide = Q.Act(torch.empty((1, 16416), dtype=torch.int8, device=U.dev()), torch.empty((1, 528), dtype=torch.uint8, device=U.dev()), 1, 16385)
    xw = torch.zeros((1, 16385), device=U.dev())
    with pytest.raises(Q.QasgError):
        ctx.rmsnorm_pack(Q.F32, xw, 16385, None, 0, None, 1e-5, None, 0, None, 0, wide, f)
    # nothing to do: accepted, nothing launched
    none = Q.Act(codes, exps, 0, 64)
    ctx.act_pack(Q.F32, None, 64, none), ctx.act_unpack(none, Q.F32, None, 64)
    ctx.rmsnorm_pack(Q.F32, None, 64, None, 0, None, 1e-5, None, 0, None, 0, none, None)
    ctx.token_logprob(Q.F32, None, 64, 0, 64, None, None, None, None)
    ctx.token_logprob_grad(Q.F32, None, 64, 0, 64, None, None, None, None, None, None, None, 64)
    assert ctx.launch_count() == before
    assert ctx.last_async_status() == Q.OK


def test_one_training_pass_on_a_side_stream_and_from_a_graph(ctx):
    """norm -> checkpoint -> weight gradient, norm gradient and log probabilities chained on one stream that is not the
    current one; then the same calls captured in a graph and replayed: the same bits."""
    rng = np.random.default_rng(21)
    rows, cols, V, M = 96, 256, 1000, 2
    x, r = (_rows(rng.standard_normal((rows, cols)), torch.bfloat16) for _ in range(2))
    w = U.to_dev(rng.standard_normal(cols).astype(np.float32))
    dlog = torch.empty((rows, V), dtype=torch.bfloat16, device=U.dev())
    wt = U.to_dev((rng.standard_normal((V, cols)) * 0.1).astype(np.float32)).to(torch.bfloat16)
    tok = U.to_dev(rng.integers(0, V, rows))
    gp = torch.full((rows,), -1.0 / rows, device=U.dev())
    act = libqasg.new_act(rows, cols)
    y, dx = torch.empty((rows, cols), dtype=torch.bfloat16, device=U.dev()), torch.empty((rows, cols), dtype=torch.bfloat16, device=U.dev())
    rstd, lp, ent, lse = (torch.empty(rows, device=U.dev()) for _ in range(4))
    g, gw = torch.empty((M, V * cols), device=U.dev()), torch.empty((M, cols), device=U.dev())
    s1 = libqasg.new_scratch(libqasg.act_wgrad_scratch_bytes(V, cols, M))
    s2 = libqasg.new_scratch(libqasg.rmsnorm_grad_scratch_bytes(cols, M))
    sh = [0, 40, rows]

    def one_pass():
        ctx.rmsnorm_pack(libqasg.BF16, x, x.stride(0), r, r.stride(0), w, 1e-5, None, 0, y, cols, act, rstd)
        logits = y @ wt.t()
        ctx.token_logprob(libqasg.BF16, logits, V, rows, V, tok, lp, ent, lse)
        ctx.token_logprob_grad(libqasg.BF16, logits, V, rows, V, tok, lse, ent, gp, None, None, dlog, V)
        ctx.act_wgrad(libqasg.BF16, dlog, V, V, act, w, M, sh, g, V * cols, cols, False, s1)
        ctx.rmsnorm_grad(libqasg.BF16, dlog @ wt, cols, None, 0, act, rstd, w, M, sh, dx, cols, gw, cols, False, s2)

    outs = (lp, ent, lse, g, gw, dx, y, dlog)
    one_pass()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    assert all(t.isfinite().all() for t in want)
    side = torch.cuda.Stream()
    for t in outs:
        t.fill_(9.0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one_pass()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one_pass()
    for t in outs:
        t.fill_(9.0)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert ctx.last_async_status() == libqasg.OK
