"""Pins of the language-model oracle: the 8-bit format by its defining properties, the gradients by differences, the
log probabilities by closed forms."""
import numpy as np
import pytest

from oracle import lm_oracle as O


def test_block_format_properties():
    rng = np.random.default_rng(0)
    a = rng.standard_normal((7, 75)) * np.exp(rng.standard_normal((7, 75)) * 3)
    codes, exps = O.pack(a)
    assert codes.shape == (7, 96) and exps.shape == (7, 3) and not codes[:, 75:].any()
    v = O.values(codes, exps, 75)
    unit = np.ldexp(1.0, exps.astype(int) - 133).repeat(32, axis=1)[:, :75]
    assert (np.abs(v - a) <= np.where(np.abs(a) > 127 * unit, unit, unit / 2)).all()
    top = np.abs(O._blocks(a)).max(-1)
    assert (np.ldexp(1.0, exps.astype(int) - 127) <= top).all() and (np.ldexp(1.0, exps.astype(int) - 126) > top).all()
    assert np.array_equal(O.pack(v)[0], codes) and np.array_equal(O.pack(v)[1], exps)   # values repack to themselves
    assert np.array_equal(v.astype(np.float32).astype(np.float64), v)
    assert not (v.astype(np.float32).view(np.uint32) & 0xFFFF).any()                     # exact in bf16


def test_block_format_edges():
    a = np.zeros((6, 32))
    a[1, 3] = 2.0 ** -126          # below the smallest exponent: code 2^-126 * 2^126
    a[2, :2] = 1.0, -1.9999        # rounds to 128, kept at 127
    a[3, 5] = np.inf
    a[4, 6] = np.nan
    a[5, :2] = 3.0, 2.5 / 64       # 3 = 96 * 2^-5; 1.25 units
    codes, exps = O.pack(a)
    assert exps[:, 0].tolist() == [7, 7, 127, 255, 255, 128]
    assert codes[1, 3] == 1 and codes[2, :2].tolist() == [64, -127] and not codes[3].any() and not codes[4].any()
    assert codes[5, :2].tolist() == [96, 1]
    assert np.isnan(O.values(codes, exps, 32)[3:5]).all()


def _numeric(f, x, d, step):
    return (f(x + step * d) - f(x - step * d)) / (2 * step)


@pytest.mark.parametrize("weighted", [False, True])
def test_rmsnorm_gradient_by_differences(weighted):
    rng = np.random.default_rng(1)
    h, dy, dres, d = (rng.standard_normal((5, 40)) for _ in range(4))
    w = rng.standard_normal(40) if weighted else None
    scale = 1.0 if w is None else w
    n, rstd = O.rmsnorm(h, 1e-3)
    dx, dwt = O.rmsnorm_grad(dy, n, rstd, w, dres)
    want = _numeric(lambda v: (dy * scale * O.rmsnorm(v, 1e-3)[0]).sum() + (dres * v).sum(), h, d, 1e-6)
    assert abs((dx * d).sum() - want) <= 1e-7 * np.abs(dx * d).sum()
    dw = rng.standard_normal(40)
    want = _numeric(lambda v: (dy * v * n).sum(), np.ones(40), dw, 1e-3)
    assert abs((dwt.sum(0) * dw).sum() - want) <= 1e-9 * np.abs(dwt).sum()


def test_wgrad_by_differences():
    rng = np.random.default_rng(2)
    a, dy, wt, dw = rng.standard_normal((9, 6)), rng.standard_normal((9, 4)), rng.standard_normal(6), rng.standard_normal((4, 6))
    shards = [0, 4, 4, 9]
    g = O.wgrad(dy, a, shards, wt)
    assert not g[1].any()
    for m, (i, j) in enumerate(zip(shards, shards[1:])):
        want = _numeric(lambda v: (dy[i:j] * ((a[i:j] * wt) @ v.T)).sum(), np.zeros((4, 6)), dw, 1e-3)
        assert abs((g[m] * dw).sum() - want) <= 1e-9 * np.abs(g[m] * dw).sum() + 1e-12


def test_logprob_closed_forms():
    r = O.token_logprob(np.zeros((2, 8)), [3, -1])
    assert np.allclose(r["logprob"], [-np.log(8), 0]) and np.allclose(r["entropy"], [np.log(8), 0])
    x = np.array([[0.0, -np.inf, np.log(3.0)], [-np.inf] * 3])
    r = O.token_logprob(x, [2, 0])
    assert np.allclose(r["logprob"][0], np.log(0.75)) and r["logprob"][1] == -np.inf and r["entropy"][1] == 0
    assert np.allclose(r["entropy"][0], -(0.25 * np.log(0.25) + 0.75 * np.log(0.75)))
    assert O.top(np.array([[1.0, np.nan, 2.0, 2.0, np.inf, -0.0, 0.0]]), 7)[0].tolist() == [1, 4, 2, 3, 0, 5, 6]


def test_logprob_gradient_by_differences():
    rng = np.random.default_rng(3)
    x, d = rng.standard_normal((4, 11)) * 2, rng.standard_normal((4, 11))
    x[1, 4] = x[2, 0] = -np.inf
    d[~np.isfinite(x)] = 0
    tokens = np.array([3, 10, 2, -1])
    gp, gh, gl = rng.standard_normal((3, 4))
    dx = O.token_logprob_grad(x, tokens, gp, gh, gl)

    def loss(v):
        r = O.token_logprob(v, tokens)
        return (gp * r["logprob"] + gh * r["entropy"] + gl * r["lse"]).sum()

    assert abs((dx * d).sum() - _numeric(loss, x, d, 1e-5)) <= 1e-8 * np.abs(dx * d).sum() + 1e-9
    assert not dx[3].any() and dx[1, 4] == 0
