"""The language-model operators together, as a training loop uses them: the gradients of one step against the fp64 formulas
on the same data, and a loss that falls."""
import math

import numpy as np
import pytest
import torch

from examples import lm_head_training as E
from oracle import lm_oracle as O
from paper_2208_05631_b200 import libqasg

pytestmark = pytest.mark.gpu


def _f64(t):
    return t.detach().cpu().double().numpy()


def test_gradients_of_one_step():
    m = E.LmHead(workers=3, tokens_per_worker=50, dim=96, vocab=130, seed=5)
    now, then = m.batch()
    loss, entropy = m.gradients(now, then)
    n, _ = O.rmsnorm(_f64(m.embedding[now].float() + m.branch[now].float()), E.EPS)
    n = O.values(*O.pack(n), m.dim)
    W, w = _f64(m.x[: m.nw].view(m.vocab, m.dim)), _f64(m.x[m.nw:])
    x = (n * w) @ W.T
    tokens = then.cpu().numpy()
    r = O.token_logprob(x, tokens)
    dlog = O.token_logprob_grad(x, tokens, _f64(m.g_logprob))
    # y, W, the logits and their gradient pass through bf16 (2^-8 each): the losses within that of the logits' size,
    # the gradients within a few of it on the whole
    assert abs(float(loss) + r["logprob"].mean()) <= 4 * 2.0 ** -8 * np.abs(x).max()
    assert abs(float(entropy) - r["entropy"].mean()) <= 8 * 2.0 ** -8 * np.abs(x).max()
    want = O.wgrad(dlog, n, m.shards, w).reshape(m.M, -1)
    got = _f64(m.g)
    assert np.linalg.norm(got[:, : m.nw] - want) <= 4 * 2.0 ** -8 * np.linalg.norm(want)
    dwt = (dlog @ W) * n
    want = np.stack([dwt[a:b].sum(0) for a, b in zip(m.shards, m.shards[1:])])
    assert np.linalg.norm(got[:, m.nw: m.d] - want) <= 4 * 2.0 ** -8 * np.linalg.norm(want) + 2.0 ** -8 * np.linalg.norm(dwt) / math.sqrt(m.rows)
    assert m.ctx.last_async_status() == libqasg.OK


def test_the_loss_falls():
    model, losses = E.train(steps=60, workers=4, tokens_per_worker=256, dim=128, vocab=200)
    assert all(math.isfinite(v) for v in losses)
    assert losses[0] > 0.8 * math.log(200)
    assert sum(losses[-5:]) / 5 < 0.5 * losses[0]
