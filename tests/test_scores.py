"""Token scores and top-logit distillation without a GPU: the oracle's gradients
against differences, and what the entry points refuse."""
import ctypes

import numpy as np
import pytest

import paper_2607_24434_amd as de
from oracle import scores as orc

FAKE = 0x7F0000000000  # aligned, never dereferenced (validation fails first)
BIG = 1 << 34


def difference(f, l, h=1e-5):
    g = np.zeros_like(l)
    for i in range(l.size):
        a, b = l.copy(), l.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


@pytest.mark.parametrize("tau", [1.0, 0.6, 2.5])
@pytest.mark.parametrize("token,g,ge", [(3, 1.0, 0.0), (0, -2.0, 0.3), (-1, 5.0, 0.7)])
def test_scores_gradient_is_the_difference_quotient(tau, token, g, ge):
    l = np.random.default_rng(1).normal(0, 2, 23)

    def f(v):
        lp, h, *_ = orc.scores(v, tau, token, 0)
        return g * lp + ge * h

    want = difference(f, l)
    # A central difference is off by h^2 f''' / 6 (third derivatives of a softmax are below
    # 1 / tau^3) and by rounding, 2^-52 |f| / h.
    assert np.allclose(orc.scores(l, tau, token, 0, g, ge)[4], want, rtol=0, atol=1e-8)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.0])
@pytest.mark.parametrize("ids", [[4, 1, 7], [2], [5, -1, 5, 30, 0], list(range(12))])
def test_distill_gradient_is_the_difference_quotient(tail, tau, ids):
    rng = np.random.default_rng(2)
    l, t = rng.normal(0, 2, 12), rng.normal(0, 2, 12)
    lp = orc.log_softmax(t, tau) if tail else t
    v = [lp[i] if 0 <= i < 12 else 9.0 for i in ids]
    want = difference(lambda x: 1.7 * orc.distill(x, ids, v, tail, tau)[0], l)
    assert np.allclose(orc.distill(l, ids, v, tail, tau, 1.7)[1], want, rtol=0, atol=1e-8)


def test_distillation_from_oneself_is_zero():
    l = np.random.default_rng(3).normal(0, 2, 40)
    ids = list(np.argsort(-l)[:6])
    loss, grad = orc.distill(l, ids, orc.log_softmax(l, 1.5)[ids], True, 1.5)
    assert abs(loss) < 1e-13 and np.abs(grad).max() < 1e-14


def grad(g=FAKE, dlogits=FAKE + 4096, ldd=100, g_entropy=None):
    return de.make_row_grad(g, dlogits, ldd, g_entropy)


def token_scores(rows=2, V=100, dtype=de.DE_F32, logits=FAKE, ld=100, tau=1.0, tokens=FAKE,
                 logp=FAKE, entropy=FAKE, m=0, top_idx=None, top_logp=None, stats=None, grad=None,
                 ws=FAKE, ws_bytes=BIG):
    return de.LIB.de_token_scores(rows, V, dtype, logits, ld, tau, tokens, logp, entropy, m,
                                  top_idx, top_logp, stats,
                                  None if grad is None else ctypes.byref(grad), ws, ws_bytes, None)


SHARED = [
    (dict(rows=0), -1), (dict(rows=-1), -1), (dict(rows=(1 << 20) + 1), -1), (dict(V=0), -1),
    (dict(V=(1 << 30) + 1, ld=(1 << 30) + 1), -1), (dict(ld=99), -1), (dict(logits=None), -1),
    (dict(logits=FAKE + 2), -1), (dict(dtype=de.DE_BF16, logits=FAKE + 1), -1),
    (dict(dtype=de.DE_Q4_0), -2), (dict(dtype=-1), -2), (dict(tau=0.0), -1), (dict(tau=-1.0), -1),
    (dict(tau=float("nan")), -1), (dict(tau=float("inf")), -1), (dict(tau=1e-31), -1),
    (dict(rows=1 << 20, V=1 << 20, ld=1 << 20), -2),
]
GRADS = [
    (grad(g=None), -1), (grad(dlogits=None), -1), (grad(dlogits=FAKE + 2), -1), (grad(ldd=99), -1),
    (grad(dlogits=FAKE, ldd=101), -1),
]


@pytest.mark.parametrize("kw,code", SHARED + [
    (dict(tokens=None), -1), (dict(m=-1), -1), (dict(m=129, top_idx=FAKE, top_logp=FAKE), -1),
    (dict(V=5, m=6, top_idx=FAKE, top_logp=FAKE), -1), (dict(m=3, top_idx=FAKE), -1),
    (dict(m=3, top_logp=FAKE), -1), (dict(logp=None, entropy=None), -1), (dict(ws=None), -4),
    (dict(ws=FAKE + 64), -4), (dict(ws_bytes=16), -4),
    (dict(m=3, top_idx=FAKE, top_logp=FAKE, grad=grad()), -2),
    (dict(tokens=None, logp=None, grad=grad()), -1)] + [(dict(grad=g), c) for g, c in GRADS])
def test_token_scores_refuses(kw, code):
    assert token_scores(**kw) == code


@pytest.mark.parametrize("kw,code", SHARED + [(dict(stats=None), -1), (dict(grad=None), -1),
                                              (dict(tokens=None), -1)] + [
    (dict(grad=g), c) for g, c in GRADS])
def test_token_scores_grad_refuses(kw, code):
    a = dict(rows=2, V=100, dtype=de.DE_F32, logits=FAKE, ld=100, tau=1.0, tokens=FAKE, stats=FAKE,
             grad=grad())
    a.update(kw)
    g = a["grad"]
    assert de.LIB.de_token_scores_grad(a["rows"], a["V"], a["dtype"], a["logits"], a["ld"],
                                       a["tau"], a["tokens"], a["stats"],
                                       None if g is None else ctypes.byref(g), None) == code


LISTS = [(dict(m=0), -1), (dict(m=129), -1), (dict(ids=None), -1)]


@pytest.mark.parametrize("kw,code", SHARED + LISTS + [
    (dict(values=None), -1), (dict(loss=None), -1), (dict(tail=2), -2), (dict(ws=None), -4),
    (dict(ws=FAKE + 64), -4), (dict(ws_bytes=16), -4), (dict(grad=grad(g_entropy=FAKE)), -1)] + [
    (dict(grad=g), c) for g, c in GRADS])
def test_topk_distill_refuses(kw, code):
    a = dict(rows=2, V=100, dtype=de.DE_F32, logits=FAKE, ld=100, m=8, ids=FAKE, values=FAKE,
             tail=0, tau=1.0, loss=FAKE, state=None, grad=None, ws=FAKE, ws_bytes=BIG)
    a.update(kw)
    g = a["grad"]
    assert de.LIB.de_topk_distill(a["rows"], a["V"], a["dtype"], a["logits"], a["ld"], a["m"],
                                  a["ids"], a["values"], a["tail"], a["tau"], a["loss"],
                                  a["state"], None if g is None else ctypes.byref(g), a["ws"],
                                  a["ws_bytes"], None) == code


@pytest.mark.parametrize("kw,code", SHARED + LISTS + [
    (dict(state=None), -1), (dict(grad=None), -1), (dict(grad=grad(g_entropy=FAKE)), -1)] + [
    (dict(grad=g), c) for g, c in GRADS])
def test_topk_distill_grad_refuses(kw, code):
    a = dict(rows=2, V=100, dtype=de.DE_F32, logits=FAKE, ld=100, m=8, ids=FAKE, tau=1.0,
             state=FAKE, grad=grad())
    a.update(kw)
    g = a["grad"]
    assert de.LIB.de_topk_distill_grad(a["rows"], a["V"], a["dtype"], a["logits"], a["ld"], a["m"],
                                       a["ids"], a["tau"], a["state"],
                                       None if g is None else ctypes.byref(g), None) == code


def test_workspace_sizes():
    b = de.de_scores_workspace_bytes
    assert b(0, 100, 0) == 0 and b(1, 0, 0) == 0 and b(1, 100, -1) == 0 and b(1, 100, 129) == 0
    for V in (1, 1000, 102400, 1 << 30):
        assert 0 < b(1, V, 0) <= b(2, V, 0) and b(1, V, 0) <= b(1, V, 128)
    # Scratch for more rows serves fewer, however the rows are split.
    for V in (1000, 9000, 20000, 102400, 260001):
        for m in (0, 5):
            sizes = [b(r, V, m) for r in (1, 2, 5, 9, 17, 40, 64, 79, 100, 155, 300, 2048)]
            assert sizes == sorted(sizes)
    # The scratch is small beside the logits.
    assert b(2048, 102400, 128) < 2048 * 102400 * 4 // 16
