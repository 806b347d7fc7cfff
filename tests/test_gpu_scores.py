"""Token scores and top-logit distillation on the GPU against the fp64 oracle.

Tolerances count roundings of u = 2^-24 (a half step of fp32, relative).  A term
exp((l - max) / tau) has its argument's three roundings, (3 u |d| absolute, |d| the scaled
difference) and the exponential's (4 u); terms of weight p have |d| <= log V + log(1 / p) on
average at most log V + 1; a sum over V terms of one thread in 1024 adds V / 1024 + 32
roundings.  So a sum's relative error is at most R(V) = (V / 1024 + 40 + 4 (log V + 1)) u.
"""
import math

import numpy as np
import pytest
import torch

import paper_2607_24434_amd as de
from gpu_support import f32, i32, require_gpu
from oracle import scores as orc

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
CODE = {torch.float32: de.DE_F32, torch.bfloat16: de.DE_BF16}
DTYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def R(V):
    return (V / 1024 + 40 + 4 * (math.log(V) + 1)) * U


def full(*shape, value=float("nan"), dtype=torch.float32):
    return torch.full(shape, value, dtype=dtype, device="cuda")


def placed(x, dtype, pad=0, shift=0):
    """The rows x [rows, V] on the GPU with `pad` more columns, `shift` elements into an
    allocation: (tensor, ld, the values as they are held)."""
    rows, V = x.shape
    ld = V + pad
    base = full(shift + rows * ld, value=7.0, dtype=dtype)
    t = base[shift:].view(rows, ld)
    t[:, :V] = torch.from_numpy(np.asarray(x, np.float32)).to("cuda").to(dtype)
    return t, ld, t[:, :V].float().cpu().numpy().astype(np.float64)


def near(got, want, tol):
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else np.asarray(got)
    want, tol = np.asarray(want, np.float64), np.broadcast_to(tol, np.shape(want))
    assert got.shape == want.shape
    same = np.isnan(got) & np.isnan(want)
    fin = np.isfinite(want)
    same |= ~fin & (got == want)
    with np.errstate(invalid="ignore"):
        same |= fin & (np.abs(got - want) <= tol)
    bad = np.argwhere(~same)
    assert bad.size == 0, (bad[:5].tolist(), got[~same][:5], want[~same][:5], tol[~same][:5])


def looked_at(rows):
    """The rows that are compared: all of a few, else a dozen over them."""
    return range(rows) if rows <= 16 else sorted({0, 1, rows // 2, rows - 2, rows - 1, *range(5, rows, rows // 7)})


def logits(rng, rows, V):
    # Many rows share 17 rows' noise and differ in their likely tokens.
    x = rng.normal(0, 2, (min(rows, 17), V))[np.arange(rows) % 17]
    for r in range(rows):
        at = rng.integers(0, V, 5)
        x[r, at] = rng.uniform(3, 12, 5)
    return x


def grad_tol(V, want, l, tau, token, g, ge, dtype):
    """Of one row's gradient: p (its relative error with |d|'s share) times what multiplies
    it, the token's own term, and the stored type's rounding."""
    l = np.where(np.isnan(l), -np.inf, l)
    lp = np.maximum(orc.log_softmax(l, tau), -1000.0)
    p, h = np.exp(lp), abs(-np.sum(np.exp(lp) * lp))
    g = g if token >= 0 else 0.0
    rel = R(V) + 8 * U * (np.abs(lp) + math.log(V))
    tol = p * (abs(g) + abs(ge) * (np.abs(lp) + h)) * 2 * rel + p * abs(ge) * 2 * R(V) * (2 + math.log(V))
    if 0 <= token < V:
        tol[token] += 4 * U * abs(g)
    tol = tol / tau + 1e-37
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    return np.nan_to_num(tol)


def run_scores(x, dtype, tau, tokens, m, pad=0, shift=0, g=None, ge=None, split=False,
               in_place=False):
    rows, V = x.shape
    t, ld, held = placed(x, dtype, pad, shift)
    tok = i32(tokens)
    logp, ent, st = full(rows), full(rows), full(rows, de.DE_SCORE_STATS)
    idx, tlp = full(rows, max(m, 1), value=-7, dtype=torch.int32), full(rows, max(m, 1))
    out, grad = None, None
    ws = de.scores_workspace(rows, V, m)
    if g is not None or ge is not None:
        out = t if in_place else full(rows, ld, value=3.0, dtype=dtype)
        grad = de.make_row_grad(None if g is None else f32(g), out, ld,
                                None if ge is None else f32(ge))
    de.de_token_scores(rows, V, CODE[dtype], t, ld, tau, tok, logp, ent, m,
                       idx if m else None, tlp if m else None, st, None if split else grad, ws)
    if split:
        de.de_token_scores_grad(rows, V, CODE[dtype], t, ld, tau, tok, st, grad)
    torch.cuda.synchronize()
    return held, logp, ent, idx, tlp, st, out


def check_scores(x, dtype, tau, tokens, m, g=None, ge=None, **kw):
    rows, V = x.shape
    held, logp, ent, idx, tlp, st, out = run_scores(x, dtype, tau, tokens, m, g=g, ge=ge, **kw)
    for r in looked_at(rows):
        gr, er = 0.0 if g is None else float(g[r]), 0.0 if ge is None else float(ge[r])
        lp, h, top, top_lp, grad = orc.scores(held[r], tau, int(tokens[r]), m, gr, er)
        near(logp[r:r + 1], [lp], [R(V) + 4 * U * abs(np.nan_to_num(lp, posinf=0, neginf=0))])
        # The mean scaled difference is at most log V, as is the logarithm of the sum.
        near(ent[r:r + 1], [h], [2 * R(V) * (2 + math.log(V))])
        if m:
            assert idx[r].cpu().tolist() == list(top)
            near(tlp[r], top_lp, R(V) + 4 * U * np.abs(np.nan_to_num(top_lp, posinf=0, neginf=0)))
        if out is not None:
            near(out[r, :V], grad, grad_tol(V, np.nan_to_num(grad), held[r], tau, int(tokens[r]),
                                            gr, er, dtype) if np.isfinite(grad).all() else 0.0)
            assert bool((out[r, V:] == (7.0 if kw.get("in_place") else 3.0)).all())
    return st


SIZES = [1, 2, 7, 64, 65, 1000, 1003, 4096, 4097, 8191, 8192, 8193, 16384, 16385, 32000, 50001,
         102400]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", SIZES)
def test_scores(V, dtype):
    rng = np.random.default_rng(V)
    rows = 3
    m = min(V, [1, 20, 64, 128][V % 4])
    tokens = rng.integers(0, V, rows)
    tokens[1] = -1
    check_scores(logits(rng, rows, V), dtype, [1.0, 0.7, 2.3][V % 3], tokens, m, pad=V % 5,
                 shift=V % 3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shift", [0, 1, 2, 3, 5, 7])
@pytest.mark.parametrize("V", [1001, 20003])
def test_rows_at_any_element(V, shift, dtype):
    rng = np.random.default_rng(shift)
    check_scores(logits(rng, 5, V), dtype, 1.0, rng.integers(0, V, 5), 33, pad=1, shift=shift)
    check_scores(logits(rng, 5, V), dtype, 1.0, rng.integers(0, V, 5), 0, pad=1, shift=shift,
                 g=rng.normal(0, 1, 5), ge=rng.normal(0, 1, 5))


def shapes(V):
    """Rows whose order is not that of noise."""
    v = np.arange(V, dtype=np.float64)
    rng = np.random.default_rng(5)
    x = rng.normal(0, 2, V)
    rows = dict(
        up=v / V * 8, down=-v / V * 8, equal=np.full(V, 0.25), signed_zero=np.where(v % 3 == 0, 0.0, -0.0),
        two=np.where(v % 1000 == 999, 3.0, 1.0), steps=np.round(x), far=x + 30000.0,
        spike=np.where(v == V // 2, 500.0, x), few=np.where(v % 977 == 5, x, -np.inf),
        one=np.where(v == V - 1, 1.0, -np.inf), nan=np.where(v % 11 == 3, np.nan, x),
        nan_only=np.where(v == 4, 1.0, np.nan), lowest=np.where(v % 5 == 0, x, np.finfo(np.float32).min),
        block=np.where(v < 300, 5 + x * 0.01, x), wide=x * 1e30)
    return rows


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,m", [(1000, 128), (5000, 20), (9000, 1), (40000, 128), (102401, 64), (260001, 128)])
def test_orders_ties_and_masked_logits(V, m, dtype):
    rows = shapes(V)
    x = np.stack(list(rows.values()))
    tokens = [(37 * i) % V for i in range(len(rows))]
    check_scores(x, dtype, 1.0, tokens, m)
    n = len(rows)
    check_scores(x, dtype, 1.0, tokens, 0, g=np.linspace(-1, 1, n), ge=np.linspace(0.5, 1, n))


@pytest.mark.parametrize("bits,dtype", [(0x7F800001, torch.float32), (-0x7EDCBB, torch.float32),
                                        (0x7F81, torch.bfloat16), (-0x7E, torch.bfloat16)])
@pytest.mark.parametrize("V", [900, 30000])
def test_a_nan_of_any_bits_counts_as_minus_infinity(V, bits, dtype):
    """Signalling NaNs too, which memory that nothing wrote may hold; a loss shows them."""
    rng = np.random.default_rng(V)
    rows, m = 3, 40
    x = torch.from_numpy(logits(rng, rows, V)).to("cuda").to(dtype)
    plain = x.clone()
    at = torch.from_numpy(rng.permutation(V)[:V // 3]).to("cuda")
    x.view(torch.int32 if dtype == torch.float32 else torch.int16)[:, at] = bits
    assert bool(torch.isnan(x[:, at]).all())
    plain[:, at] = float("-inf")
    got = []
    for t in (x, plain):
        idx, tlp, logp, ent = full(rows, m, value=-7, dtype=torch.int32), full(rows, m), full(rows), full(rows)
        d = full(rows, V, dtype=dtype)
        ws = de.scores_workspace(rows, V, m)
        tok = i32([0, 1, 2])
        de.de_token_scores(rows, V, CODE[dtype], t, V, 1.0, tok, logp, ent, m, idx, tlp, ws=ws)
        de.de_token_scores(rows, V, CODE[dtype], t, V, 1.0, tok, logp,
                           grad=de.make_row_grad(f32(np.ones(rows)), d, V), ws=ws)
        got.append((idx, tlp, logp, ent, d))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    loss, d = full(rows, value=0.0), full(rows, V, value=0.0, dtype=dtype)
    de.de_topk_distill(rows, V, CODE[dtype], x, V, m, idx, tlp, 1, 1.0, loss,
                       grad=de.make_row_grad(f32(np.ones(rows)), d, V), ws=ws)
    assert bool(torch.isnan(loss).all()) and bool(torch.isnan(d).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [5, 3000, 50000])
def test_rows_without_a_distribution(V, dtype):
    x = np.zeros((5, V))
    x[0] = -np.inf
    x[1, 2] = np.inf
    x[2] = np.nan
    x[3, 1:] = -np.inf
    x[4, 3] = -np.inf
    tokens = [0, 1, 2, 1, V]  # row 3: a token of probability 0; row 4: an id outside
    check_scores(x, dtype, 1.0, tokens, min(V, 9))
    check_scores(x, dtype, 1.0, tokens, 0, g=np.ones(5), ge=np.ones(5))
    # Weights of zero, and rows without a token, whatever the logits are.
    check_scores(x, dtype, 1.0, [-1] * 5, 0, g=np.ones(5))
    check_scores(x, dtype, 1.0, tokens, 0, g=np.zeros(5), ge=np.zeros(5))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("rows,V", [(1, 1), (4, 1000), (3, 8200), (2, 50001), (300, 2049),
                                    (260, 20011), (130, 32769), (130, 65536), (129, 102397),
                                    (128, 102400), (3, 70001), (100, 102409)])
def test_scores_gradient(rows, V, in_place, split, dtype):
    rng = np.random.default_rng(rows + V)
    tokens = rng.integers(-1, V, rows)
    g, ge = rng.normal(0, 1, rows), rng.normal(0, 0.3, rows)
    g[rows // 2] = 0.0
    x = logits(rng, rows, V)
    check_scores(x, dtype, 0.8, tokens, 0, g=g, ge=ge, pad=3, split=split, in_place=in_place)
    check_scores(x, dtype, 1.0, tokens, 0, g=g, pad=3, split=split, in_place=in_place)
    check_scores(x, dtype, 1.0, tokens, 0, ge=ge, pad=3, split=split, in_place=in_place)


# ---------------------------------------------------------------- distillation


def lists(rng, t, m, tail, tau, ragged=True):
    """A teacher's lists from its logits t [rows, V]: the best m, some rows shorter, one with
    a repeated id and one with ids outside the vocabulary."""
    rows, V = t.shape
    ids = np.full((rows, m), -1, np.int32)
    val = np.full((rows, m), 9.0, np.float32)
    for r in range(rows):
        n = min(m, V)
        top = np.argsort(-t[r], kind="stable")[:n]
        ids[r, :n] = top
        val[r, :n] = orc.log_softmax(t[r], tau)[top] if tail else t[r][top]
        if ragged and r % 4 == 1:
            ids[r, n // 2:] = -1
        if ragged and r % 4 == 2 and n > 2:
            ids[r, n - 1] = ids[r, 0]
            ids[r, n // 2] = V + r
    return ids, val


def run_distill(x, dtype, ids, val, tail, tau, g=None, pad=0, shift=0, split=False,
                in_place=False):
    rows, V = x.shape
    m = ids.shape[1]
    t, ld, held = placed(x, dtype, pad, shift)
    loss, state = full(rows), full(rows, m + de.DE_DISTILL_STATE)
    di, dv = i32(ids), f32(val)
    out, grad = None, None
    ws = de.scores_workspace(rows, V)
    if g is not None:
        out = t if in_place else full(rows, ld, value=3.0, dtype=dtype)
        grad = de.make_row_grad(f32(g), out, ld)
    de.de_topk_distill(rows, V, CODE[dtype], t, ld, m, di, dv, tail, tau, loss,
                       state if split else None, None if split else grad, ws)
    if split:
        de.de_topk_distill_grad(rows, V, CODE[dtype], t, ld, m, di, tau, state, grad)
    torch.cuda.synchronize()
    return held, loss, out


def check_distill(x, dtype, ids, val, tail, tau, g=None, **kw):
    rows, V = x.shape
    held, loss, out = run_distill(x, dtype, ids, val, tail, tau, g, **kw)
    val = np.asarray(val, np.float32).astype(np.float64)
    for r in looked_at(rows):
        gr = 1.0 if g is None else float(np.float32(g[r]))
        want, grad = orc.distill(held[r], list(ids[r]), list(val[r]), tail, tau, gr)
        # Two logarithms of sums, weighted by at most one each; the rest is in 64 bits.
        near(loss[r:r + 1], [want], [2 * tau * tau * R(V) + 2 * U * abs(np.nan_to_num(want, posinf=0))])
        if out is None:
            continue
        tol = 0.0
        if np.isfinite(grad).all() and np.any(grad):
            lq = np.maximum(orc.log_softmax(held[r], tau), -1000.0)
            q = np.exp(lq)
            # q_v and q_v P / Q each with R(V) and their argument's share; P / Q from the
            # gradient itself: |grad| <= g tau (q_v + q_v P / Q).
            both = q * abs(gr) * tau + np.abs(q * gr * tau - grad)
            slots = [ids[r][j] for j in orc.entries(list(ids[r]), V)]
            tol = both * (2 * R(V) + 8 * U * (np.abs(lq) + math.log(V))) + 1e-37
            tol[slots] = (2 * R(V) * q[slots] + 8 * U * both[slots] / (abs(gr) * tau)) * abs(gr) * tau + 1e-37
            if dtype == torch.bfloat16:
                tol = tol + 2.0 ** -8 * (np.abs(grad) + tol)
        near(out[r, :V], grad, tol)
        assert bool((out[r, V:] == (7.0 if kw.get("in_place") else 3.0)).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", SIZES)
def test_distill(V, tail, dtype):
    rng = np.random.default_rng(V + 1)
    rows, m, tau = 5, [1, 16, 63, 128][V % 4], [1.0, 2.0, 0.7][V % 3]
    t = logits(rng, rows, V)
    ids, val = lists(rng, t, m, tail, tau)
    check_distill(t + rng.normal(0, 0.7, t.shape), dtype, ids, val, tail, tau,
                  g=rng.normal(0, 1, rows), pad=V % 5, shift=V % 3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("rows,V,m", [(1, 1, 1), (5, 1000, 8), (3, 8200, 64), (2, 50001, 128),
                                      (300, 2049, 5), (260, 20011, 33), (130, 32769, 128),
                                      (130, 65536, 9), (129, 102397, 100), (128, 102400, 64),
                                      (3, 70001, 128), (100, 102409, 20)])
def test_distill_gradient(rows, V, m, in_place, split, dtype):
    rng = np.random.default_rng(rows + V)
    t = logits(rng, rows, V)
    for tail in (False, True):
        ids, val = lists(rng, t, m, tail, 1.5)
        g = rng.normal(0, 1, rows)
        g[rows // 2] = 0.0
        check_distill(t + rng.normal(0, 0.7, t.shape), dtype, ids, val, tail, 1.5, g=g, pad=3,
                      split=split, in_place=in_place)


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [40, 9000, 60000])
def test_distill_edges(V, tail, split):
    rng = np.random.default_rng(9)
    m = 40
    t = np.broadcast_to(logits(rng, 1, V), (12, V)).copy()
    ids, val = lists(rng, t, m, tail, 1.0, ragged=False)
    ids, val = ids.copy(), val.copy()
    x = t + rng.normal(0, 0.5, t.shape)
    ids[0] = -1                                  # no entry
    ids[1] = V                                   # none either
    x[1] = np.nan                                # ... whatever the logits
    x[2, 30] = np.nan
    x[3, 31] = np.inf
    x[4, ids[4, 3]] = -np.inf                    # an entry with no probability
    val[5, 2] = -np.inf                          # a teacher's zero
    x[6, [v for v in range(V) if v not in set(ids[6])]] = -np.inf  # nothing outside the list
    x[7] = -np.inf
    val[8, 1] = np.nan
    ids[9, 1:] = ids[9, 0]                       # one entry, repeated
    ids[10, :] = ids[10, ::-1].copy()            # a list in another order
    val[10, :] = val[10, ::-1].copy()
    x[11] = x[11] * 40                           # almost all mass on one token
    for g in (np.linspace(0.5, 2, 12), np.zeros(12)):
        check_distill(x, torch.float32, ids, val, tail, 1.0, g=g, split=split)


def test_a_list_of_the_whole_vocabulary_has_no_tail():
    rng = np.random.default_rng(4)
    t = logits(rng, 3, 100)
    ids, val = lists(rng, t, 128, True, 1.0, ragged=False)
    check_distill(t + rng.normal(0, 1, t.shape), torch.float32, ids, val, True, 1.0, g=np.ones(3))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,V", [(4, 1003), (3, 20000), (2, 80001)])
def test_gradients_at_other_elements_than_the_logits(rows, V, dtype):
    """dlogits with a row length and a start of its own: the same gradient to the bit."""
    rng = np.random.default_rng(V)
    t, ld, _ = placed(logits(rng, rows, V), dtype, 3, 1)
    tok, g = i32(rng.integers(0, V, rows)), f32(rng.normal(0, 1, rows))
    ids, val = lists(rng, t[:, :V].float().cpu().numpy(), 17, True, 1.0)
    ws = de.scores_workspace(rows, V)
    got = []
    for pad, shift in ((3, 1), (6, 3), (0, 0)):
        base = full(rows * (V + pad) + shift, value=3.0, dtype=dtype)
        out = base[shift:].view(rows, V + pad)
        grad = de.make_row_grad(g, out, V + pad)
        de.de_token_scores(rows, V, CODE[dtype], t, ld, 1.0, tok, grad=grad, ws=ws)
        a = out[:, :V].clone()
        de.de_topk_distill(rows, V, CODE[dtype], t, ld, 17, i32(ids), f32(val), 1, 1.0, full(rows),
                           grad=grad, ws=ws)
        got.append((a, out[:, :V].clone()))
        assert bool((out[:, V:] == 3.0).all()) and bool((base[:shift] == 3.0).all())
    for a, b in got[1:]:
        assert torch.equal(a, got[0][0]) and torch.equal(b, got[0][1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 7, 100, 600])
@pytest.mark.parametrize("V", [1, 2047, 8190, 8192, 8194, 16384, 16390, 32766, 65537])
def test_nothing_past_the_scratch(V, rows, dtype):
    """The calls' scratch is all that they use of it, rows at whole slots and at any element."""
    m, guard = min(V, 11), 4096
    base = torch.randn(rows * (V + 1) + 8, device="cuda").to(dtype)
    tok = torch.zeros(rows, dtype=torch.int32, device="cuda")
    g = torch.ones(rows, device="cuda")
    d = full(rows, V, dtype=dtype)
    for shift, ld in ((0, (V + 7) // 8 * 8 if rows * ((V + 7) // 8 * 8) <= base.numel() else V), (1, V + 1)):
        t = base[shift:]
        for k in (m, 0):
            n = de.de_scores_workspace_bytes(rows, V, k)
            ws = torch.full((n + guard,), 171, dtype=torch.uint8, device="cuda")
            args = (rows, V, CODE[dtype], t, ld)
            grad = de.make_row_grad(g, d, V)
            idx, tlp = full(rows, m, value=-7, dtype=torch.int32), full(rows, m)
            if k:
                de.de_token_scores(*args, 1.0, tok, full(rows), m=k, top_idx=idx, top_logp=tlp, ws=ws[:n])
                assert int(idx.min()) >= 0 and int(idx.max()) < V
            else:
                de.de_token_scores(*args, 1.0, tok, full(rows), grad=grad, ws=ws[:n])
                de.de_topk_distill(*args, m, idx.clamp(min=0), tlp, 0, 1.0, full(rows), grad=grad, ws=ws[:n])
            assert bool((ws[n:] == 171).all())


@pytest.mark.parametrize("rows,V,m", [(200000, 7, 3), (1 << 20, 1, 1), (70001, 130, 20),
                                      (2, 20000003, 128)])
def test_many_rows_and_long_ones(rows, V, m):
    """Against 64 bits on the GPU: more rows than a grid's other dimensions take, and a row of
    twenty million."""
    gen = torch.Generator(device="cuda").manual_seed(V)
    x = torch.empty(rows, V, device="cuda").normal_(0, 3, generator=gen)
    tok = torch.randint(V, (rows,), generator=gen, device="cuda").int()
    g = torch.empty(rows, device="cuda").normal_(generator=gen)
    idx, tlp, logp, ent = full(rows, m, value=-7, dtype=torch.int32), full(rows, m), full(rows), full(rows)
    d, loss, dl = full(rows, V), full(rows), full(rows, V)
    ws = de.scores_workspace(rows, V, m)
    de.de_token_scores(rows, V, de.DE_F32, x, V, 1.0, tok, logp, ent, m, idx, tlp, ws=ws)
    de.de_token_scores(rows, V, de.DE_F32, x, V, 1.0, tok, grad=de.make_row_grad(g, d, V), ws=ws)
    lp = torch.log_softmax(x.double(), 1)
    p = lp.exp()
    want = lp.gather(1, tok.long()[:, None])[:, 0]
    assert bool(((logp - want).abs() <= R(V) + 4 * U * want.abs()).all())
    assert bool(((ent + (p * lp).sum(1)).abs() <= 2 * R(V) * (2 + math.log(V))).all())
    best = lp.topk(m, 1)
    assert bool(((tlp - best.values).abs() <= R(V) + 4 * U * best.values.abs()).all())
    assert torch.equal(x.gather(1, idx.long()), x.gather(1, best.indices))
    assert m == 1 or bool(((tlp[:, 1:] < tlp[:, :-1]) | (idx[:, 1:] != idx[:, :-1])).all())
    want = -p * g[:, None].double()
    want.scatter_add_(1, tok.long()[:, None], g.double()[:, None])
    # p's error, with its argument's share, and the token's own rounding.
    tol = p * g.abs()[:, None] * (2 * R(V) + 8 * U * (lp.abs() + math.log(V))) + 1e-37
    tol.scatter_add_(1, tok.long()[:, None], 4 * U * g.abs().double()[:, None])
    assert bool(((d - want).abs() <= tol).all())
    # Distillation towards the row's own best entries: p = q / (1 - Q), loss -log(1 - Q).
    de.de_topk_distill(rows, V, de.DE_F32, x, V, m, idx, x.gather(1, idx.long()), 0, 1.0, loss,
                       grad=de.make_row_grad(g, dl, V), ws=ws)
    mass = p.gather(1, idx.long()).sum(1, keepdim=True)
    assert bool(((loss + mass[:, 0].log()).abs() <= 2 * R(V) + 2 * U * mass[:, 0].log().abs()).all())
    dist = torch.zeros_like(p).scatter_(1, idx.long(), p.gather(1, idx.long()) / mass)
    want = (p - dist) * g[:, None].double()
    tol = (p + dist) * g.abs()[:, None] * (2 * R(V) + 8 * U * (lp.abs() + math.log(V))) + 1e-37
    assert bool(((dl - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_offsets_beyond_32_bits(dtype):
    """Rows 2^30 + 8 elements apart: the last one starts past 2^31 elements."""
    rng = np.random.default_rng(6)
    rows, V, m, ld = 3, 1500, 12, (1 << 30) + 8
    x = logits(rng, rows, V)
    big = torch.empty((rows - 1) * ld + V, dtype=dtype, device="cuda")
    t = big.as_strided((rows, V), (ld, 1))
    t.copy_(torch.from_numpy(x).to("cuda").to(dtype))
    held = t.float().cpu().numpy().astype(np.float64)
    tok = i32([5, 6, 7])
    logp, idx, tlp, st = full(rows), full(rows, m, value=-7, dtype=torch.int32), full(rows, m), full(rows, 4)
    ws = de.scores_workspace(rows, V, m)
    de.de_token_scores(rows, V, CODE[dtype], big, ld, 1.0, tok, logp, None, m, idx, tlp, st, ws=ws)
    for r in range(rows):
        lp, _, top, _, _ = orc.scores(held[r], 1.0, 5 + r, m)
        assert idx[r].cpu().tolist() == list(top)
        near(logp[r:r + 1], [lp], [R(V) + 4 * U * abs(lp)])
    # The gradient in place.
    loss = full(rows)
    de.de_topk_distill(rows, V, CODE[dtype], big, ld, m, idx, tlp, 1, 1.0, loss,
                       grad=de.make_row_grad(f32(np.ones(rows)), big, ld), ws=ws)
    assert float(loss.abs().max()) <= 2 * R(V) + 1e-6
    # A teacher's own list: P = Q and p = q up to the list's own rounding.
    assert float(t.float().abs().max()) <= 1e-5
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,V", [(2, 1000), (9, 102400), (300, 20000)])
def test_the_same_bits_whatever_the_scratch_holds(rows, V, dtype):
    rng = np.random.default_rng(8)
    m = 32
    t = torch.from_numpy(logits(rng, rows, V)).to("cuda").to(dtype)
    tok = i32(rng.integers(0, V, rows))
    ws = de.scores_workspace(rows, V, m)
    got = []
    for fill in (0, 255, 17):
        ws.fill_(fill)
        idx, tlp, logp, ent = full(rows, m, value=-7, dtype=torch.int32), full(rows, m), full(rows), full(rows)
        de.de_token_scores(rows, V, CODE[dtype], t, V, 1.0, tok, logp, ent, m, idx, tlp, ws=ws)
        ws.fill_(fill)
        loss, d = full(rows), full(rows, V, dtype=dtype)
        de.de_topk_distill(rows, V, CODE[dtype], t * 0.9, V, m, idx, tlp, 1, 1.0, loss,
                           grad=de.make_row_grad(logp, d, V), ws=ws)
        got.append([v.clone() for v in (idx, tlp, logp, ent, loss, d)])
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("rows,V", [(4, 1000), (9, 102400), (300, 9000)])
def test_captured_and_replayed(rows, V):
    """A graph of all four calls, replayed with new logits between eager calls."""
    rng = np.random.default_rng(10)
    m = 24
    t = torch.empty(rows, V, device="cuda")
    s = torch.empty(rows, V, device="cuda")
    tok = i32(rng.integers(0, V, rows))
    g = f32(rng.normal(0, 1, rows))

    def buffers():
        return dict(idx=full(rows, m, value=-7, dtype=torch.int32), tlp=full(rows, m), logp=full(rows),
                    stats=full(rows, 4), loss=full(rows), d1=full(rows, V), d2=full(rows, V),
                    ws=de.scores_workspace(rows, V, m))

    def step(b):
        de.de_token_scores(rows, V, de.DE_F32, t, V, 1.0, tok, None, None, m, b["idx"], b["tlp"], ws=b["ws"])
        de.de_topk_distill(rows, V, de.DE_F32, s, V, m, b["idx"], b["tlp"], 1, 1.0, b["loss"],
                           grad=de.make_row_grad(g, b["d1"], V), ws=b["ws"])
        de.de_token_scores(rows, V, de.DE_F32, s, V, 1.0, tok, b["logp"], stats=b["stats"], ws=b["ws"])
        de.de_token_scores_grad(rows, V, de.DE_F32, s, V, 1.0, tok, b["stats"],
                                de.make_row_grad(g, b["d2"], V))

    def fill(seed):
        x = logits(np.random.default_rng(seed), rows, V).astype(np.float32)
        t.copy_(torch.from_numpy(x))
        s.copy_(t * 0.8)

    fill(0)
    a, b = buffers(), buffers()
    step(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    for seed in range(1, 5):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        step(b)
        for k in a:
            if k != "ws":
                assert torch.equal(a[k], b[k]), (seed, k)


def test_on_another_stream():
    rng = np.random.default_rng(12)
    rows, V, m = 6, 30000, 10
    t = torch.from_numpy(logits(rng, rows, V).astype(np.float32)).to("cuda")
    tok = i32(rng.integers(0, V, rows))
    torch.cuda.synchronize()
    want, got = None, None
    for stream in (None, torch.cuda.Stream()):
        idx, tlp, logp = full(rows, m, value=-7, dtype=torch.int32), full(rows, m), full(rows)
        ws = de.scores_workspace(rows, V, m)
        torch.cuda.synchronize()
        de.de_token_scores(rows, V, de.DE_F32, t, V, 1.0, tok, logp, None, m, idx, tlp, ws=ws, stream=stream)
        torch.cuda.synchronize()
        want, got = got, (idx, tlp, logp)
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_a_teacher_and_a_drafter_together():
    """The set as it is used: a stack's target logits give the stored lists, the drafter's
    logits their loss and gradient, the token term its own; each against the oracle."""
    from test_gpu_distill import TINY, _device_model
    from workloads import gen
    dm = _device_model(TINY, 8)
    T, V, m, tau = 8, TINY.vocab, 20, 1.5
    toks = i32([gen.start_token(TINY, redraw=r) for r in range(T)])
    lt, ld = full(T, V), full(T, V)
    amax = full(T, value=-7, dtype=torch.int32)
    dm.forward(toks, de.DE_TARGET, lt, amax)
    dm.forward(toks, de.DE_DRAFT, ld)
    idx, tlp = full(T, m, value=-7, dtype=torch.int32), full(T, m)
    loss, logp, d1, d2 = full(T), full(T), full(T, V), full(T, V)
    ws = de.scores_workspace(T, V, m)
    de.de_token_scores(T, V, de.DE_F32, lt, V, tau, m=m, top_idx=idx, top_logp=tlp, ws=ws)
    de.de_topk_distill(T, V, de.DE_F32, ld, V, m, idx, tlp, 1, tau, loss,
                       grad=de.make_row_grad(f32(np.ones(T)), d1, V), ws=ws)
    de.de_token_scores(T, V, de.DE_F32, ld, V, 1.0, amax, logp,
                       grad=de.make_row_grad(f32(-np.ones(T)), d2, V), ws=ws)
    assert torch.equal(idx[:, 0], amax)
    # Eq. 9's term and the divergences of the same rows, from the row call.
    kl, ce = full(T), full(T)
    de.de_row_kl(T, V, lt, V, ld, V, None, False, tau, kl, ce)
    near(-logp, ce.double().cpu().numpy(), 1e-6 + 1e-4 * np.abs(ce.cpu().numpy()))
    # Lumping the tokens outside the list never adds divergence (1e-4: the row call's own).
    assert bool((loss <= kl * (1 + 1e-4) + 1e-5).all())
    a, b = lt.double().cpu().numpy(), ld.double().cpu().numpy()
    ids, val = idx.cpu().numpy(), tlp.double().cpu().numpy()
    for r in range(T):
        want, grad = orc.distill(b[r], list(ids[r]), list(val[r]), True, tau)
        near(loss[r:r + 1], [want], [2 * tau * tau * R(V) + 2 * U * abs(want)])
        near(d1[r], grad, 4 * R(V) * tau * (np.exp(orc.log_softmax(b[r], tau)) * 20 + np.abs(grad)) + 1e-12)
        lp, _, _, _, grad = orc.scores(b[r], 1.0, int(amax[r]), 0, -1.0)
        near(logp[r:r + 1], [lp], [R(V) + 4 * U * abs(lp)])
        near(d2[r], grad, grad_tol(V, grad, b[r], 1.0, int(amax[r]), -1.0, 0.0, torch.float32))
