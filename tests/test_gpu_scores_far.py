"""Token scores and top-logit distillation over rows more than 2^31 elements apart: every
call with its gradient, in place, where a teacher's list differs from the student's.

Tolerances: R(V) of the sums as in test_gpu_distill_gradients.  A token's gradient is
p = e / s times (g + g_entropy (log p + H)): p is right to R(V) + u (8 + 3 |log p|), the bracket
to 2 R(V) (2 + log V) (two logarithms of sums, and a mean of at most log V) and its own
roundings; the token's own term has four.
"""
import math

import numpy as np
import pytest
import torch

import paper_2607_24434_amd as de
from gpu_support import f32, i32, require_gpu
from oracle import scores as orc
from test_gpu_distill_gradients import CODE, R, U, near, teacher, tolerances

pytestmark = pytest.mark.gpu

ROWS, LD, TAU = 3, (1 << 30) + 8, 1.5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def score_tol(lp, token, g, ge, want, dtype):
    lp = np.maximum(lp, -1000.0)
    p, n = np.exp(lp), math.log(lp.size)
    h = -np.sum(p * lp)
    r = R(lp.size)
    tol = p * (abs(g) + abs(ge) * (np.abs(lp) + h)) * (r + U * (8 + 3 * np.abs(lp)))
    tol += p * abs(ge) * (2 * r * (2 + n) + 4 * U * (np.abs(lp) + h))
    tol[token] += 4 * U * abs(g)
    tol = tol / TAU + 1e-37
    return tol + 2.0 ** -8 * (np.abs(want) + tol) if dtype == torch.bfloat16 else tol


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1500, 70001])
def test_rows_that_start_past_2_to_the_31_elements(V, dtype):
    """Whole rows of one block, and parts joined by a second launch."""
    rng = np.random.default_rng(V)
    m = 20
    x, ids, val = teacher(rng, ROWS, V, m, TAU)
    tokens, g, ge = [V - 1, 0, V // 2], [0.7, -1.2, 1.9], [0.3, 0.5, -0.4]
    big = torch.empty((ROWS - 1) * LD + V, dtype=dtype, device="cuda")
    t = big.as_strided((ROWS, V), (LD, 1))
    near_rows = torch.from_numpy(x.astype(np.float32)).to("cuda").to(dtype)
    held = near_rows.float().cpu().numpy().astype(np.float64)
    val64 = val.astype(np.float32).astype(np.float64)
    dids, dval, tok, gd, ged = i32(ids), f32(val), i32(tokens), f32(g), f32(ge)
    ws = de.scores_workspace(ROWS, V, m)
    head = (ROWS, V, CODE[dtype], big, LD)

    def new(*shape, fill=7.0, dt=torch.float32):
        return torch.full(shape, fill, dtype=dt, device="cuda")

    for split in (False, True):
        t.copy_(near_rows)
        loss, state = new(ROWS), new(ROWS, m + de.DE_DISTILL_STATE)
        grad = de.make_row_grad(gd, big, LD)
        de.de_topk_distill(*head, m, dids, dval, 1, TAU, loss, state if split else None,
                           None if split else grad, ws)
        if split:
            de.de_topk_distill_grad(*head, m, dids, TAU, state, grad)
        loss, out = loss.double().cpu().numpy(), t.float().cpu().numpy().astype(np.float64)
        for r in range(ROWS):
            gr = float(np.float32(g[r]))
            want, wgrad = orc.distill(held[r], list(ids[r]), list(val64[r]), True, TAU, gr)
            loss_tol, tol = tolerances(held[r], ids[r], val64[r], 1, TAU, gr, want, wgrad, dtype)
            assert np.max(np.abs(wgrad)) > 50 * np.max(tol)  # far from a gradient of zeros
            near(loss[r:r + 1], np.asarray([want]), loss_tol, (split, r, "loss"))
            near(out[r], wgrad, tol, (split, r, "distillation"))

    for split in (False, True):
        t.copy_(near_rows)
        logp, ent, st = new(ROWS), new(ROWS), new(ROWS, de.DE_SCORE_STATS)
        grad = de.make_row_grad(gd, big, LD, ged)
        idx, top = new(ROWS, m, fill=-7, dt=torch.int32), new(ROWS, m)
        de.de_token_scores(*head, TAU, tok, m=m, top_idx=idx, top_logp=top, ws=ws)
        de.de_token_scores(*head, TAU, tok, logp, ent, stats=st, grad=None if split else grad, ws=ws)
        if split:
            de.de_token_scores_grad(*head, TAU, tok, st, grad)
        out = t.float().cpu().numpy().astype(np.float64)
        for r in range(ROWS):
            gr, er = float(np.float32(g[r])), float(np.float32(ge[r]))
            lp, h, best, best_lp, wgrad = orc.scores(held[r], TAU, tokens[r], m, gr, er)
            assert idx[r].cpu().tolist() == list(best)
            near(top[r].double().cpu().numpy(), best_lp, R(V) + 4 * U * np.abs(best_lp), (split, r, "best"))
            near(logp[r:r + 1].double().cpu().numpy(), np.asarray([lp]), R(V) + 4 * U * abs(lp), (split, r, "logp"))
            near(ent[r:r + 1].double().cpu().numpy(), np.asarray([h]), 2 * R(V) * (2 + math.log(V)), (split, r, "entropy"))
            tol = score_tol(orc.log_softmax(held[r], TAU), tokens[r], gr, er, wgrad, dtype)
            near(out[r], wgrad, tol, (split, r, "token scores"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_longest_row(dtype):
    """2^30 logits from an odd element on, every call with its gradient in place, against 64
    bits on the GPU.  Parts of 8192 logits at least: a thread adds 64 terms one after another
    and joins at most V / 8192 / 256 parts, each of which may rescale what came before (10 u)."""
    V, m, shift = 1 << 30, 5, 1
    r_sum = (64 + 32 + 10 * V / 8192 / 256 + 40 + 4 * (math.log(V) + 1)) * U
    gen = torch.Generator(device="cuda").manual_seed(5)
    base = torch.empty(shift + V + 1, dtype=dtype, device="cuda").fill_(3.0)
    plain = torch.empty(V, dtype=dtype, device="cuda").normal_(0, 1, generator=gen)
    at, up = [V - 1, 0, (1 << 29) + 3, 77, V - 9000], [24.0, 23.0, 22.0, 21.0, 20.0]
    plain[at] = torch.tensor(up, dtype=dtype, device="cuda")
    x = base[shift:shift + V]
    tok, g, ge = i32([at[2]]), 0.75, -0.5
    ids, val = i32([at]), f32([np.log(np.array([0.4, 0.3, 0.1, 0.05, 0.05]))])
    ws = de.scores_workspace(1, V, m)
    head = (1, V, CODE[dtype], x, V)

    def new(n, fill=7.0, dt=torch.float32):
        return torch.full((n,), fill, dtype=dt, device="cuda")

    z = plain.double()
    log_sum = float(torch.logsumexp(z, 0))
    zp = z.sub(log_sum).exp_()
    entropy = log_sum - float((zp * z).sum())
    del z, zp

    def compare(want_of, tol_of):
        step = 1 << 26
        for i in range(0, V, step):
            lp = plain[i:i + step].double() - log_sum
            p = lp.exp()
            own = [(k, j - i) for k, j in enumerate(at) if i <= j < i + step]
            want, tol = want_of(lp, p, own), tol_of(lp, p, own)
            if dtype == torch.bfloat16:
                tol += 2.0 ** -8 * (want.abs() + tol)
            bad = (x[i:i + step].double() - want).abs() > tol + 1e-37
            assert not bool(bad.any()), (i, int(bad.sum()), int(bad.int().argmax()))
        assert float(base[0]) == 3.0 and float(base[-1]) == 3.0

    def scores_want(lp, p, own):
        out = -p * (g + ge * (lp + entropy))
        for k, j in own:
            out[j] += g if k == 2 else 0.0
        return out

    def scores_tol(lp, p, own):
        out = p * (abs(g) + abs(ge) * (lp.abs() + entropy)) * (r_sum + U * (8 + 3 * lp.abs()))
        out += p * abs(ge) * (2 * r_sum * (2 + math.log(V)) + 4 * U * (lp.abs() + entropy))
        for k, j in own:
            out[j] += 4 * U * abs(g)
        return out

    for split in (False, True):
        x.copy_(plain)
        logp, ent, st, idx, top = new(1), new(1), new(4), new(m, -7, torch.int32), new(m)
        grad = de.make_row_grad(f32([g]), x, V, f32([ge]))
        de.de_token_scores(*head, 1.0, tok, m=m, top_idx=idx, top_logp=top, ws=ws)
        de.de_token_scores(*head, 1.0, tok, logp, ent, stats=st, grad=None if split else grad, ws=ws)
        if split:
            de.de_token_scores_grad(*head, 1.0, tok, st, grad)
        assert idx.tolist() == at
        for k in range(m):
            assert abs(float(top[k]) - (up[k] - log_sum)) <= r_sum + 4 * U * abs(up[k] - log_sum)
        assert abs(float(logp) - (up[2] - log_sum)) <= r_sum + 4 * U * abs(up[2] - log_sum)
        assert abs(float(ent) - entropy) <= 2 * r_sum * (2 + math.log(V))
        compare(scores_want, scores_tol)

    lv = val[0].double()
    pt = 1.0 - float(lv.exp().sum())
    lq = torch.tensor(up, dtype=torch.float64, device="cuda") - log_sum
    qt = 1.0 - float(lq.exp().sum())
    want_loss = float((lv.exp() * (lv - lq)).sum()) + pt * math.log(pt / qt)

    def distill_want(lp, p, own):
        out = p * (1.0 - pt / qt)
        for k, j in own:
            out[j] = p[j] - lv[k].exp()
        return out * g

    def distill_tol(lp, p, own):
        out = p * (1.0 + pt / qt) * (r_sum + U * (8 + 3 * lp.abs()))
        for k, j in own:
            out[j] = p[j] * r_sum + 4 * U * abs(p[j] - lv[k].exp())
        return out * g

    for split in (False, True):
        x.copy_(plain)
        loss, state = new(1), new(m + de.DE_DISTILL_STATE)
        grad = de.make_row_grad(f32([g]), x, V)
        de.de_topk_distill(*head, m, ids, val, 1, 1.0, loss, state if split else None,
                           None if split else grad, ws)
        if split:
            de.de_topk_distill_grad(*head, m, ids, 1.0, state, grad)
        assert abs(float(loss) - want_loss) <= 2 * r_sum + 2 * U * abs(want_loss)
        compare(distill_want, distill_tol)
    torch.cuda.synchronize()
