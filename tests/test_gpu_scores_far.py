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
