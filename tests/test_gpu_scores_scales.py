"""The vocabulary calls over the temperatures that they accept, and the statistics that they hand
out.  Tolerances: R(V) and the gradients' as in test_gpu_distill_gradients and
test_gpu_scores_far; 1e-37 more (results below fp32's smallest normal value may be flushed)."""
import math

import numpy as np
import pytest
import torch

import paper_2607_24434_amd as de
from gpu_support import f32, i32, require_gpu
from oracle import scores as orc
from test_gpu_distill_gradients import CODE, R, U, near, teacher, tolerances

pytestmark = pytest.mark.gpu

ROWS, M = 3, 20


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def new(*shape, fill=7.0, dt=torch.float32):
    return torch.full(shape, fill, dtype=dt, device="cuda")


def host(t):
    return t.double().cpu().numpy()


def inputs(V, dtype, tau):
    rng = np.random.default_rng(V)
    x, ids, val = teacher(rng, ROWS, V, M, tau)
    t = torch.from_numpy(x.astype(np.float32)).to("cuda").to(dtype)
    return t, host(t), ids, val


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tau", [1e-30, 1e-6, 0.05, 1e6, 1e30])
@pytest.mark.parametrize("V", [1000, 70001])
def test_token_scores_at_any_temperature(V, tau, dtype):
    tau = float(np.float32(tau))
    t, held, _, _ = inputs(V, dtype, 1.0)
    tokens = [int(np.argmax(held[0])), 5, V - 1]
    g = [1.0, -0.5, 2.0]
    logp, ent, st = new(ROWS), new(ROWS), new(ROWS, de.DE_SCORE_STATS)
    idx, top, out = new(ROWS, M, fill=-7, dt=torch.int32), new(ROWS, M), new(ROWS, V, dt=dtype)
    ws = de.scores_workspace(ROWS, V, M)
    head = (ROWS, V, CODE[dtype], t, V, tau, i32(tokens))
    de.de_token_scores(*head, logp, ent, M, idx, top, st, ws=ws)
    de.de_token_scores(*head, grad=de.make_row_grad(f32(g), out, V), ws=ws)
    apart = new(ROWS, V, dt=dtype)
    de.de_token_scores_grad(*head, st, de.make_row_grad(f32(g), apart, V))
    for r in range(ROWS):
        lp, h, best, best_lp, want = orc.scores(held[r], tau, tokens[r], M, g[r], 0.0)
        assert idx[r].cpu().tolist() == list(best)
        near(host(top[r]), best_lp, R(V) + 4 * U * np.abs(best_lp), "best")
        near(host(logp[r:r + 1]), np.asarray([lp]), R(V) + 4 * U * abs(lp), "logp")
        near(host(ent[r:r + 1]), np.asarray([h]), 2 * R(V) * (2 + math.log(V)), "entropy")
        d = (held[r] - held[r].max()) / tau
        s = np.sum(np.exp(d))
        want_st = np.asarray([held[r].max(), s, h, held[r].max() / tau + math.log(s)])
        near(host(st[r]), want_st,
             np.asarray([0.0, s * R(V), 2 * R(V) * (2 + math.log(V)), R(V) + 4 * U * abs(want_st[3])]), "stats")
        full_lp = np.maximum(orc.log_softmax(held[r], tau), -1000.0)
        tol = np.exp(full_lp) * abs(g[r]) * (R(V) + U * (8 + 3 * np.abs(full_lp)))
        tol[tokens[r]] += 4 * U * abs(g[r])
        # A summand e <= 1 below 2^-126, fp32's smallest normal value, is taken as 0, and the sum that
        # divides it is at least 1: p is off by 2^-126 at most, its gradient by |g| / tau times that.
        tol = (tol + 2.0 ** -126 * abs(g[r])) / tau + 1e-37
        if dtype == torch.bfloat16:
            tol += 2.0 ** -8 * (np.abs(want) + tol)
        near(host(out[r]), want, tol, "gradient")
        near(host(apart[r]), want, tol, "gradient apart")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("tau", [1e-30, 1e-6, 0.05, 1e3, 1e15])
@pytest.mark.parametrize("V", [1000, 70001])
def test_distillation_at_any_temperature(V, tau, tail, dtype):
    tau = float(np.float32(tau))
    t, held, ids, val = inputs(V, dtype, tau)
    if not tail:
        val = np.take_along_axis(held, ids.astype(np.int64), 1)
        val = val + np.linspace(-1, 1, M)
    g = [1.0, -0.5, 2.0]
    ws = de.scores_workspace(ROWS, V)
    v64 = val.astype(np.float32).astype(np.float64)
    for split in (False, True):
        loss, state, out = new(ROWS), new(ROWS, M + de.DE_DISTILL_STATE), new(ROWS, V, dt=dtype)
        grad = de.make_row_grad(f32(g), out, V)
        head = (ROWS, V, CODE[dtype], t, V, M, i32(ids))
        de.de_topk_distill(*head, f32(val), tail, tau, loss, state if split else None,
                           None if split else grad, ws)
        if split:
            de.de_topk_distill_grad(*head, tau, state, grad)
        for r in range(ROWS):
            want, wgrad = orc.distill(held[r], list(ids[r]), list(v64[r]), tail, tau, g[r])
            loss_tol, tol = tolerances(held[r], ids[r], v64[r], tail, tau, g[r], want, wgrad, dtype)
            near(host(loss[r:r + 1]), np.asarray([want]), loss_tol + 1e-37, (split, r, "loss"))
            near(host(out[r]), wgrad, tol, (split, r, "gradient"))
