"""Distillation's gradients on the GPU where the list's masses do not sum to one with the
mass beside them, or where the student gives one side of the list nothing.

Tolerances count roundings of u = 2^-24 (half a step of fp32, relative).  A thread adds at
most V / 256 terms one after another (a block of 256 threads holds a whole row; longer rows
take larger blocks or shorter parts), the joins over waves, blocks and parts at most 32 more, and
each batch of 32 or more terms may rescale what came before (9 u): together below V / 128 + 32.
A term's own error is 3 u |d| (its argument: difference, scale, product) and 8 u (the power of
two and two products), and |d| averages at most log V + 1 under the terms' weights.  So a sum is
right to R(V) = (V / 128 + 40 + 4 (log V + 1)) u.  What belongs to the list is in 64 bits.
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
# Whole rows; parts joined by a second launch (two rows of more than 65536: in every form).
SIZES = [300, 9000, 60000, 70001]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


def R(V):
    return (V / 128 + 40 + 4 * (math.log(V) + 1)) * U


def near(got, want, tol, what):
    tol = np.broadcast_to(tol, want.shape)
    with np.errstate(invalid="ignore"):
        ok = (np.isnan(got) & np.isnan(want)) | (got == want) | (np.abs(got - want) <= tol)
    bad = np.argwhere(~ok)[:5]
    assert bad.size == 0, (what, bad.tolist(), got[~ok][:5], want[~ok][:5], tol[~ok][:5])


def tolerances(l, ids, val, tail, tau, g, want, wgrad, dtype):
    """Of one row's loss and of its gradient."""
    V = l.size
    slots = orc.entries(list(ids), V)
    at = [ids[j] for j in slots]
    v = val[slots] if tail else orc.log_softmax(val[slots], tau)
    mass = 1.0 if not tail or not np.isfinite(v).any() else float(np.sum(np.exp(v)))
    total = mass + max(0.0, 1.0 - mass)
    # The logarithms of the sums carry weights of mass and P at most, twice.
    loss_tol = tau * tau * 2 * total * R(V) + 2 * U * abs(np.nan_to_num(want, posinf=0.0))
    if not np.isfinite(wgrad).all():
        return loss_tol, 0.0
    lq = np.maximum(orc.log_softmax(l, tau), -1000.0)
    q = np.exp(lq)
    # q_v W and q_v P / Q each with R(V) and the argument's share; P / Q from the gradient
    # itself.
    both = tau * abs(g) * q * total + np.abs(tau * g * q * total - wgrad)
    tol = both * (R(V) + U * (8 + 3 * np.abs(lq))) + 1e-37
    tol[at] = tau * abs(g) * total * q[at] * R(V) + 4 * U * np.abs(wgrad[at]) + 1e-37
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(wgrad) + tol)
    return loss_tol, tol


def check(x, dtype, ids, val, tail, tau, g, split):
    """Loss and gradient of every row against the oracle; a finite gradient sums to zero."""
    rows, V = x.shape
    m = ids.shape[1]
    t = torch.from_numpy(np.asarray(x, np.float32)).to("cuda").to(dtype)
    held = t.float().cpu().numpy().astype(np.float64)
    loss = torch.full((rows,), 7.0, device="cuda")
    state = torch.full((rows, m + de.DE_DISTILL_STATE), 7.0, device="cuda")
    out = torch.full((rows, V), 3.0, dtype=dtype, device="cuda")
    grad = de.make_row_grad(f32(g), out, V)
    ws = de.scores_workspace(rows, V)
    de.de_topk_distill(rows, V, CODE[dtype], t, V, m, i32(ids), f32(val), tail, tau, loss,
                       state if split else None, None if split else grad, ws)
    if split:
        de.de_topk_distill_grad(rows, V, CODE[dtype], t, V, m, i32(ids), tau, state, grad)
    torch.cuda.synchronize()
    loss, out = loss.cpu().numpy().astype(np.float64), out.float().cpu().numpy().astype(np.float64)
    val = np.asarray(val, np.float32).astype(np.float64)
    tau = float(np.float32(tau))
    for r in range(rows):
        gr = float(np.float32(g[r]))
        want, wgrad = orc.distill(held[r], list(ids[r]), list(val[r]), tail, tau, gr)
        loss_tol, tol = tolerances(held[r], ids[r], val[r], tail, tau, gr, want, wgrad, dtype)
        near(loss[r:r + 1], np.asarray([want]), loss_tol, (r, "loss"))
        if np.isfinite(wgrad).all():
            assert abs(np.sum(out[r])) <= np.sum(tol), (r, np.sum(out[r]), np.sum(tol))
        near(out[r], wgrad, tol, (r, "gradient"))


def teacher(rng, rows, V, m, tau):
    """A student's and a teacher's logits, and the teacher's m best with their log probabilities."""
    t = rng.normal(0, 2, (rows, V))
    for r in range(rows):
        t[r, rng.integers(0, V, 5)] = rng.uniform(6, 14, 5)
    ids = np.argsort(-t, axis=1, kind="stable")[:, :m].astype(np.int32)
    val = np.stack([orc.log_softmax(t[r], tau)[ids[r]] for r in range(rows)])
    return t + rng.normal(0, 0.7, t.shape), ids, val


def with_mass(val, mass):
    return val + np.log(mass / np.sum(np.exp(val)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.0])
@pytest.mark.parametrize("V", SIZES)
def test_lists_of_any_mass(V, tau, split, dtype):
    rng = np.random.default_rng(V)
    m = 40
    x, ids, val = teacher(rng, 7, V, m, tau)
    for r, mass in enumerate((1.27, 1.004, 0.85, 1.3, 0.5)):
        val[r] = with_mass(val[r], mass)
    for r in (2, 3):  # nothing outside the list
        keep = x[r, ids[r]].copy()
        x[r] = -np.inf
        x[r, ids[r]] = keep
    # A stored list in bf16: its masses as they come out.
    val[5] = torch.from_numpy(val[5]).to(torch.bfloat16).double().numpy()
    check(x, dtype, ids, val, 1, tau, np.linspace(0.5, 2.0, 7), split)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("mass", [0.9, 1.0, 1.1])
def test_a_list_of_the_vocabulary_of_any_mass(mass, split, dtype):
    rng = np.random.default_rng(4)
    x, ids, val = teacher(rng, 3, 100, 100, 1.0)
    val = np.stack([with_mass(v, mass) for v in val])
    check(x, dtype, ids, val, 1, 1.0, np.ones(3), split)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("at,tau", [(-1000.0, 1.0), (-30.0, 0.01), (1000.0, 1.0), (0.0, 1.0)])
@pytest.mark.parametrize("V", SIZES)
def test_a_student_that_gives_the_list_nothing(V, at, tau, split, dtype):
    """An infinite loss, or a finite one where the teacher's mass is all outside the list, and
    a finite gradient, wherever the other logits lie."""
    rng = np.random.default_rng(V + 1)
    x, ids, val = teacher(rng, 4, V, 24, 1.0)
    np.put_along_axis(x, ids.astype(np.int64), -np.inf, 1)
    x += at
    ids[1, 3:] = -1
    val[3] = -np.inf
    g = np.linspace(0.5, 2.0, 4)
    check(x, dtype, ids, val, 1, tau, g, split)
    check(x[:3], dtype, ids[:3], val[:3], 0, tau, g[:3], split)


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("V", [300, 9000, 70001])
def test_values_that_are_no_numbers(V, tail, split):
    """A NaN loss and gradient, the tokens that the student gives nothing among them."""
    rng = np.random.default_rng(V + 2)
    x, ids, val = teacher(rng, 6, V, 24, 1.0)
    val[0, 3], val[1, 0], val[2, 5] = np.nan, np.inf, np.nan
    for r in (0, 1, 3):  # nothing outside the list
        keep = x[r, ids[r]].copy()
        x[r] = -np.inf
        x[r, ids[r]] = keep
    val[3] = -np.inf  # no distribution with tail = 0, no entry's mass with tail = 1
    x[4] = -np.inf
    ids[5, 7], val[5, 7] = -1, np.nan  # not an entry
    check(x, torch.float32, ids, val, tail, 1.0, np.linspace(0.5, 2.0, 6), split)
