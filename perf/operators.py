"""Timed calls of the row operators over a vocabulary: token scores and distillation
from a teacher's top logits, each with its gradient.

A case is a dict of plain values; ``prepare`` builds what a scoring or training
program holds before the call, ``run`` makes one pass and returns every output,
``exact`` gives the same outputs in 64 bits.  With ``own`` false ``run`` computes the
operators from elementary torch operations in 32 bits.

Kinds:
  scores         ``de_token_scores``: log probabilities of given tokens, entropies and
                 the m best alternatives of every row;
  scores_step    the same without alternatives, then ``de_token_scores_grad`` with the
                 incoming gradients of both: a policy-gradient step, whose weights
                 depend on the log probabilities;
  scores_train   ``de_token_scores`` with its gradient in the same call: a cross
                 entropy, whose weights are known beforehand;
  distill        ``de_topk_distill``: the loss against a teacher's list of m entries a row;
  distill_step   the same, then ``de_topk_distill_grad`` with the loss's incoming gradient;
  distill_train  ``de_topk_distill`` with its gradient in the same call.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
VOCAB = 102400
MOST = 2048 * VOCAB * 4  # bytes of the largest listed logits


def listed():
    return [
        # The smallest call: the five rows of a tiny block. Latency only.
        dict(name="scores-5-tiny", kind="scores", rows=5, vocab=1000, pad=0, dtype="f32", m=5, tau=1.0, masked=0),
        # One decoded token with the alternatives that a serving interface shows.
        dict(name="scores-1", kind="scores", rows=1, vocab=VOCAB, pad=0, dtype="f32", m=20, tau=1.0, masked=0),
        # The positions of a long verify block (16 drafts).
        dict(name="scores-17", kind="scores", rows=17, vocab=VOCAB, pad=0, dtype="f32", m=20, tau=0.7, masked=0),
        # A prompt's log probabilities, or a teacher's lists for distillation: the largest
        # scoring call, over a vocabulary whose last entries are padding.
        dict(name="scores-2048", kind="scores", rows=2048, vocab=VOCAB, pad=0, dtype="f32", m=64, tau=1.0, masked=400),
        # bf16 logits of an odd vocabulary: rows that start at any 2-byte boundary.
        dict(name="scores-1000-bf16-odd", kind="scores", rows=1000, vocab=50001, pad=0, dtype="bf16", m=50, tau=1.0, masked=0),
        # A policy-gradient step over sampled tokens, with an entropy bonus.
        dict(name="scores-step-512", kind="scores_step", rows=512, vocab=VOCAB, pad=0, dtype="f32", m=0, tau=1.0, masked=0),
        # The token term of a training batch (cross entropy) on bf16 logits.
        dict(name="scores-train-2048-bf16", kind="scores_train", rows=2048, vocab=VOCAB, pad=0, dtype="bf16", m=0, tau=1.0, masked=0),
        # The divergence of a block's positions, as a signal: no gradient.
        dict(name="distill-32", kind="distill", rows=32, vocab=VOCAB, pad=0, dtype="f32", m=16, tau=2.0, masked=0, tail=False),
        # The smallest training call.
        dict(name="distill-train-5-tiny", kind="distill_train", rows=5, vocab=1000, pad=0, dtype="f32", m=8, tau=1.0, masked=0, tail=True),
        # A training batch against stored lists of 64 log probabilities and the mass beside them.
        dict(name="distill-train-1024", kind="distill_train", rows=1024, vocab=VOCAB, pad=0, dtype="f32", m=64, tau=1.0, masked=400, tail=True),
        # The same in bf16, long lists, an odd vocabulary in padded rows.
        dict(name="distill-train-2048-bf16", kind="distill_train", rows=2048, vocab=65537, pad=7, dtype="bf16", m=128, tau=2.0, masked=0, tail=False),
        # Loss and gradient as two calls, the loss's weight known only in between.
        dict(name="distill-step-333-bf16", kind="distill_step", rows=333, vocab=32000, pad=0, dtype="bf16", m=32, tau=1.0, masked=0, tail=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["scores", "scores", "scores_step", "scores_train", "distill", "distill_step", "distill_train"])
    dtype = rng.choice(["f32", "bf16"])
    vocab = _log(rng, 1000, 152064)
    if rng.random() < 0.5:
        vocab = max(1000, vocab // 64 * 64)
    rows = min(_log(rng, 1, 2048), MOST // (vocab * 4 * (1 if kind in ("scores", "distill") else 2)))
    c = dict(kind=kind, rows=rows, vocab=vocab, pad=rng.choice([0, 0, 0, 1, 8, 61]), dtype=dtype,
             tau=rng.choice([1.0, 1.0, 0.7, 1.3, 2.0]), masked=rng.choice([0, 0, vocab // 200]))
    if kind.startswith("distill"):
        return dict(c, m=_log(rng, 1, 128), tail=rng.random() < 0.5)
    return dict(c, m=_log(rng, 1, 128) if kind == "scores" else 0)


# ---------------------------------------------------------------- inputs


def _logits(case, gen):
    """Rows as a language model's head gives them: a broad bulk and a few likely tokens."""
    rows, vocab, ld = case["rows"], case["vocab"], case["vocab"] + case["pad"]
    x = torch.empty(rows, ld, device="cuda").normal_(0.0, 2.0, generator=gen)
    at = torch.randint(vocab - case["masked"], (rows, 12), generator=gen, device="cuda")
    up = torch.empty(rows, 12, device="cuda").uniform_(4.0, 14.0, generator=gen)
    x.scatter_reduce_(1, at, up, "amax")
    if case["masked"]:
        x[:, vocab - case["masked"]:vocab] = -math.inf
    return x, at


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 17)
    rows, vocab, m, kind = case["rows"], case["vocab"], case["m"], case["kind"]
    ld, dt = vocab + case["pad"], DTYPES[case["dtype"]]
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    teacher, likely = _logits(case, gen)
    s = dict(case, ld=ld)
    if kind.startswith("distill"):
        # The teacher's stored list: its m best entries' log probabilities at the loss's
        # temperature (what de_token_scores gives), or their plain logits; a tenth of the
        # lists end early (id -1).
        t = teacher[:, :vocab] / case["tau"]
        ids = t.topk(m, dim=1).indices
        val = t.gather(1, ids) - t.logsumexp(1, keepdim=True) if case["tail"] else teacher.gather(1, ids)
        short = torch.rand(rows, 1, generator=gen, device="cuda") < 0.1
        ends = torch.randint(1, m + 1, (rows, 1), generator=gen, device="cuda")
        ids = ids.int().masked_fill_(short & (torch.arange(m, device="cuda") >= ends), -1)
        noise = torch.empty(rows, ld, device="cuda").normal_(0.0, 0.7, generator=gen)
        s.update(ids=ids.contiguous(), values=val.contiguous(), logits=(teacher + noise).to(dt),
                 loss=new(rows), state=new(rows, m + 4))
    else:
        # Half the tokens are likely ones, one row in ten has none (padding).
        tok = torch.randint(vocab - case["masked"], (rows,), generator=gen, device="cuda")
        tok = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.5, likely[:, 0], tok)
        tok[torch.rand(rows, generator=gen, device="cuda") < 0.1] = -1
        s.update(tokens=tok.int(), logits=teacher.to(dt), logp=new(rows), entropy=new(rows), stats=new(rows, 4),
                 top_idx=new(rows, max(m, 1), dtype=torch.int32), top_logp=new(rows, max(m, 1)))
    if kind.endswith(("step", "train")):
        g = torch.empty(rows, device="cuda").normal_(0.0, 1.0, generator=gen)
        s.update(g=g if kind == "scores_step" else (g.abs() + 0.5) * (-1.0 if kind == "scores_train" else 1.0),
                 g_entropy=torch.full((rows,), 0.01, device="cuda") if kind == "scores_step" else None,
                 dlogits=new(rows, ld, dtype=dt))
    if own:  # the kernels' scratch, which a program allocates once; the inputs are the same without it
        import paper_2607_24434_amd as de
        s["ws"] = de.scores_workspace(rows, vocab, m if kind == "scores" else 0)
    return s


# ---------------------------------------------------------------- the calls


def _run_own(s):
    import paper_2607_24434_amd as de
    rows, vocab, m, kind = s["rows"], s["vocab"], s["m"], s["kind"]
    head = (rows, vocab, de.DE_F32 if s["dtype"] == "f32" else de.DE_BF16, s["logits"], s["ld"])
    grad = de.make_row_grad(s["g"], s["dlogits"], s["ld"], s.get("g_entropy")) if "g" in s else None
    if kind == "scores":
        de.de_token_scores(*head, s["tau"], s["tokens"], s["logp"], s["entropy"], m, s["top_idx"], s["top_logp"], ws=s["ws"])
        return s["logp"], s["entropy"], s["top_idx"], s["top_logp"]
    if kind == "scores_step":
        de.de_token_scores(*head, s["tau"], s["tokens"], s["logp"], s["entropy"], stats=s["stats"], ws=s["ws"])
        de.de_token_scores_grad(*head, s["tau"], s["tokens"], s["stats"], grad)
        return s["logp"], s["entropy"], s["dlogits"][:, :vocab]
    if kind == "scores_train":
        de.de_token_scores(*head, s["tau"], s["tokens"], s["logp"], s["entropy"], grad=grad, ws=s["ws"])
        return s["logp"], s["entropy"], s["dlogits"][:, :vocab]
    entries = (m, s["ids"], s["values"], s["tail"], s["tau"])
    if kind == "distill":
        de.de_topk_distill(*head, *entries, s["loss"], ws=s["ws"])
        return (s["loss"],)
    if kind == "distill_step":
        de.de_topk_distill(*head, *entries, s["loss"], state=s["state"], ws=s["ws"])
        de.de_topk_distill_grad(*head, m, s["ids"], s["tau"], s["state"], grad)
    else:
        de.de_topk_distill(*head, *entries, s["loss"], grad=grad, ws=s["ws"])
    return s["loss"], s["dlogits"][:, :vocab]


def _scores(s):
    z = s["logits"][:, :s["vocab"]].float()
    top = z.max(1, keepdim=True).values
    d = (z - top) / s["tau"]
    e = d.exp()
    total = e.sum(1, keepdim=True)
    log_total = total.log()
    entropy = log_total - (e * d.clamp(min=-1e4)).sum(1, keepdim=True) / total
    tok = s["tokens"].long()[:, None]
    there = tok >= 0
    logp = torch.where(there, d.gather(1, tok.clamp(min=0)) - log_total, 0.0)
    out = [logp[:, 0], entropy[:, 0]]
    if s["m"]:
        # The best m, ties to the lowest index: one whole number orders value and index.
        bits = (z + 0.0).view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32
        key = key | (0xFFFFFFFF - torch.arange(s["vocab"], device=z.device))
        idx = 0xFFFFFFFF - (key.topk(s["m"], dim=1).values & 0xFFFFFFFF)
        out += [idx.int(), d.gather(1, idx) - log_total]
    if "g" in s:
        p = e / total
        g = torch.where(there[:, 0], s["g"], 0.0)[:, None]
        dz = -g * p
        if s["g_entropy"] is not None:
            dz -= s["g_entropy"][:, None] * p * (d.clamp(min=-1e4) - log_total + entropy)
        dz.scatter_add_(1, tok.clamp(min=0), g)
        out.append((dz / s["tau"]).to(s["logits"].dtype))
    return tuple(out)


def _distill(s):
    tau, ids, val = s["tau"], s["ids"].long(), s["values"].double()
    z = s["logits"][:, :s["vocab"]].float()
    there = ids >= 0
    at = ids.clamp(min=0)
    top = z.max(1, keepdim=True).values
    e = ((z - top) / tau).exp()
    total = e.sum(1, keepdim=True)
    # What belongs to the list is in 64 bits: a loss is a small difference of its terms.
    logq = (z.gather(1, at).double() - top) / tau - total.double().log()
    if s["tail"]:
        # The masses outside the list; the student's is summed without the list's entries.
        logp = torch.where(there, val, -math.inf)
        p_tail = (1.0 - logp.exp().sum(1, keepdim=True)).clamp(min=0.0)
        where = torch.where(there, at, s["vocab"])
        mark = torch.zeros(z.shape[0], s["vocab"] + 1, dtype=torch.bool, device=z.device).scatter_(1, where, True)
        rest = torch.where(mark[:, :-1], -math.inf, z)
        rest_top = rest.max(1, keepdim=True).values
        rest_sum = ((rest - rest_top) / tau).exp().sum(1, keepdim=True).double()
        log_tail = (rest_top.double() - top) / tau + rest_sum.log() - total.double().log()
    else:
        logp = torch.where(there, val / tau, -math.inf)
        logp = logp - logp.max(1, keepdim=True).values
        logp = logp - logp.exp().sum(1, keepdim=True).log()
    p = logp.exp()
    loss = torch.where(p > 0, p * (logp - logq), 0.0).sum(1, keepdim=True)
    keep = 1.0
    if s["tail"]:
        loss = loss + torch.where(p_tail > 0, p_tail * (p_tail.log() - log_tail), 0.0)
        keep = (1.0 - p_tail / log_tail.exp()).float()
    loss = (tau * tau * loss)[:, 0].float()
    if "g" not in s:
        return (loss,)
    dz = e / total * keep
    # An entry's own gradient in place of what the tokens outside the list get; a slot
    # without an entry (id -1) writes to a column of its own.
    dz = torch.cat([dz, torch.zeros_like(top)], 1)
    dz.scatter_(1, torch.where(there, at, s["vocab"]), (logq.exp() - p).float())
    return loss, (dz[:, :-1] * (s["g"][:, None] * tau)).to(s["logits"].dtype)


def run(s):
    if own:
        return _run_own(s)
    return _distill(s) if s["kind"].startswith("distill") else _scores(s)


def work(case):
    elems = case["rows"] * case["vocab"]
    size = 4 if case["dtype"] == "f32" else 2
    grad = case["kind"].endswith(("step", "train"))
    listed_bytes = case["rows"] * (case["m"] * 8 + 24)
    # Difference, scale, exponential, sum; an entropy's product; a gradient's two products.
    per = 4 + (2 if case["kind"].startswith("scores") else 0) + (3 if grad else 0)
    return {"bytes": elems * size * (2 if grad else 1) + listed_bytes, "flops": elems * per}


# ---------------------------------------------------------------- 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    tau = s["tau"]
    lp = torch.log_softmax(s["logits"][:, :s["vocab"]].double() / tau, 1)
    p = lp.exp()
    if not s["kind"].startswith("distill"):
        h = -torch.special.xlogy(p, p).sum(1)
        tok = s["tokens"].long()
        real = tok >= 0
        pick = tok.clamp(min=0)[:, None]
        out = [torch.where(real, lp.gather(1, pick)[:, 0], 0.0), h]
        if s["m"]:
            out += [None, lp.topk(s["m"], dim=1).values]
        if "g" in s:
            # d logp / dz = [v = token] - p; d H / dz = -p (log p + H)
            g = s["g"].double() * real
            dz = torch.zeros_like(p).scatter_(1, pick, g[:, None]) - p * g[:, None]
            if s["g_entropy"] is not None:
                dz -= s["g_entropy"].double()[:, None] * (torch.special.xlogy(p, p) + p * h[:, None])
            out.append(dz / tau)
        return tuple(out)
    rows, vocab = p.shape
    dist = torch.zeros(rows, vocab + 1, dtype=torch.float64, device=p.device)  # the last column: no entry
    slot = torch.where(s["ids"] >= 0, s["ids"].long(), vocab)
    dist.scatter_(1, slot, s["values"].double().exp() if s["tail"] else 1.0)
    member = torch.zeros_like(dist, dtype=torch.bool).scatter_(1, slot, True)[:, :vocab]
    dist = dist[:, :vocab]
    if not s["tail"]:
        raw = torch.zeros(rows, vocab + 1, dtype=torch.float64, device=p.device)
        raw = raw.scatter_(1, slot, s["values"].double())[:, :vocab]
        dist = torch.softmax(torch.where(member, raw / tau, -math.inf), 1)
    loss = (torch.special.xlogy(dist, dist) - torch.where(dist > 0, dist * lp, 0.0)).sum(1)
    ratio = torch.zeros(rows, dtype=torch.float64, device=p.device)
    if s["tail"]:
        rest = (1.0 - dist.sum(1)).clamp(min=0.0)
        mass = torch.where(member, 0.0, p).sum(1)
        loss += torch.special.xlogy(rest, rest / mass)
        ratio = rest / mass
    # Inside the list q - p; outside q (1 - teacher's mass there / student's mass there).
    dz = torch.where(member, p - dist, p * (1.0 - ratio[:, None]))
    loss = loss * tau * tau
    if "g" not in s:
        return (loss,)
    return loss, dz * (s["g"].double()[:, None] * tau)
