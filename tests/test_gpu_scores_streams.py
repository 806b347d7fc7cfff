"""Vocabulary calls at once on two streams, each with scratch of its own: the bits of the
calls one after another."""
import numpy as np
import pytest
import torch

import paper_2607_24434_amd as de
from gpu_support import f32, i32, require_gpu
from test_gpu_distill_gradients import CODE, teacher

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    torch.cuda.set_device(0)
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,V", [(5, 1000), (40, 70001), (150, 102400)])
def test_two_streams_at_once(rows, V, dtype):
    m = 20
    rng = np.random.default_rng(V)
    few, ids, val = teacher(rng, 5, V, m, 1.0)
    at = np.arange(rows) % 5
    x = torch.from_numpy(few[at].astype(np.float32)).to("cuda").to(dtype)
    dids, dval, tok = i32(ids[at]), f32(val[at]), i32(rng.integers(0, V, rows))
    g = f32(rng.normal(0, 1, rows))

    def buffers():
        new = lambda *s, dt=torch.float32: torch.full(s, 7, dtype=dt, device="cuda")  # noqa: E731
        return dict(ws=de.scores_workspace(rows, V, m), loss=new(rows), logp=new(rows), stats=new(rows, 4),
                    idx=new(rows, m, dt=torch.int32), top=new(rows, m), d1=new(rows, V, dt=dtype),
                    d2=new(rows, V, dt=dtype))

    def step(b):
        head = (rows, V, CODE[dtype], x, V)
        de.de_token_scores(*head, 1.0, tok, m=m, top_idx=b["idx"], top_logp=b["top"], ws=b["ws"])
        de.de_topk_distill(*head, m, dids, dval, 1, 1.0, b["loss"], grad=de.make_row_grad(g, b["d1"], V), ws=b["ws"])
        de.de_token_scores(*head, 1.0, tok, b["logp"], stats=b["stats"], ws=b["ws"])
        de.de_token_scores_grad(*head, 1.0, tok, b["stats"], de.make_row_grad(g, b["d2"], V))

    want, got, streams = buffers(), [buffers(), buffers()], [torch.cuda.Stream(), torch.cuda.Stream()]
    step(want)
    torch.cuda.synchronize()
    for _ in range(4):
        for b, s in zip(got, streams):
            with torch.cuda.stream(s):
                step(b)
    torch.cuda.synchronize()
    for b in got:
        for k in want:
            if k != "ws":
                assert torch.equal(b[k], want[k]), k
