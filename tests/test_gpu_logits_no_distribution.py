"""GPU: every output of a row without a distribution is no number, in every form that a row may take and wherever what spoils it stands: at a token
of the teacher or at another."""
import numpy as np
import pytest

import oracle
from test_gpu_logits import TYPES, _dev, _host, _logits
from test_gpu_logits_far import STEPS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab", STEPS)
def test_outputs_of_the_distance(gpu_lib, rows, vocab, rest, kind):
    import torch
    q = gpu_lib
    vocab = vocab // 2 if kind == "fp32" else vocab
    x = _logits(rows, vocab, kind, 1)
    tokens = np.tile([5, vocab - 1, 9, -1], (rows, 1)).astype(np.int32)
    teacher = np.log(np.tile([0.3, 0.2, 0.1, 0.1], (rows, 1))).astype(np.float32)
    bad = float("nan"), float("inf")
    for r, (value, at) in enumerate([(v, at) for v in bad for at in (5, vocab - 1, 0)]):
        x[r, at] = value
    x[6] = float("-inf")
    want = oracle.ref_distill(_host(x[:8]), teacher[:8], tokens[:8], rest)
    t, at = _dev(teacher), _dev(tokens, np.int32)
    size = q.quamba_distill_loss_workspace_size(rows, vocab, 4)
    for workspace in (True, False):
        space = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if workspace else None
        for step in (False, True):
            losses, sums, rests = (torch.full((rows,), 7.0, device="cuda") for _ in range(3))
            dx = torch.full_like(x, 3.0) if step else None
            q.quamba_distill_loss(x, t, at, losses, log_sums=sums, log_rests=rests, grad_logits=dx, rest=rest, workspace=space)
            for got, name in ((losses, "losses"), (sums, "log_sums"), (rests, "log_rests")):
                assert np.array_equal(np.isnan(_host(got)[:8]), np.isnan(want[name])), (workspace, step, name, got[:8])
            if not rest:
                assert not rests.any()
            if step:
                assert bool(dx[:7].isnan().all()) and not bool(dx[7:].isnan().any())
    dx = torch.full_like(x, 3.0)
    q.quamba_distill_backward(x, t, at, sums, _dev(np.ones(rows)), dx, log_rests=rests if rest else None, rest=rest)
    assert bool(dx[:7].isnan().all()) and not bool(dx[7:].isnan().any())
