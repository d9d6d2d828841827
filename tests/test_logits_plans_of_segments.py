"""Which form takes the sizes of test_gpu_logits_far.py (no GPU: planned for 256 compute units)."""
import pytest

import paper_2503_22879_amd as q
from test_logits_plans import ALTERNATIVES, BF16, DISTANCE, F32, STEP, SUMS, _form, _plan


def test_logits_far_from_0():
    from test_gpu_logits_far import FORMS, STEPS
    for kind in (F32, BF16):
        for work in (SUMS, ALTERNATIVES):
            plans = [_plan(rows, vocab, kind, work) for rows, vocab in FORMS]
            assert [p.threads for p in plans[:3]] == [64, 256, 1024] and plans[4].threads == 256 and plans[4].segments == 1
            assert plans[3].segments > 1
        forms = [_form(rows, vocab // 2 if kind == F32 else vocab, kind) for rows, vocab in STEPS]
        want = [(64, 4), (256, 4), (512, 4), (512, 8), (512, 16), (1024, 16), (1024, 32), (0, 0), (0, 0)]
        assert [(f.threads, f.vectors) for f in forms] == want
    assert (_form(72, 130001, BF16, True).threads, _form(72, 130001, BF16, True).vectors) == (512, 32)
    for rows, vocab in STEPS[-1:]:
        assert _plan(rows, vocab, BF16, STEP).segments > 1 and _plan(rows, vocab, BF16, DISTANCE).segments > 1
        assert q.quamba_distill_loss_workspace_size(rows, vocab, 6) > 16 * rows
