"""Which form takes the sizes of test_gpu_logits_far.py and test_gpu_logits_segments.py (no GPU: planned for 256 compute units)."""
import pytest

import paper_2503_22879_amd as q
from test_logits_plans import ALTERNATIVES, BF16, DISTANCE, F16, F32, MANY, STEP, SUMS, _form, _plan


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


@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_rows_that_are_cut(kind):
    from test_gpu_logits_segments import VOCAB
    for rows in (1, 3, 4, 7, 10):
        for work in (SUMS, 1, ALTERNATIVES, MANY):
            for entropy in (False, True):
                plan = _plan(rows, VOCAB, kind, work, entropy)
                assert plan.segments > 1 and q.quamba_token_logprobs_workspace_size(rows, VOCAB, max(work, 0)) > 0
        for work in (DISTANCE, STEP):
            assert _plan(rows, VOCAB, kind, work).segments > 1
        assert q.quamba_distill_loss_workspace_size(rows, VOCAB, 8) > 16 * rows
    # whole numbers as sums: rows by a wave, by 256 and 1024 threads, in segments
    assert [_plan(r, v, BF16, SUMS).threads for r, v in ((600, 2049), (520, 9001))] == [256, 256]
    if kind != F32:  # held by a wave, and in two passes in segments of the gradient with a row's sum from one workgroup
        assert _form(1100, 2003, kind).threads == 64 and _form(33, 270001, kind).threads == 0
