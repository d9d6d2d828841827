"""How rows of logits are cut and which kernels take them, by the library's own arithmetic (no GPU: planned for 256 compute units)."""
import ctypes as C
import itertools

import pytest

import paper_2503_22879_amd as q

F32, F16, BF16 = range(3)
SUMS, ALTERNATIVES, MANY, DISTANCE, STEP = 0, 8, 128, -1, -2      # so many alternatives, or a distance, alone and with its gradient


class Plan(C.Structure):
    _fields_ = [("threads", C.c_int), ("segments", C.c_int), ("vectors", C.c_int)]


def _internal(name, restype, *argtypes):
    f = getattr(q.load_library(), name)      # library-internal
    f.restype, f.argtypes = restype, argtypes
    return f


def _plan(rows, vocab, kind, work, entropy=False, workspace=True):
    f = _internal("_ZN6quamba11logits_planEliiNS_10LogitsWorkEibb", Plan, C.c_int64, C.c_int32, C.c_int32, C.c_int, C.c_int32, C.c_bool, C.c_bool)
    return f(rows, vocab, kind, max(-work, 0), max(work, 0), entropy, workspace)


def _form(rows, vocab, kind, rest=False, in_place=False, workspace=True):
    f = _internal("_ZN6quamba12distill_formEliibbb", Plan, C.c_int64, C.c_int32, C.c_int32, C.c_bool, C.c_bool, C.c_bool)
    return f(rows, vocab, kind, rest, in_place, workspace)


def _vectors(vocab, kind):
    """16-byte pieces that a row touches at most, wherever it begins."""
    return (vocab + 2 * (4 if kind == F32 else 8) - 2) // (4 if kind == F32 else 8)


ROWS = [1, 2, 5, 31, 32, 33, 64, 65, 256, 257, 1000, 4096, 100000, 1 << 22, 1 << 31]
VOCABS = [1, 7, 8, 9, 500, 1025, 2048, 4100, 16000, 32768, 50021, 60001, 65536, 100001, 131072, 200000, 1 << 20, (1 << 26) - 1, 1 << 26]


@pytest.mark.parametrize("kind", [F32, F16, BF16])
@pytest.mark.parametrize("work", [SUMS, ALTERNATIVES, MANY, DISTANCE, STEP])
def test_segments_hold_the_whole_row(work, kind):
    for rows in ROWS:
        for vocab in VOCABS:
            size = (q.quamba_distill_loss_workspace_size(rows, vocab, 8) if work < 0
                    else q.quamba_token_logprobs_workspace_size(rows, vocab, work))
            for entropy in (False, True):
                assert _plan(rows, vocab, kind, work, entropy, False).segments == 1     # they need a place to meet
                plan = _plan(rows, vocab, kind, work, entropy)
                assert plan.threads in (64, 256, 1024)
                if plan.segments == 1:
                    assert plan.vectors == 0
                else:
                    assert plan.segments <= 256 and plan.threads == 256
                    assert plan.segments * plan.vectors >= _vectors(vocab, kind) > (plan.segments - 1) * plan.vectors
                    assert size >= rows * plan.segments * (16 + 8 * max(work, 0))
                if work < 0:
                    assert size >= 16 * rows * plan.segments
                if plan.threads == 64:
                    assert _vectors(vocab, kind) <= 8 * 64


@pytest.mark.parametrize("vectors", [256, 768])
@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_a_gradients_segments_hold_the_whole_row(kind, vectors):
    f = _internal("_ZN6quamba13gradient_planEiii", Plan, C.c_int32, C.c_int32, C.c_int)
    for vocab in VOCABS:
        plan = f(vocab, kind, vectors)
        assert plan.threads == 256 and plan.vectors <= vectors
        assert plan.segments * plan.vectors >= _vectors(vocab, kind) > (plan.segments - 1) * plan.vectors
        assert plan.segments <= 1 << 22      # a launch takes a row's


@pytest.mark.parametrize("kind", [F32, F16, BF16])
def test_a_row_in_registers_is_all_there(kind):
    """A thread has room for its vectors (16 in registers, as many again are read twice), and the row a vector that lies inside it wherever
    it begins."""
    for rows in ROWS:
        for vocab in VOCABS:
            for rest, in_place, workspace in itertools.product((False, True), repeat=3):
                form = _form(rows, vocab, kind, rest, in_place, workspace)
                if form.threads:
                    assert _vectors(vocab, kind) <= form.threads * form.vectors and vocab >= (8 if kind == F32 else 16)
                    assert form.segments == 1 and form.vectors in (4, 8, 16, 32)
                    assert _plan(rows, vocab, kind, DISTANCE if in_place else STEP, False, workspace).segments == 1


def test_each_form_has_a_size_that_is_tested():
    from test_gpu_logits import HELD
    forms = {}
    for kind in (F32, BF16):
        for rest in (False, True):
            of = [_form(rows, vocab // 2 if kind == F32 else vocab, kind, rest) for rows, vocab in HELD]
            forms[kind, rest] = [(form.threads, form.vectors) for form in of]
    want = [(64, 4), (64, 4), (256, 4), (512, 4), (512, 8), (512, 16), (1024, 16), (1024, 32), (1024, 32), (0, 0)]
    assert forms[F32, False] == forms[F32, True] == want + [(512, 16), (1024, 16)]
    assert forms[BF16, False] == want + [(0, 0), (0, 0)]
    want[6] = (512, 32)
    assert forms[BF16, True] == want + [(0, 0), (0, 0)]
    assert all(_plan(r, v, BF16, STEP).segments > 1 for r, v in HELD[-2:])
    # sums, alternatives and distances by 64, 256 and 1024 threads and in segments: of test_logprobs and test_distill
    assert {_plan(r, v, BF16, SUMS).threads for r, v in ((3, 7), (3, 40000), (700, 52001))} == {64, 256, 1024}
    assert {_plan(r, v, BF16, ALTERNATIVES).threads for r, v in ((5, 33), (33, 4099), (4, 90001))} == {64, 256, 1024}
    assert all(_plan(2, 300001, k, w).segments > 1 for k in (F32, F16, BF16) for w in (SUMS, ALTERNATIVES, DISTANCE, STEP))
