"""What the projections', the beam selection's and the reordering's entry points refuse, before a device is touched."""
import ctypes as C

import pytest

import paper_2503_22879_amd as q
from paper_2503_22879_amd.binding import _BeamCacheStruct

NULL, SHAPE, WORKSPACE, INVALID = -1, -2, -3, -5


@pytest.fixture
def p():
    room = C.create_string_buffer(256)
    yield C.addressof(room) + (-C.addressof(room) % 16)


def _call(f, good, **change):
    return f(*{**good, **change}.values())


def test_quantize(p):
    f = q.load_library().quamba_fp8_quantize
    good = dict(rows=3, cols=200, block_rows=1, x=p, x_type=0, x_stride=200, q=p, q_stride=200, scales=p, stream=None)
    for name in ("x", "q", "scales"):
        assert _call(f, good, **{name: None}) == NULL
    for bad in (dict(rows=-1), dict(cols=-1), dict(rows=2 ** 31), dict(cols=2 ** 30 + 1, x_stride=2 ** 31, q_stride=2 ** 31),
                dict(x_stride=199), dict(q_stride=199)):
        assert _call(f, good, **bad) == SHAPE
    for bad in (dict(x_type=3), dict(x_type=-1), dict(block_rows=0), dict(block_rows=64), dict(block_rows=-128)):
        assert _call(f, good, **bad) == INVALID
    assert _call(f, good, rows=0, x=None) == 0 and _call(f, good, cols=0, q=None) == 0


def test_matmul(p):
    f = q.load_library().quamba_fp8_matmul
    good = dict(m=3, n=5, k=200, x=p, x_stride=200, xs=p, w=p, w_stride=200, ws=p, y=p, y_type=0, y_stride=5, space=None, bytes=0,
                stream=None)
    for name in ("x", "xs", "w", "ws", "y"):
        assert _call(f, good, **{name: None}) == NULL
    for bad in (dict(m=-1), dict(n=0), dict(k=0), dict(n=-5), dict(k=-1), dict(m=2 ** 31), dict(n=2 ** 31, y_stride=2 ** 32),
                dict(k=2 ** 30 + 1, x_stride=2 ** 31, w_stride=2 ** 31), dict(x_stride=199), dict(w_stride=199), dict(y_stride=4)):
        assert _call(f, good, **bad) == SHAPE
    for bad in (dict(y_type=3), dict(y_type=-1)):
        assert _call(f, good, **bad) == INVALID
    assert _call(f, good, m=0, x=None) == 0
    for sizes in ((-1, 5, 5), (0, 5, 5), (3, 0, 5), (3, 5, 0), (3, 5, 2 ** 31)):
        assert q.quamba_fp8_matmul_workspace_size(*sizes) == 0


def test_every_form_of_the_product_has_a_size_that_is_tested():
    """The form that a size takes, as it is planned without a GPU, for 256 compute units."""
    from test_gpu_fp8 import FORMS

    class Plan(C.Structure):
        _fields_ = [("form", C.c_int), ("splits", C.c_int), ("us", C.c_double)]
    plan = getattr(q.load_library(), "_ZN6quamba15fp8_matmul_planEiiib")      # library-internal
    plan.restype, plan.argtypes = Plan, [C.c_int32] * 3 + [C.c_bool]
    for form, sizes in enumerate(FORMS.values()):
        for m, n, k in sizes:
            got = plan(m, n, -(-k // 128), True)
            assert got.form == form, (m, n, k, got.form)
            size = q.quamba_fp8_matmul_workspace_size(m, n, k)
            assert (size > 0) == (got.splits > 1) and size == (got.splits * m * -(-n // 4) * 16 if size else 0)
            without = plan(m, n, -(-k // 128), False)
            assert without.splits == 1
    assert plan(100, 500, 33, True).splits > 1


def test_every_form_of_the_product_of_unaligned_rows_has_a_size_that_is_tested():
    from test_gpu_fp8 import FORMS, UNALIGNED

    class Plan(C.Structure):
        _fields_ = [("form", C.c_int), ("splits", C.c_int), ("us", C.c_double)]
    plan = getattr(q.load_library(), "_ZN6quamba25fp8_matmul_plan_unalignedEiiii")      # library-internal
    plan.restype, plan.argtypes = Plan, [C.c_int32] * 4
    for form, sizes in UNALIGNED.items():
        for m, n, k in sizes:
            got = plan(m, n, -(-k // 128), 16)
            assert got.form == list(FORMS).index(form), (m, n, k, got.form)
            size = q.quamba_fp8_matmul_workspace_size(m, n, k)
            assert size == (got.splits * m * -(-n // 4) * 16 if got.splits > 1 and k % 16 else size)
            assert plan(m, n, -(-k // 128), 1).splits == 1
    assert plan(100, 500, 33, 16).splits > 1 and plan(100, 500, 33, 2).splits <= 2


def test_select(p):
    f = q.load_library().quamba_beam_select
    size = q.quamba_beam_select_workspace_size(1, 2, 10, 4)
    assert 0 < size
    good = dict(batch=1, beams=2, vocab=10, count=4, logits=p, type=0, stride=10, scores=p, finished=None, pad=0, out=p, parents=p,
                tokens=p, space=p, bytes=size, stream=None)
    for name in ("logits", "scores", "out", "parents", "tokens"):
        assert _call(f, good, **{name: None}) == NULL
    for bad in (dict(batch=-1), dict(beams=0), dict(beams=65), dict(vocab=0), dict(count=0), dict(count=129), dict(stride=9),
                dict(vocab=2 ** 30 + 1, stride=2 ** 31), dict(beams=64, vocab=2 ** 27, stride=2 ** 27), dict(batch=2 ** 30)):
        assert _call(f, good, **bad) == SHAPE
    for bad in (dict(type=3), dict(type=-1), dict(pad=-1), dict(pad=10)):
        assert _call(f, good, **bad) == INVALID
    for bad in (dict(space=None), dict(bytes=size - 1), dict(space=p + 8)):
        assert _call(f, good, **bad) == WORKSPACE
    assert _call(f, good, batch=0, logits=None) == 0
    for sizes in ((1, 65, 10, 4), (1, 2, 0, 4), (1, 2, 10, 129), (-1, 2, 10, 4)):
        assert q.quamba_beam_select_workspace_size(*sizes) == 0


def test_reorder(p):
    f = q.load_library().quamba_beam_reorder
    cache = (_BeamCacheStruct * 2)(_BeamCacheStruct(p, 64), _BeamCacheStruct(p, 64))
    good = dict(batch=1, beams=2, parents=p, n=2, caches=cache, stream=None)
    assert _call(f, good, parents=None) == NULL and _call(f, good, caches=None) == NULL
    for bad in (dict(batch=-1), dict(beams=0), dict(beams=65), dict(n=-1)):
        assert _call(f, good, **bad) == SHAPE
    for c, rc in ((_BeamCacheStruct(p, -1), SHAPE), (_BeamCacheStruct(None, 64), NULL), (_BeamCacheStruct(p, 2 ** 34 + 1), SHAPE)):
        assert _call(f, good, caches=(_BeamCacheStruct * 2)(cache[0], c)) == rc
    assert _call(f, good, batch=0, parents=None) == 0 and _call(f, good, n=0, caches=None) == 0
    # one beam has nowhere to go: nothing is launched
    assert _call(f, good, beams=1) == 0


def test_the_binding_refuses_tensors_of_the_host_and_of_other_kinds():
    import torch
    x, code, scale = torch.zeros(2, 128), torch.zeros(2, 128, dtype=torch.uint8), torch.zeros(2, 1)
    for args in ((x, code, scale), (None, code, scale), (x[0], code, scale), (7, code, scale)):
        with pytest.raises((ValueError, TypeError)):
            q.quamba_fp8_quantize(*args, stream=0)
    with pytest.raises(ValueError):
        q.quamba_fp8_matmul(code, scale, code, scale, x, stream=0)
    with pytest.raises(ValueError):
        q.quamba_beam_select(x, scale, scale, scale, scale, None, stream=0)
    with pytest.raises(ValueError):
        q.quamba_beam_select(torch.zeros(1, 2, 3), scale, scale, scale, scale, None, stream=0)
    with pytest.raises(ValueError):
        q.quamba_beam_reorder(torch.zeros(1, 2, dtype=torch.int32), [x], stream=0)
    with pytest.raises(ValueError):
        q.quamba_beam_reorder(None, [x], stream=0)


@pytest.mark.gpu
def test_the_binding_checks_types_shapes_and_strides(gpu_lib):
    import torch
    dev = dict(device="cuda")
    x, code, scale = torch.zeros(4, 256, **dev), torch.zeros(4, 256, dtype=torch.uint8, **dev), torch.zeros(4, 2, **dev)
    w, ws, y = torch.zeros(8, 256, dtype=torch.uint8, **dev), torch.zeros(1, 2, **dev), torch.zeros(4, 8, **dev)
    gpu_lib.quamba_fp8_quantize(x, code, scale)
    for bad in ((x.double(), code, scale), (x, code.short(), scale), (x, code[:, :200], scale), (x, code, scale[:3]), (x.t(), code.t(), scale),
                (x, code, scale.half()), (x[:1].expand(4, 256), code, scale)):
        with pytest.raises(ValueError):
            gpu_lib.quamba_fp8_quantize(*bad)
    with pytest.raises(gpu_lib.QuambaError) as e:
        gpu_lib.quamba_fp8_quantize(x, code, torch.zeros(1, 2, **dev), block_rows=64)
    assert e.value.status == INVALID
    gpu_lib.quamba_fp8_matmul(code, scale, w, ws, y)
    for bad in ((code, scale, w[:, :128], ws, y), (code, scale[:, :1], w, ws, y), (code, scale, w, ws.t(), y), (code, scale, w, ws, y.t()),
                (code, scale, w, ws, y.int()), (code.char(), scale, w, ws, y), (code, scale, w, ws, y[:, :7])):
        with pytest.raises(ValueError):
            gpu_lib.quamba_fp8_matmul(*bad)
    logits, s, o = torch.zeros(2, 3, 9, **dev), torch.zeros(2, 3, **dev), torch.zeros(2, 3, **dev)
    i = torch.zeros(2, 3, dtype=torch.int32, **dev)
    space = torch.zeros(1 << 16, dtype=torch.uint8, **dev)
    gpu_lib.quamba_beam_select(logits, s, o, i, i.clone(), space)
    for bad in ((logits.double(), s, o, i, i, space), (logits.transpose(0, 1), s, o, i, i, space), (logits, s[:, :2], o, i, i, space),
                (logits, s, o, i.long(), i, space), (logits[:, :, ::2], s, o, i, i, space)):
        with pytest.raises(ValueError):
            gpu_lib.quamba_beam_select(*bad)
    with pytest.raises(gpu_lib.QuambaError) as e:
        gpu_lib.quamba_beam_select(logits, s, o, i, i, None)
    assert e.value.status == WORKSPACE
    for bad in ([s.t()], [logits[:, :2]], [logits[:, :, ::2]], [logits.cpu()], [1], logits):
        with pytest.raises((ValueError, TypeError)):
            gpu_lib.quamba_beam_reorder(i, bad)
