"""What the entry points over rows of logits refuse, before a device is touched."""
import ctypes as C

import pytest

import paper_2503_22879_amd as q

NULL, SHAPE, INVALID = -1, -2, -5


@pytest.fixture
def p():
    room = C.create_string_buffer(4096)
    yield C.addressof(room) + (-C.addressof(room) % 16)


def _call(f, good, **change):
    return f(*{**good, **change}.values())


BAD_ROWS = (dict(rows=-1), dict(rows=2 ** 31 + 1), dict(vocab=0), dict(vocab=-4), dict(vocab=2 ** 26 + 1, stride=2 ** 27), dict(stride=9),
            dict(stride=2 ** 40 + 1), dict(rows=2 ** 20, stride=2 ** 27), dict(rows=2 ** 31, stride=2 ** 40))
BAD_VALUES = (dict(type=3), dict(type=-1), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")),
              dict(temperature=float("inf")), dict(temperature=2.0 ** -101), dict(temperature=2.0 ** 101))


def test_token_logprobs(p):
    f = q.load_library().quamba_token_logprobs
    good = dict(rows=3, vocab=10, logits=p, type=0, stride=10, temperature=1.0, targets=p, logprobs=p, log_sums=p, entropies=p, count=4,
                top=p, tokens=p, space=None, bytes=0, stream=None)
    for name in ("logits", "targets", "logprobs", "top", "tokens"):  # one of targets and logprobs without the other
        assert _call(f, good, **{name: None}) == NULL
    for bad in BAD_ROWS + (dict(count=-1), dict(count=129)):
        assert _call(f, good, **bad) == SHAPE
    for bad in BAD_VALUES + (dict(logits=p + 2), dict(logits=p + 1, type=1)):
        assert _call(f, good, **bad) == INVALID
    assert _call(f, good, rows=0, logits=None) == 0
    # nothing is asked for
    assert _call(f, good, targets=None, logprobs=None, log_sums=None, entropies=None, count=0, top=None, tokens=None) == 0
    for sizes in ((-1, 10, 4), (3, 0, 4), (3, 2 ** 26 + 1, 4), (3, 10, 129), (3, 10, -1)):
        assert q.quamba_token_logprobs_workspace_size(*sizes) == 0
    assert q.quamba_token_logprobs_workspace_size(1, 128000, 8) > 0 and q.quamba_token_logprobs_workspace_size(100000, 128000, 8) == 0


def test_token_logprobs_backward(p):
    f = q.load_library().quamba_token_logprobs_backward
    good = dict(rows=3, vocab=10, logits=p, type=0, stride=10, temperature=1.0, targets=p, log_sums=p, entropies=p, grad_logprobs=p,
                grad_entropies=p, grad=p + 2048, grad_stride=10, stream=None)
    for name in ("logits", "log_sums", "entropies", "grad_logprobs", "grad_entropies", "grad", "targets"):
        assert _call(f, good, **{name: None}) == NULL
    for bad in BAD_ROWS + (dict(grad_stride=9), dict(grad_stride=2 ** 40 + 1)):
        assert _call(f, good, **bad) == SHAPE
    for bad in BAD_VALUES + (dict(logits=p + 2), dict(grad=p + 2049)):
        assert _call(f, good, **bad) == INVALID
    # a gradient that lies on other logits than its own
    for bad in (dict(grad=p + 4), dict(grad=p + 40), dict(grad=p + 116), dict(grad=p, grad_stride=11), dict(stride=20, grad_stride=20, grad=p + 36),
                dict(stride=19, grad_stride=19, grad=p + 40), dict(stride=20, grad_stride=21, grad=p + 40), dict(logits=p + 64, grad=p + 24)):
        assert _call(f, good, **bad) == INVALID
    assert _call(f, good, rows=0, logits=None, grad=None) == 0


def test_distill(p):
    f = q.load_library().quamba_distill_loss
    good = dict(rows=3, vocab=10, logits=p, type=0, stride=10, temperature=1.0, places=4, teacher=p, tokens=p, rest=0, weights=None, losses=p,
                log_sums=None, log_rests=None, grad=p + 2048, grad_stride=10, space=None, bytes=0, stream=None)
    for name in ("logits", "teacher", "tokens", "losses"):
        assert _call(f, good, **{name: None}) == NULL
    for bad in BAD_ROWS + (dict(places=0), dict(places=129), dict(places=-1), dict(grad_stride=9)):
        assert _call(f, good, **bad) == SHAPE
    for bad in BAD_VALUES + (dict(logits=p + 2), dict(grad=p + 2049), dict(grad=p + 4), dict(rest=2), dict(rest=-1)):
        assert _call(f, good, **bad) == INVALID
    assert _call(f, good, rows=0, logits=None) == 0
    for sizes in ((-1, 10, 4), (3, 0, 4), (3, 10, 0), (3, 10, 129)):
        assert q.quamba_distill_loss_workspace_size(*sizes) == 0
    g = q.load_library().quamba_distill_backward
    good = dict(rows=3, vocab=10, logits=p, type=0, stride=10, temperature=1.0, places=4, teacher=p, tokens=p, rest=1, log_sums=p, log_rests=p,
                grad_losses=p, grad=p + 2048, grad_stride=10, stream=None)
    for name in ("logits", "teacher", "tokens", "log_sums", "log_rests", "grad_losses", "grad"):
        assert _call(g, good, **{name: None}) == NULL
    for bad in BAD_ROWS + (dict(places=0), dict(places=129), dict(grad_stride=9)):
        assert _call(g, good, **bad) == SHAPE
    for bad in BAD_VALUES + (dict(grad=p + 4), dict(rest=2)):
        assert _call(g, good, **bad) == INVALID
    assert _call(g, good, rows=0, grad=None) == 0


def test_the_binding_refuses_tensors_of_the_host():
    import torch
    x, row, tokens = torch.zeros(2, 9), torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: q.quamba_token_logprobs(x, tokens, row, stream=0), lambda: q.quamba_token_logprobs_backward(x, tokens, row, row, x, stream=0),
                 lambda: q.quamba_distill_loss(x, x, tokens, row, stream=0), lambda: q.quamba_distill_backward(x, x, tokens, row, row, x, stream=0)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_the_binding_checks_types_shapes_and_strides(gpu_lib):
    import torch
    q = gpu_lib
    dev = dict(device="cuda")
    x, row, i, top = torch.zeros(4, 9, **dev), torch.zeros(4, **dev), torch.zeros(4, dtype=torch.int32, **dev), torch.zeros(4, 3, **dev)
    tokens = torch.zeros(4, 3, dtype=torch.int32, **dev)
    q.quamba_token_logprobs(x, i, row, top_logprobs=top, top_tokens=tokens)
    for bad in (dict(logits=x.double()), dict(logits=x.t()), dict(logits=x[:, ::2]), dict(logits=x[:1].expand(4, 9)), dict(logits=x[0]),
                dict(logits=x.cpu()), dict(targets=i.long()), dict(targets=i[:3]), dict(logprobs=row.half()), dict(log_sums=row[:2]),
                dict(entropies=row.cpu()), dict(top_tokens=tokens.long()), dict(top_logprobs=top[:, :2]), dict(top_tokens=tokens[0]),
                dict(workspace=torch.zeros(9))):
        with pytest.raises(ValueError):
            q.quamba_token_logprobs(**{**dict(logits=x, targets=i, logprobs=row, top_logprobs=top, top_tokens=tokens), **bad})
    for bad in (dict(top_tokens=None, top_logprobs=top), dict(targets=None), dict(logprobs=None)):
        with pytest.raises(q.QuambaError) as e:
            q.quamba_token_logprobs(**{**dict(logits=x, targets=i, logprobs=row), **bad})
        assert e.value.status == NULL
    with pytest.raises(TypeError):
        q.quamba_token_logprobs(x, i, row, temperature="hot")
    dx = torch.zeros_like(x)
    good = dict(logits=x, targets=i, log_sums=row, grad_logprobs=row, grad_logits=dx)
    q.quamba_token_logprobs_backward(**good)
    for bad in (dict(grad_logits=dx.half()), dict(grad_logits=dx[:, :8]), dict(grad_logits=None), dict(grad_logits=dx.cpu()), dict(log_sums=row[:1]),
                dict(entropies=row.half())):
        with pytest.raises(ValueError):
            q.quamba_token_logprobs_backward(**{**good, **bad})
    good = dict(logits=x, teacher=top, teacher_tokens=tokens, losses=row)
    q.quamba_distill_loss(**good)
    for bad in (dict(teacher=top.half()), dict(teacher=None), dict(teacher=row), dict(teacher_tokens=tokens.long()), dict(teacher_tokens=tokens[:, :2]),
                dict(losses=row[:2]), dict(weights=row.double()), dict(grad_logits=dx.half()), dict(grad_logits=dx[:2]), dict(log_rests=row.cpu())):
        with pytest.raises(ValueError):
            q.quamba_distill_loss(**{**good, **bad})
    good = dict(logits=x, teacher=top, teacher_tokens=tokens, log_sums=row, grad_losses=row, grad_logits=dx)
    q.quamba_distill_backward(**good)
    with pytest.raises(q.QuambaError) as e:
        q.quamba_distill_backward(**good, rest=True)
    assert e.value.status == NULL
    for bad in (dict(grad_logits=None), dict(grad_losses=row[:2]), dict(teacher=top[:2])):
        with pytest.raises(ValueError):
            q.quamba_distill_backward(**{**good, **bad})
