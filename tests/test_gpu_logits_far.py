"""GPU parity of the log probabilities and of the distance from a teacher where x / temperature is so large that its step in fp32 is above 1: masks
that are finite, whole rows of them, and temperatures near 0; in every form that a row may take, against plain loops in float64."""
import numpy as np
import pytest

import oracle
from test_gpu_logits import TYPES, U, _as, _check_backward, _dev, _gradient_close, _host, _logits, _near, _run, _sum_error, _torch_type, _value_tolerance

pytestmark = pytest.mark.gpu

MASKS = [-1e9, -1e10, -1.1 * 2 ** 33, -1e12, -1e20, 3e10]
# logits by a wave, by 256 and 1024 threads, in segments, and by 256 threads past the caches (test_logits_plans_of_segments.py checks which)
FORMS = [(8, 403), (8, 9001), (8, 70001), (8, 130001), (320, 120001)]
# loss and gradient: held by 64, 256, 512 (4, 8, 16 vectors), 1024 threads, in part, in two passes, and in segments
STEPS = [(8, 403), (8, 3501), (8, 15001), (8, 30001), (72, 60001), (72, 130001), (72, 250001), (72, 270001), (8, 130001)]


def _some(rows):
    """Rows that are compared: the first 8, which are all different."""
    return np.arange(min(rows, 8))


def _rows(rows, vocab, kind, mask, seed=1):
    """Eight rows, again and again: all forbidden, the first half, all but the last tokens, all but some, every other vector of 16 bytes, two
    masks, logits of that size, none forbidden."""
    import torch
    r = np.random.default_rng(seed)
    x = r.standard_normal((8, vocab)).astype(np.float32) * 2
    x[0] = mask
    x[1, :vocab // 2] = mask
    x[2, :-9] = mask
    keep = r.choice(vocab, 5, replace=False)
    x[3, np.setdiff1d(np.arange(vocab), keep)] = mask
    per = 4 if kind == "fp32" else 8
    x[4, np.arange(vocab) // per % 2 == 0] = mask
    x[5] = np.where(r.random(vocab) < 0.5, mask, mask * (1 + 2.0 ** -7))
    x[6] *= abs(mask)
    return torch.from_numpy(x).cuda().to(_torch_type(kind)).repeat((rows + 7) // 8, 1)[:rows].contiguous()


def _check_values(q, x, targets, count, T=1.0):
    """With a workspace and without, with every output and with the log probabilities alone (which sum without the entropy)."""
    some = _some(len(x))
    h = _host(x[:len(some)])
    want = oracle.ref_token_logprobs(h, [targets[r] for r in some], count, T)
    for workspace in (True, False):
        for everything in (True, False):
            got = {k: v[:len(some)].cpu().numpy() for k, v in _run(q, x, targets, count, T, workspace, everything).items()}
            assert np.array_equal(got["top_tokens"], want["top_tokens"])
            for r in some:
                tol = _value_tolerance(h[r], T)
                assert _near(got["logprobs"][r], want["logprobs"][r], tol(h[r, targets[r]])), r
                n = (want["top_tokens"][r] >= 0).sum()
                assert _near(got["top_logprobs"][r, :n], want["top_logprobs"][r, :n], tol(h[r, want["top_tokens"][r, :n]])), r
                if everything:
                    assert _near(got["log_sums"][r], want["log_sums"][r], tol(h[r].max()) + 4 * U * abs(h[r].max() / T)), r
                    H = want["entropies"][r]
                    assert abs(got["entropies"][r] - H) <= 2 * U * (H + np.log(h.shape[1]) + 8) * (_sum_error(h[r] / T, h.shape[1]) + 8), r
    return want


def _from_sums(x, q, left, tokens, valid, sums, rests, w, T):
    """The gradient as the definition has it, from log sums that are given."""
    dx = np.zeros(x.shape)
    with np.errstate(over="ignore"):
        for r in range(len(x)):
            if w[r] == 0 or not valid[r].any():
                continue
            p = np.exp(x[r] / T - sums[r])
            dx[r] = p * (q[r].sum() + left[r])
            np.add.at(dx[r], tokens[r][valid[r]], -q[r][valid[r]])
            if left[r] > 0:
                named = np.zeros(x.shape[1], bool)
                named[tokens[r][valid[r]]] = True
                dx[r] -= np.where(named, 0, left[r] * np.exp(x[r] / T - rests[r]))
    return dx * np.asarray(w)[:, None] / T


def _check_steps(q, x, teacher, tokens, rest, T=1.0, in_place=False, w=None):
    """Loss and gradient at once, the loss alone, and the gradient alone from what that left, whose log sums are rounded to fp32: a half step of theirs is
    a factor of the probabilities that the comparison takes as given."""
    import torch
    kind = {v: k for k, v in ((k, _torch_type(k)) for k in TYPES)}[x.dtype]
    rows, vocab = x.shape
    some = _some(rows)
    n, K = len(some), teacher.shape[1]
    teacher, tokens, w = _as(np.float32, teacher), _as(np.int32, tokens), np.ones(rows, np.float32) if w is None else _as(np.float32, w)
    h, keep = _host(x[:n]), x.clone()
    want = oracle.ref_distill(h, teacher[:n], tokens[:n], rest, w[:n], T)
    qs, left, log_p = want["q"], want["left"], want["log_p"]
    valid = (tokens[:n] >= 0) & (tokens[:n] < vocab) & (teacher[:n] != -np.inf)
    named = np.zeros(h.shape, bool)
    for r in some:
        named[r, tokens[r][valid[r]]] = True
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        # A sum's relative error; a value's argument has four roundings and the sum's error; q three of its argument's, the exponential and K additions.
        err = np.array([U * _sum_error(h[r] / T, vocab) for r in some])
        p, size = np.exp(log_p), np.abs(np.where(log_p > -np.inf, log_p, 0))
        p_rest = (p * ~named).sum(1)
        lq = np.abs(np.log(np.where(qs > 0, qs, 1)))
        lp = np.take_along_axis(size, np.clip(tokens[:n], 0, vocab - 1), 1)
        eq = U * (3 * (lq + 3) + 8 + K)
        of_left = (qs * eq).sum(1) + U * K
        logs = np.abs(np.log(np.where(left > 0, left, 1))) + np.abs(np.log(np.where((left > 0) & (p_rest > 0), p_rest, 1)))
        loss = (qs * (eq * (lq + lp + 1) + U * (8 * (lp + 8) + 4 * np.log(vocab)) + err[:, None])).sum(1) \
            + rest * (of_left * (logs + 2) + left * (2 * err + U * (6 * logs + 16))) + 1e-37
        share = np.where(named | (p_rest == 0)[:, None], 0, p / np.where(p_rest > 0, p_rest, 1)[:, None])
        of_q = np.zeros(h.shape)
        for r in some:
            np.add.at(of_q[r], tokens[r][valid[r]], (qs[r] * (eq[r] + U * K))[valid[r]])
        scale = (np.abs(w[:n]) / T)[:, None]
        gradient = scale * (p * (U * (4 * size + 30) + 2 * err[:, None] + of_left[:, None]) + of_q
                            + rest * share * (left[:, None] * (U * (4 * size + 30) + 3 * err[:, None]) + of_left[:, None]))
    f = lambda: torch.full((rows,), 7.0, device="cuda")
    t, at, wd = _dev(teacher), _dev(tokens, np.int32), _dev(w)
    bytes_ = q.quamba_distill_loss_workspace_size(rows, vocab, K)
    for workspace in (True, False):
        space = torch.full((bytes_,), 0xFF, dtype=torch.uint8, device="cuda") if workspace else None
        for step in (False, True):
            x.copy_(keep)
            losses, sums, rests, dx = f(), f(), f(), None if not step else x if in_place else torch.full_like(x, 3.0)
            q.quamba_distill_loss(x, t, at, losses, log_sums=sums, log_rests=rests, weights=wd, grad_logits=dx, rest=rest, temperature=T, workspace=space)
            got = _host(losses)[:n]
            assert _near(got, want["losses"], loss), (workspace, step, got, want["losses"])
            top = np.abs(h.max(1) / T)
            live = valid.any(1) & (w[:n] != 0)
            assert _near(_host(sums)[:n][live], want["log_sums"][live], (err + U * (8 * top + 8 + 4 * np.log(vocab)))[live])
            if step:
                _gradient_close(_host(dx)[:n], want["gradient"], kind, np.nan_to_num(gradient))
    x.copy_(keep)
    dx = x if in_place else torch.full_like(x, 3.0)
    q.quamba_distill_backward(x, t, at, sums, wd, dx, log_rests=rests if rest else None, rest=rest, temperature=T)
    S, R = _host(sums)[:n], _host(rests)[:n]
    given = _from_sums(h, qs, left, tokens[:n], valid, S, R, w[:n], T)
    with np.errstate(over="ignore", invalid="ignore"):
        lp = np.where(np.isfinite(h), h / T - S[:, None], 0)
        lr = np.where(np.isfinite(h) & ~named & np.isfinite(R)[:, None], h / T - R[:, None], 0)
        # an argument is a difference, a product and what the sum's product with the temperature leaves, which is within half a step of that sum
        rounds = lambda a, sum_: U * (4 * np.abs(a) + 30 + 2 * U * np.abs(sum_)[:, None])
        mass = np.where(np.isfinite(h), np.exp(np.minimum(lp, 80)), 0)
        others = np.where(np.isfinite(h) & ~named, np.exp(np.minimum(lr, 80)), 0) * rest
        arithmetic = scale * (mass * (rounds(lp, S) + of_left[:, None]) + of_q + others * (left[:, None] * (rounds(lr, R) + rounds(lp, S)) + of_left[:, None]))
    _gradient_close(_host(dx)[:n], given, kind, np.nan_to_num(arithmetic))
    x.copy_(keep)


def _teacher(rows, vocab, rest, T=1.0, K=6):
    """Distinct tokens, the first and the last among them; with a rest log probabilities that leave 0.2."""
    r = np.random.default_rng(vocab)
    tokens = np.stack([r.choice(np.arange(1, vocab - 1), K, replace=False) for _ in range(8)])
    tokens[:, 0], tokens[:, K - 1] = 0, vocab - 1
    log_q = np.log(0.8 * r.dirichlet(np.ones(K), 8))
    t = log_q if rest else log_q * T
    again = lambda v: np.tile(v, ((rows + 7) // 8, 1))[:rows]
    return again(t), again(tokens)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("count", [0, 9])
@pytest.mark.parametrize("rows,vocab", FORMS)
def test_logprobs_beside_finite_masks(gpu_lib, rows, vocab, count, kind):
    for mask in MASKS if rows == 8 else MASKS[1:2]:
        x = _rows(rows, vocab, kind, mask)
        targets = np.resize([vocab - 1, vocab // 2, vocab - 1, 0, vocab - 2, 1, 2, 3], rows)
        _check_values(gpu_lib, x, targets, count)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("count", [0, 9])
@pytest.mark.parametrize("rows,vocab", FORMS[:4])
def test_logprobs_at_temperatures_near_0(gpu_lib, rows, vocab, count, kind):
    """Largest logits are equal ones."""
    x = (_logits(rows, vocab, "fp32", vocab) * 2).round().div(2).to(_torch_type(kind))
    x[3] = 0
    x[4, 100:] = float("-inf")
    for T in (float(np.float32(1e-5)), float(np.float32(1e-8)), 2.0 ** -27, 2.0 ** -60, 2.0 ** -100, 2.0 ** 100):
        _check_values(gpu_lib, x, [0, 1, 2, 3, 99, 5, 6, vocab - 1], count, T)


@pytest.mark.parametrize("count", [0, 9])
@pytest.mark.parametrize("rows,vocab", FORMS[:4])
def test_logprobs_where_a_step_of_fp32_reaches_1(gpu_lib, rows, vocab, count):
    """Around 2^23 and 2^24, over log2(e) and as they are, neighbours among them."""
    import torch
    r = np.random.default_rng(vocab)
    x = np.stack([s * v + r.integers(-6, 7, vocab) for s in (1, -1) for v in (2 ** 23 / 1.4426950, 2 ** 23, 2 ** 24 / 1.4426950, 2 ** 24)])
    _check_values(gpu_lib, torch.from_numpy(x.astype(np.float32)).cuda(), np.arange(8), count)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("T", [2.0 ** -20, 2.0 ** -27, 2.0 ** -60])
def test_gradient_of_logprobs_at_temperatures_near_0(gpu_lib, T, kind):
    """From the log sums in fp32, which hold the largest logit and no more."""
    x = (_logits(8, 9001, "fp32", 3) * 2).round().div(2).to(_torch_type(kind))
    targets = [0, 1, 2, 3, 4, -1, 6, 9000]
    forward = oracle.ref_token_logprobs(_host(x), targets, 0, T)
    g, h = np.linspace(-1, 1, 8) * T, np.linspace(1, 2, 8) * T
    _check_backward(gpu_lib, x, targets, forward, g, None, T)
    _check_backward(gpu_lib, x, targets, forward, g, h, T)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab", STEPS)
def test_distill_beside_finite_masks(gpu_lib, rows, vocab, rest, kind):
    vocab = vocab // 2 if kind == "fp32" else vocab
    teacher, tokens = _teacher(rows, vocab, rest)
    for mask in MASKS if vocab < 40000 else MASKS[1:2]:
        _check_steps(gpu_lib, _rows(rows, vocab, kind, mask), teacher, tokens, rest, in_place=mask == MASKS[3])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab", [(8, 403), (8, 9001), (8, 130001)])
def test_distill_at_temperatures_near_0(gpu_lib, rows, vocab, rest, kind):
    x = (_logits(rows, vocab, "fp32", vocab) * 2).round().div(2).to(_torch_type(kind))
    x[3] = 0
    for T in (2.0 ** -20, 2.0 ** -27, 2.0 ** -60):
        teacher, tokens = _teacher(rows, vocab, rest, T)
        _check_steps(gpu_lib, x, teacher, tokens, rest, T, w=np.linspace(-1, 1, rows) * T)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("T", [2.0 ** 20, 2.0 ** 100])
def test_distill_at_high_temperatures(gpu_lib, T, rest, kind):
    """Every token is as likely as any other; the weights bring the gradient back into fp32's and fp16's range."""
    for rows, vocab in ((8, 403), (8, 9001), (8, 130001)):
        teacher, tokens = _teacher(rows, vocab, rest)
        _check_steps(gpu_lib, _logits(rows, vocab, kind, vocab), teacher, tokens, rest, T, w=np.linspace(-1, 1, rows) * T)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("size", [1e10, -1e10, 1e20, -1e20, 2.0 ** 25, -2.0 ** 31])
def test_gradient_alone_from_log_sums_of_that_size(gpu_lib, size, rest, kind):
    """No sum is made here: the log sums are float64's, in fp32."""
    import torch
    x = _rows(8, 5003, kind, size)
    teacher, tokens = _teacher(8, 5003, rest)
    h = _host(x)
    want = oracle.ref_distill(h, teacher, tokens, rest)
    S, R = (_as(np.float32, want[k]) for k in ("log_sums", "log_rests"))
    dx = torch.full_like(x, 3.0)
    gpu_lib.quamba_distill_backward(x, _dev(teacher), _dev(tokens, np.int32), _dev(S), _dev(np.ones(8)), dx, log_rests=_dev(R) if rest else None, rest=rest)
    given = _from_sums(h, want["q"], want["left"], tokens, np.ones(tokens.shape, bool), _as(np.float64, S), _as(np.float64, R), np.ones(8), 1.0)
    # terms: p, q and p / p_R, each with the roundings of an argument of at most 88 (below that they are 0) and the factor's; the teacher's sum is exact to 6 places' additions
    most = np.exp(np.minimum(h - S[:, None], 80)) + np.where(rest, np.exp(np.minimum(h - (R if rest else S)[:, None], 80)), 0) + 1
    _gradient_close(_host(dx), given, kind, U * (4 * 88 + 60) * most)
