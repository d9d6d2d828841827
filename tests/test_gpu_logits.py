"""GPU parity of the log probabilities (tokens exactly, values to fp32 rounding), of the distance from a teacher and of their gradients, through
the C ABI, against plain loops in float64."""
import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu

TYPES = ("fp32", "fp16", "bf16")
U = 2.0 ** -24                                  # half a unit of fp32, relative
HALF = {"fp32": U, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}      # of the gradient's type
TINY = {"fp32": 2.0 ** -140, "fp16": 2.0 ** -25, "bf16": 2.0 ** -134}


def _torch_type(name):
    import torch
    return {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}[name]


def _logits(rows, vocab, kind, seed, spread=2.0):
    import torch
    r = np.random.default_rng(seed)
    return torch.from_numpy((r.standard_normal((rows, vocab)) * spread).astype(np.float32)).cuda().to(_torch_type(kind))


def _as(dtype, v):
    return np.asarray(v, dtype)


def _host(t):
    return t.double().cpu().numpy()


def _dev(v, dtype=None):
    import torch
    return None if v is None else torch.from_numpy(np.ascontiguousarray(np.asarray(v, dtype or np.float32))).cuda()


def _additions(vocab):
    """How many additions stand behind one another in a row's sum: a thread's vectors of 4 or 8 logits, the 8 of one, those of 16 waves and of the segments."""
    return vocab / (4 * 256) + 8 + 16 + 256


def _sum_error(z, vocab):
    """Relative error of a row's sum of exponentials, in units of 2^-24: every term's argument has three roundings (the difference, the
    factor, their product) relative to its size, which is counted from a reference that may lie 2^8 below the largest, the exponential is
    good to two units (half steps four), and every addition rounds once.  Terms count by their share."""
    d = z - z.max()
    p = np.exp(d) / np.exp(d).sum()
    return (p * np.where(p > 0, 3 * (np.abs(np.where(p > 0, d, 0)) + 6) + 4, 0)).sum() + _additions(vocab)


def _value_tolerance(x, T):
    """Of the values ln p of a row: function of the exact ones.  The difference from the reference, 1 / T and the product round once each, the
    logarithm's result twice and the last difference once."""
    z = x / T
    err = _sum_error(z, x.size)
    top = z[np.isfinite(z)].max()
    return lambda logit: U * (4 * (np.abs(logit / T - top) + 6) + err + 4 * (6 + np.log(x.size)) + np.abs(logit / T - top))


def _near(got, want, tolerance):
    """Within the tolerance, and infinite where the value has no place in fp32 (the lowest logit over a temperature below 1)."""
    got, want = _as(np.float64, got), _as(np.float64, want)
    beyond = np.abs(want) > np.finfo(np.float32).max
    with np.errstate(invalid="ignore"):
        return np.where(beyond, got == np.copysign(np.inf, want), np.abs(got - want) <= tolerance).all()


def _run(q, logits, targets, count, T=1.0, workspace=True, everything=True):
    import torch
    rows, vocab = logits.shape
    o = dict(logprobs=torch.full((rows,), 7.0, device="cuda"), log_sums=torch.full((rows,), 7.0, device="cuda"),
             entropies=torch.full((rows,), 7.0, device="cuda"), top_logprobs=torch.full((rows, count), 7.0, device="cuda"),
             top_tokens=torch.full((rows, count), -9, dtype=torch.int32, device="cuda"))
    size = q.quamba_token_logprobs_workspace_size(rows, vocab, count)
    space = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if workspace and size else None
    q.quamba_token_logprobs(logits, _dev(targets, np.int32), None if targets is None else o["logprobs"],
                            log_sums=o["log_sums"] if everything else None, entropies=o["entropies"] if everything else None,
                            top_logprobs=o["top_logprobs"] if count else None, top_tokens=o["top_tokens"] if count else None, temperature=T,
                            workspace=space)
    return o


def _check(q, logits, targets, count=0, T=1.0, rows=slice(None)):
    """Of all rows, or of some of a call with more."""
    x, of_all = _host(logits[rows]), targets
    targets = None if targets is None else np.asarray(targets)[rows]
    want = oracle.ref_token_logprobs(x, targets, count, T)
    for workspace in (True, False):
        got = {k: v[rows].cpu().numpy() for k, v in _run(q, logits, of_all, count, T, workspace).items()}
        assert np.array_equal(got["top_tokens"], want["top_tokens"])
        for r in range(x.shape[0]):
            if targets is not None and not 0 <= targets[r] < x.shape[1] or np.isnan(want["log_sums"][r]):
                for k in ("log_sums", "entropies") + (("logprobs",) if targets is not None else ()):
                    assert np.array_equal(got[k][r], want[k][r], equal_nan=True), (k, r)
                assert np.isneginf(got["top_logprobs"][r]).all()
                continue
            tol = _value_tolerance(x[r], T)
            if targets is not None:
                assert _near(got["logprobs"][r], want["logprobs"][r], tol(x[r, targets[r]])), r
            assert _near(got["log_sums"][r], want["log_sums"][r], tol(x[r].max()) + 4 * U * abs(x[r].max() / T)), r
            n = (want["top_tokens"][r] >= 0).sum()
            assert _near(got["top_logprobs"][r, :n], want["top_logprobs"][r, :n], tol(x[r, want["top_tokens"][r, :n]])), r
            assert np.isneginf(got["top_logprobs"][r, n:]).all()
            # the entropy: ln S and the weighted mean of the arguments, each with the sum's error and its own roundings
            H = want["entropies"][r]
            assert abs(got["entropies"][r] - H) <= 2 * U * (H + np.log(x.shape[1]) + 8) * (_sum_error(x[r] / T, x.shape[1]) + 8), r
    return want


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,vocab,count", [(1, 1, 1), (1, 5, 8), (3, 7, 0), (5, 33, 128), (2, 2049, 5), (1, 50021, 20), (33, 4099, 64), (1100, 517, 3),
                                              (2, 300001, 128), (1, 131072, 1), (3, 40000, 0), (1025, 1000, 1), (520, 3001, 9)])
def test_logprobs(gpu_lib, rows, vocab, count, kind):
    r = np.random.default_rng(vocab)
    _check(gpu_lib, _logits(rows, vocab, kind, vocab + rows), r.integers(0, vocab, rows), count)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("T", [0.05, 0.7, 3.0, 1000.0])
def test_logprobs_at_a_temperature(gpu_lib, T, kind):
    _check(gpu_lib, _logits(3, 5003, kind, 1), [0, 5002, 77], 6, T)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows", [1, 20, 600])
def test_padding(gpu_lib, rows, kind):
    x = _logits(rows, 9001, kind, 2)
    targets = np.random.default_rng(3).integers(0, 9001, rows)
    targets[::3] = np.resize([-1, 9001, -100, 2 ** 31 - 1, -2 ** 31], targets[::3].size)
    x[::3] = float("nan")                                         # and is not read
    _check(gpu_lib, x, targets, 4)


@pytest.mark.parametrize("kind", TYPES)
def test_masks(gpu_lib, kind):
    """Rows with every logit forbidden, with few allowed ones, with the type's lowest value for a mask (in part, throughout), NaN and
    infinity in a row, logits far below 0, far above the rest, and a target that is forbidden."""
    import torch
    vocab = 9001
    x = _logits(10, vocab, kind, 8)
    low = torch.finfo(x.dtype).min
    x[0] = -np.inf
    x[1, 5:] = -np.inf
    x[2, 3:] = low
    x[3] = low
    x[4, 77] = np.nan
    x[5, 8999] = np.inf
    x[6] -= 10000 if kind != "fp16" else 1000
    x[7, 9000] = 60000.0
    x[8, :8990] = -np.inf
    x[9] = -np.inf
    x[9, 4321] = low
    targets = [3, 4, 2, 9000, 5, 8999, 17, 0, 5, 4321]
    _check(gpu_lib, x, targets, 9)
    for r in range(10):                                           # each alone, in many segments, and in a batch that has one each
        _check(gpu_lib, x[r:r + 1], [targets[r]], 20)
    _check(gpu_lib, x.repeat(60, 1), targets * 60, 3)
    wide = torch.cat([x] * 6, 1)                                  # threads see several vectors
    _check(gpu_lib, wide, targets, 40, 0.5)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab,count", [(1000, 6), (70000, 128), (2500, 65), (30000, 20)])
def test_ties(gpu_lib, vocab, count, kind):
    """Few different logits, or one, zeros of both signs: the lowest tokens first; in segments and by one workgroup."""
    import torch
    r = np.random.default_rng(5)
    rows = [r.integers(0, 3, vocab), np.zeros(vocab), np.full(vocab, -3.0), np.where(r.random(vocab) < 0.5, 0.0, -0.0),
            np.where(np.arange(vocab) < vocab - 3, -0.0, 0.0), np.where(np.arange(vocab) % 1000 == 999, 1.0, -2.0)]
    x = torch.from_numpy(np.stack(rows).astype(np.float32)).cuda().to(_torch_type(kind))
    _check(gpu_lib, x, [0] * len(rows), count)
    if vocab < 5000:
        _check(gpu_lib, x.repeat(200, 1), [1] * 1200, count)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("count", [1, 8, 128])
def test_rows_in_order(gpu_lib, count, kind):
    """Rising logits (every vector better than all before it), falling ones, the best all at one end, and logits that rise so far
    that the sum's reference is replaced again and again."""
    x = _logits(8, 70001, kind, 21)
    x[0] = x[0].sort().values
    x[1] = x[1].sort(descending=True).values
    x[2, 69900:] += 30
    x[3, :100] += 30
    x[4] = x[4].sort().values * 100
    x[5] = x[5].sort(descending=True).values * 100
    x[6, 35000:] = -np.inf
    x[7] = (x[7] * 4).round()
    _check(gpu_lib, x, [70000, 0, 69950, 99, 70000, 0, 1, 1], count)


@pytest.mark.parametrize("kind", TYPES)
def test_a_padded_vocabulary_at_odd_addresses(gpu_lib, kind):
    """Rows further apart than they are long; what lies between is not read as logits."""
    import torch
    for left in (0, 1, 3, 7):
        for vocab in (5003, 4, 8, 1):
            wide = torch.full((6, vocab + 11), float("inf"), dtype=_torch_type(kind), device="cuda")
            wide[:, left:left + vocab] = _logits(6, vocab, kind, 9)
            _check(gpu_lib, wide[:, left:left + vocab], [0, vocab - 1, vocab // 2, 0, -1, 0], 5)


def test_offsets_beyond_32_bits(gpu_lib):
    """Rows over 4 GiB from the first, with their gradient."""
    import torch
    far = 3 << 29
    wide = torch.empty(2 * far + 4000, dtype=torch.float16, device="cuda")
    x = wide.as_strided((3, 4000), (far, 1))
    x.copy_(_logits(3, 4000, "fp16", 10))
    want = _check(gpu_lib, x, [5, 6, 3999], 6)
    _check_backward(gpu_lib, x, [5, 6, 3999], want, [1.0, -2.0, 0.5], None, 1.0, out=x)


def test_more_rows_than_a_launch_takes(gpu_lib):
    import torch
    rows = (1 << 22) + 1000
    x = torch.randn(rows, 3, device="cuda").bfloat16()
    targets = torch.randint(-1, 3, (rows,), dtype=torch.int32, device="cuda")
    out, top = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
    tokens = torch.empty(rows, 2, dtype=torch.int32, device="cuda")
    sums = torch.empty(rows, device="cuda")
    gpu_lib.quamba_token_logprobs(x, targets, out, log_sums=sums, top_logprobs=top, top_tokens=tokens)
    log_p = torch.log_softmax(x.double(), 1)
    live = targets >= 0
    want = torch.where(live, log_p.gather(1, targets.clamp(min=0).long()[:, None])[:, 0], 0.0)
    assert float((out - want).abs().max()) < 3e-6
    dx = torch.empty_like(x)
    gpu_lib.quamba_token_logprobs_backward(x, targets, sums, torch.ones(rows, device="cuda"), dx)
    want = torch.zeros_like(log_p).scatter_(1, targets.clamp(min=0).long()[:, None], 1.0) - log_p.exp()
    assert float((dx - torch.where(live[:, None], want, 0.0)).abs().max()) < 2.0 ** -8
    losses = torch.empty(rows, device="cuda")
    gpu_lib.quamba_distill_loss(x, torch.zeros(rows, 1, device="cuda"), targets[:, None], losses, grad_logits=dx)
    assert float((losses + torch.where(live, log_p.gather(1, targets.clamp(min=0).long()[:, None])[:, 0], 0.0)).abs().max()) < 3e-6
    assert float((dx + torch.where(live[:, None], want, 0.0)).abs().max()) < 2.0 ** -8


def test_what_is_not_asked_for(gpu_lib):
    """Each output alone has the bits that it has beside the others; no target; nothing at all."""
    import torch
    q = gpu_lib
    for rows in (2, 700):
        x, targets = _logits(rows, 9011, "bf16", 12), np.arange(rows)
        full = _run(q, x, targets, 5)
        alone = torch.empty(rows, device="cuda")
        q.quamba_token_logprobs(x, None, None, top_logprobs=(v := torch.empty(rows, 5, device="cuda")),
                                top_tokens=(t := torch.empty(rows, 5, dtype=torch.int32, device="cuda")),
                                workspace=torch.empty(q.quamba_token_logprobs_workspace_size(rows, 9011, 5), dtype=torch.uint8, device="cuda"))
        assert torch.equal(t, full["top_tokens"]) and torch.allclose(v, full["top_logprobs"], atol=1e-5, rtol=0)
        q.quamba_token_logprobs(x, None, None, log_sums=alone)
        assert torch.allclose(alone, full["log_sums"], atol=1e-5, rtol=0)
        q.quamba_token_logprobs(x, None, None, entropies=alone)
        assert torch.allclose(alone, full["entropies"], atol=1e-5, rtol=0)
        q.quamba_token_logprobs(x, None, None)
    q.quamba_token_logprobs(torch.empty(0, 9, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda"))


def test_the_same_call_gives_the_same_bits(gpu_lib):
    import torch
    for rows, vocab in ((1, 128000), (40, 50021), (600, 20011), (9000, 1031), (700, 40009)):
        x = _logits(rows, vocab, "bf16", 13)
        a, b = (_run(gpu_lib, x, np.zeros(rows, int), 64) for _ in range(2))
        assert all(torch.equal(a[k], b[k]) for k in a)


# ---------------------------------------------------------------- gradients


def _gradient_close(got, want, kind, arithmetic):
    """Half a step of the type, and the arithmetic's error in front of it."""
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    off = np.abs(got - want, where=fin, out=np.zeros_like(want))
    bound = HALF[kind] * np.abs(want) + (1 + HALF[kind]) * arithmetic + TINY[kind]
    assert (off[fin] <= bound[fin]).all(), (off[fin] - bound[fin]).max()


def _check_backward(q, logits, targets, forward, g, h, T, out=None, some=slice(None)):
    import torch
    x, kind = _host(logits[some]), {v: k for k, v in ((k, _torch_type(k)) for k in TYPES)}[logits.dtype]
    sums, entropies = _as(np.float32, forward["log_sums"]), _as(np.float32, forward["entropies"])
    of_all = dict(targets=_dev(targets, np.int32), sums=_dev(sums), g=_dev(g), entropies=None if h is None else _dev(entropies), h=_dev(h))
    sums, entropies = sums[some], entropies[some]
    targets, g, h = (None if v is None else np.asarray(v)[some] for v in (targets, g, h))
    want = oracle.ref_token_logprobs_backward(x, targets, sums, entropies, None if g is None else _as(np.float32, g), None if h is None else _as(np.float32, h), T)
    dx = torch.full_like(logits, 3.0) if out is None else out
    q.quamba_token_logprobs_backward(logits, of_all["targets"], of_all["sums"], of_all["g"], dx, entropies=of_all["entropies"],
                                     grad_entropies=of_all["h"], temperature=T)
    got = _host(dx[some])
    with np.errstate(invalid="ignore", over="ignore"):
        log_p = x / T - sums[:, None]
        p = np.exp(log_p)
        # the argument has four roundings of its size, p two more and four half steps of the exponential, what it is multiplied with four, and 1 / T
        gg, hh = (np.abs(np.zeros(len(x)) if v is None else _as(np.float64, _as(np.float32, v)))[:, None] for v in (g, h))
        slope = gg + hh * (np.abs(np.where(p > 0, log_p, 0)) + np.abs(entropies[:, None]))
        arithmetic = U * np.where(p > 0, p * slope * (4 * np.abs(np.where(p > 0, log_p, 0)) + 16), 0) / T
        if targets is not None:
            live = (np.asarray(targets) >= 0) & (np.asarray(targets) < x.shape[1])
            rows = np.nonzero(live)[0]
            arithmetic[rows, np.asarray(targets)[rows]] += 4 * U * gg[rows, 0] / T
    _gradient_close(got, want, kind, np.nan_to_num(arithmetic))
    return want


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("rows,vocab,T", [(1, 1, 1.0), (2, 9, 0.5), (3, 4099, 1.0), (1, 50021, 2.0), (70, 8192, 0.7), (1100, 333, 1.0)])
def test_backward(gpu_lib, rows, vocab, T, entropy, kind):
    r = np.random.default_rng(vocab)
    x, targets = _logits(rows, vocab, kind, vocab), r.integers(0, vocab, rows)
    targets[1::5] = -1
    forward = oracle.ref_token_logprobs(_host(x), targets, 0, T)
    g, h = r.standard_normal(rows), r.standard_normal(rows) if entropy else None
    g[::7] = 0
    _check_backward(gpu_lib, x, targets, forward, g, h, T)
    if entropy:
        _check_backward(gpu_lib, x, None, oracle.ref_token_logprobs(_host(x), None, 0, T), None, h, T)
    _check_backward(gpu_lib, x, targets, forward, g, h, T, out=x)      # in the logits' place


@pytest.mark.parametrize("kind", TYPES)
def test_backward_of_masked_rows_and_of_rows_without_a_distribution(gpu_lib, kind):
    import torch
    x = _logits(7, 3001, kind, 14)
    x[0, 5:] = -np.inf
    x[1, 9:] = torch.finfo(x.dtype).min
    x[2] = torch.finfo(x.dtype).min
    x[3, 4] = np.nan                                        # its gradients are 0: it is not read
    x[4] = np.nan                                           # padding
    x[5, 7] = np.nan
    x[6, 7] = -np.inf                                       # the target
    targets = [2, 3, 1, 5, -1, 8, 7]
    forward = oracle.ref_token_logprobs(_host(x), targets)
    g, h = [1.0, 2.0, -1.0, 0.0, 3.0, 1.0, 1.0], [0.5, 0.0, 1.0, 0.0, 1.0, 1.0, 0.0]
    want = _check_backward(gpu_lib, x, targets, forward, g, None, 1.0)
    assert np.isnan(want[5]).all() and not want[3:5].any()
    _check_backward(gpu_lib, x, targets, forward, g, h, 1.0)


@pytest.mark.parametrize("kind", TYPES)
def test_gradients_among_other_columns(gpu_lib, kind):
    """Logits and their gradient as columns of wide matrices, at addresses that differ in 16 bytes: what lies between stays."""
    import torch
    dt = _torch_type(kind)
    for left, right, vocab in ((0, 3, 1003), (5, 5, 77), (1, 0, 2), (3, 2, 4096)):
        wide, room = torch.full((4, vocab + 9), float("nan"), dtype=dt, device="cuda"), torch.full((4, vocab + 13), 5.0, dtype=dt, device="cuda")
        x, out = wide[:, left:left + vocab], room[:, right:right + vocab]
        x.copy_(_logits(4, vocab, kind, 15))
        forward = oracle.ref_token_logprobs(_host(x), [0, 1, -1, vocab - 1])
        _check_backward(gpu_lib, x, [0, 1, -1, vocab - 1], forward, [1.0, 2, 3, -1], [1.0, 0, 3, 1], 1.0, out=out)
        assert (room[:, :right] == 5).all() and (room[:, right + vocab:] == 5).all()
        room.fill_(5.0)
        tokens, teacher = np.tile([0, vocab - 1], (4, 1)), np.log(np.tile([0.5, 0.3], (4, 1)))
        _check_distill(gpu_lib, x, teacher, tokens, True, [1.0, 2, 0, -1], 1.0, out=out)
        assert (room[:, :right] == 5).all() and (room[:, right + vocab:] == 5).all()
    both = torch.zeros(4, 128, dtype=dt, device="cuda")      # side by side in one matrix
    both[:, :60] = _logits(4, 60, kind, 16)
    forward = oracle.ref_token_logprobs(_host(both[:, :60]), [0, 1, 2, 3])
    _check_backward(gpu_lib, both[:, :60], [0, 1, 2, 3], forward, [1.0] * 4, None, 1.0, out=both[:, 60:120])


def test_backward_against_differences(gpu_lib):
    """Central differences of the kernel's own outputs, which are good to some 2^-22 of 10."""
    import torch
    q = gpu_lib
    x, targets, T = _logits(2, 40, "fp32", 17), [3, 11], 0.8
    g, h = _as(np.float32, [1.0, -0.5]), _as(np.float32, [0.3, 0.7])
    forward = {k: v.cpu().numpy() for k, v in _run(q, x, targets, 0, T).items()}
    dx = torch.empty_like(x)
    q.quamba_token_logprobs_backward(x, _dev(targets, np.int32), _dev(forward["log_sums"]), _dev(g), dx, entropies=_dev(forward["entropies"]),
                                     grad_entropies=_dev(h), temperature=T)
    for r, v in ((0, 3), (0, 4), (1, 11), (1, 39)):
        value = []
        for step in (0.03, -0.03):
            y = x.clone()
            y[r, v] += step
            o = _run(q, y, targets, 0, T)
            value.append((o["logprobs"].cpu().numpy() * g + o["entropies"].cpu().numpy() * h)[r])
        # a third derivative of at most 10 / T^3 over 6, and two values' rounding over 0.06
        assert abs((value[0] - value[1]) / 0.06 - float(dx[r, v])) <= 0.03 ** 2 * 10 / T ** 3 / 6 + 2 * 2.0 ** -22 * 10 / 0.06


# ---------------------------------------------------------------- a teacher


def _teacher(rows, vocab, K, rest, seed, T=1.0, empty=True):
    r = np.random.default_rng(seed)
    tokens = np.stack([r.permutation(vocab)[:K] if K <= vocab else r.integers(0, vocab, K) for _ in range(rows)]).astype(np.int32)
    t = np.sort(r.standard_normal((rows, K)) * 2, 1)[:, ::-1] + 3
    if rest:
        t = t / T
        t = t - np.log(np.exp(t).sum(1, keepdims=True)) + np.log1p(-np.exp(r.uniform(np.log(0.003), np.log(0.6), (rows, 1))))
    if empty:
        tokens[::4, K // 2:] = np.resize([-1, vocab, 2 ** 31 - 1, -2 ** 31], tokens[::4, K // 2:].shape[1])
        t[1::4, K // 3:] = -np.inf
    return _as(np.float32, t), tokens


def _check_distill(q, logits, teacher, tokens, rest, weights=None, T=1.0, out=None, losses_only=False, some=slice(None)):
    """Of all rows, or of some of a call with more."""
    import torch
    kind = {v: k for k, v in ((k, _torch_type(k)) for k in TYPES)}[logits.dtype]
    x = _host(logits[some])
    rows, vocab = x.shape
    K = teacher.shape[1]
    teacher, tokens = _as(np.float32, teacher), _as(np.int32, tokens)
    w = None if weights is None else _as(np.float32, weights)
    of_all = dict(teacher=_dev(teacher), tokens=_dev(tokens, np.int32), w=_dev(w))
    all_rows = len(teacher)
    teacher, tokens, w = teacher[some], tokens[some], None if w is None else w[some]
    want = oracle.ref_distill(x, teacher, tokens, rest, w, T)
    keep = logits.clone()
    size = q.quamba_distill_loss_workspace_size(all_rows, vocab, K)
    dead = np.array([(want["q"][r] == 0).all() and not np.isnan(want["losses"][r]) for r in range(rows)])
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        err = np.array([U * _sum_error(x[r] / T, vocab) if np.isfinite(want["log_sums"][r]) and not dead[r] else 0.0 for r in range(rows)])
        top = np.where(np.isfinite(x), x, -1e30).max(1) / T
        absp = np.abs(np.where(want["log_p"] > -np.inf, want["log_p"], 0))
        p = np.where(dead[:, None] | np.isnan(want["losses"])[:, None], 0, np.exp(want["log_p"]))
        at = np.clip(tokens, 0, vocab - 1)
        lq = np.abs(np.log(np.where(want["q"] > 0, want["q"], 1)))
        lp = np.take_along_axis(absp, at, 1)
        # q: three roundings of the teacher's argument, the exponential, the normalisation (K additions, a division); its logarithm alike
        eq = U * (3 * (lq + 3) + 8 + K)
        wp = np.ones(rows) if w is None else np.abs(_as(np.float64, w))
        named = np.zeros(x.shape, bool)
        for r in range(rows):
            for k in range(K):
                if 0 <= tokens[r, k] < vocab and teacher[r, k] != -np.inf:
                    named[r, tokens[r, k]] = True
        pr = (p * ~named).sum(1)
        left = want["left"]
        leftover = (want["q"] * eq).sum(1) + U * K                                              # of q_R, absolute
        log_left = np.abs(np.log(np.where(left > 0, left, 1))) + np.abs(np.log(np.where((left > 0) & (pr > 0), pr, 1)))
        tol = (want["q"] * (eq * (lq + lp + 1) + U * (6 * (lp + 8) + 4 * np.log(vocab)) + err[:, None])).sum(1) \
            + np.where(rest, leftover * (log_left + 2) + left * (2 * err + U * (4 * log_left + 8)), 0) + U * (K + 8) * np.abs(np.where(np.isfinite(want["losses"]), want["losses"], 0)) + 1e-37
        # the gradient: p's error, q's, and of the other tokens the share of the rest
        eqsum = np.zeros(x.shape)
        for r in range(rows):
            np.add.at(eqsum[r], at[r], want["q"][r] * (eq[r] + U * K))
        share = np.where(named | (pr[:, None] == 0) | (left[:, None] == 0), 0, p * (left / np.where(pr > 0, pr, 1))[:, None])
        arithmetic = (wp / T)[:, None] * (p * (U * (4 * absp + 30) + 2 * err[:, None] + leftover[:, None]) + eqsum
                                          + share * (U * (4 * absp + 30) + 3 * err[:, None])
                                          + np.where(named | (pr[:, None] == 0), 0, p / np.where(pr > 0, pr, 1)[:, None] * leftover[:, None] * bool(rest)))
    for workspace in (True, False):
        for gradient in ((False,) if losses_only else (False, True)):
            logits.copy_(keep)
            o = {k: torch.full((all_rows,), 7.0, device="cuda") for k in ("losses", "log_sums", "log_rests")}
            dx = None if not gradient else torch.full_like(logits, 3.0) if out is None else out
            space = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if workspace and size else None
            q.quamba_distill_loss(logits, of_all["teacher"], of_all["tokens"], o["losses"], log_sums=o["log_sums"], log_rests=o["log_rests"],
                                  weights=of_all["w"], grad_logits=dx, rest=rest, temperature=T, workspace=space)
            got = _host(o["losses"][some])
            fin = np.isfinite(want["losses"])
            assert np.array_equal(got[~fin], want["losses"][~fin], equal_nan=True)
            assert (np.abs(got[fin] - want["losses"][fin]) <= tol[fin]).all(), (np.abs(got[fin] - want["losses"][fin]) / tol[fin]).max()
            ok = fin & ~dead
            sums, rests = _host(o["log_sums"][some]), _host(o["log_rests"][some])
            assert (np.abs(sums[ok] - want["log_sums"][ok]) <= (err + U * (8 * np.abs(top) + 8 + 4 * np.log(vocab)))[ok]).all()
            if rest:
                few = ok & np.isfinite(want["log_rests"])
                assert (np.abs(rests[few] - want["log_rests"][few]) <= (2 * err + U * (8 * np.abs(top) + 8 * np.abs(want["log_rests"]) + 64))[few]).all()
            assert (sums[dead] == 0).all() and (rests[dead] == 0).all()
            if gradient:
                _gradient_close(_host(dx[some]), want["gradient"], kind, np.nan_to_num(arithmetic))
    if losses_only:
        return want
    # the gradient alone, from what the call left; the log sums' rounding goes into p
    logits.copy_(keep)
    dx = torch.full_like(logits, 3.0) if out is None else out
    q.quamba_distill_backward(logits, of_all["teacher"], of_all["tokens"], o["log_sums"], _dev(np.ones(all_rows)) if w is None else of_all["w"], dx,
                              log_rests=o["log_rests"] if rest else None, rest=rest, temperature=T)
    with np.errstate(invalid="ignore"):
        size_of_sums = np.abs(sums) + np.where(np.isfinite(rests), np.abs(rests), 0)
        saved = (p * (1 + left)[:, None] + share) * (U * 4 * (size_of_sums + 8) + np.abs(top) * U * 8)[:, None] * (wp / T)[:, None]
    _gradient_close(_host(dx[some]), want["gradient"], kind, np.nan_to_num(arithmetic + saved))
    logits.copy_(keep)
    return want


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab,K", [(1, 1, 1), (2, 9, 4), (3, 4099, 16), (1, 50021, 128), (70, 8192, 8), (1100, 333, 5), (2, 300001, 64), (5, 131, 128)])
def test_distill(gpu_lib, rows, vocab, K, rest, kind):
    r = np.random.default_rng(vocab)
    teacher, tokens = _teacher(rows, vocab, K, rest, vocab + K)
    w = r.uniform(-1, 2, rows)
    w[2::6] = 0
    _check_distill(gpu_lib, _logits(rows, vocab, kind, vocab), teacher, tokens, rest, w)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("T", [0.3, 2.0])
def test_distill_at_a_temperature(gpu_lib, T, rest, kind):
    teacher, tokens = _teacher(5, 6007, 20, rest, 3, T)
    _check_distill(gpu_lib, _logits(5, 6007, kind, 4), teacher, tokens, rest, None, T)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows", [2, 1200])
def test_distill_in_the_logits_place(gpu_lib, rows, rest, kind):
    teacher, tokens = _teacher(rows, 1501, 7, rest, 5)
    x = _logits(rows, 1501, kind, 6)
    _check_distill(gpu_lib, x, teacher, tokens, rest, None, 1.0, out=x)


@pytest.mark.parametrize("kind", TYPES)
def test_distill_masks_and_rows_without_a_teacher(gpu_lib, kind):
    """No place, no student, NaN on either side, a teacher's token that the student forbids, all others forbidden, all tokens the
    teacher's, a student whose rest is small."""
    import torch
    vocab, K = 3001, 6
    for rest in (False, True):
        teacher, tokens = _teacher(10, vocab, K, rest, 9, empty=False)
        x = _logits(10, vocab, kind, 11)
        tokens[0] = -1
        teacher[1] = -np.inf
        x[2] = -np.inf
        x[3, 70] = np.nan
        teacher[4, 2] = np.nan
        x[5, int(tokens[5, 1])] = -np.inf
        x[6] = -np.inf
        x[6, tokens[6].tolist()] = torch.arange(K, device="cuda").to(x.dtype)
        x[7, tokens[7].tolist()] += 18.0                     # the rest is some 10^-6
        x[8] = torch.finfo(x.dtype).min
        x[9, tokens[9].tolist()] = 0.0
        x[9, 0] = np.inf
        _check_distill(gpu_lib, x, teacher, tokens, rest)
        for r in range(10):
            _check_distill(gpu_lib, x[r:r + 1].clone(), teacher[r:r + 1], tokens[r:r + 1], rest)
    small = _logits(3, 5, kind, 12)
    every = np.tile(np.arange(5, dtype=np.int32), (3, 1))
    _check_distill(gpu_lib, small, np.log(np.full((3, 5), 0.15)), every, True)      # all tokens are the teacher's: no rest
    _check_distill(gpu_lib, small, np.zeros((3, 5)), every, False)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rest", [False, True])
def test_a_token_in_several_places(gpu_lib, rest, kind):
    r = np.random.default_rng(1)
    for rows, vocab in ((3, 4000), (600, 50)):
        tokens = r.integers(0, 9, (rows, 40)).astype(np.int32)
        teacher = np.log(r.dirichlet(np.ones(41), rows)[:, :40])
        _check_distill(gpu_lib, _logits(rows, vocab, kind, 2), teacher, tokens, rest)


def test_distill_of_a_vocabulary_that_is_marked_in_parts(gpu_lib):
    """More logits than are marked at once, by one workgroup and in segments."""
    teacher, tokens = _teacher(2, 1 << 20, 128, True, 13)
    tokens[1, :4] = [(1 << 17) - 1, 1 << 17, (1 << 18) - 5, (1 << 20) - 1]
    x = _logits(2, (1 << 20) + 3, "bf16", 14)
    _check_distill(gpu_lib, x[:, 3:], teacher, tokens, True)


# Of 16-bit logits, half as many of fp32: a size of each form that holds a row, or most of it, in registers (test_logits_plans.py checks which), one that
# does not, and two that are cut into segments.
HELD = [(3, 901), (2200, 2003), (3, 7001), (3, 15001), (3, 30001), (40, 60001), (70, 130001), (70, 133001), (66, 261001), (70, 270001),
        (3, 60001), (40, 130001)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab", HELD)
def test_loss_and_gradient_of_rows_in_registers(gpu_lib, rows, vocab, rest, kind):
    """At odd addresses; the teacher's tokens at both ends of a row, behind one another, in several places, and with the same low bits."""
    import torch
    vocab = vocab // 2 if kind == "fp32" else vocab
    some = np.unique(np.linspace(0, rows - 1, 12).astype(int))
    teacher, tokens = _teacher(rows, vocab, 100, rest, vocab + rows)
    tokens[:, :6] = [0, vocab - 1, 1, 2, 3, vocab // 2]
    tokens[1::3, 7] = vocab - 1
    if vocab > 1 << 15:
        tokens[:, 8] = 1 + (1 << 15)
        tokens[:, 9:13] = vocab // 2 + np.arange(4)
    wide = torch.zeros(rows, vocab + 5, dtype=_torch_type(kind), device="cuda")
    x = wide[:, 3:vocab + 3]
    x.copy_(_logits(rows, vocab, kind, vocab))
    w = np.linspace(-0.5, 2, rows)
    w[some[1]] = 0                    # a row that is left out, and one without a teacher
    teacher[some[2]] = -np.inf
    _check_distill(gpu_lib, x, teacher, tokens, rest, w, some=some)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab", [(3, 130001), (40, 60001), (70, 133001), (66, 261001), (33, 270001)])
def test_loss_and_gradient_of_long_rows_in_the_logits_place(gpu_lib, rows, vocab, rest, kind):
    """Held, held in part, in segments and in two passes."""
    vocab = vocab // 2 if kind == "fp32" else vocab
    some = np.array([0, 1, rows - 1])
    teacher, tokens = _teacher(rows, vocab, 33, rest, vocab)
    teacher[1] = -np.inf
    x = _logits(rows, vocab, kind, rows)
    _check_distill(gpu_lib, x, teacher, tokens, rest, None, 1.3 if not rest else 1.0, out=x, some=some)


@pytest.mark.parametrize("kind,rows,vocab", [("bf16", 700, 52001), ("fp16", 300, 131501), ("fp32", 300, 70001)])
def test_logits_that_no_cache_holds(gpu_lib, kind, rows, vocab):
    """More than 64 MiB of them, in all operators, padded rows between the others."""
    some = np.array([0, 1, 2, rows // 2, rows - 1])
    x = _logits(rows, vocab, kind, 21)
    targets = np.arange(rows) * 71 % vocab
    targets[1::4] = -1
    for count in (0, 9):
        want = _check(gpu_lib, x, targets, count, 0.8, some)
    forward = {k: np.zeros(rows) for k in ("log_sums", "entropies")}
    for k in forward:
        forward[k][some] = want[k]
    _check_backward(gpu_lib, x, targets, forward, np.linspace(-1, 1, rows), np.linspace(1, 2, rows), 0.8, some=some)
    for rest in (False, True):
        teacher, tokens = _teacher(rows, vocab, 9, rest, 22, 0.8)
        _check_distill(gpu_lib, x, teacher, tokens, rest, None, 0.8, some=some)


def test_distill_against_differences(gpu_lib):
    import torch
    q = gpu_lib
    x, T = _logits(2, 40, "fp32", 17), 0.8
    for rest in (False, True):
        teacher, tokens = _teacher(2, 40, 6, rest, 18, T, empty=False)
        w = _as(np.float32, [1.0, -0.5])

        def losses(y, dx=None):
            o = torch.empty(2, device="cuda")
            q.quamba_distill_loss(y, _dev(teacher), _dev(tokens, np.int32), o, weights=_dev(w), grad_logits=dx, rest=rest, temperature=T)
            return _host(o) * w
        dx = torch.empty_like(x)
        losses(x, dx)
        for r, v in ((0, 3), (0, int(tokens[0, 1])), (1, int(tokens[1, 0])), (1, 39)):
            value = []
            for step in (0.03, -0.03):
                y = x.clone()
                y[r, v] += step
                value.append(losses(y)[r])
            assert abs((value[0] - value[1]) / 0.06 - float(dx[r, v])) <= 0.03 ** 2 * 4 / T ** 3 / 6 + 2 * 2.0 ** -22 * 10 / 0.06


# ---------------------------------------------------------------- together, in graphs and on streams


@pytest.mark.parametrize("rows", [3, 1100])
def test_a_teachers_answers_to_a_students_gradient_in_a_graph(gpu_lib, rows):
    """The teacher's log probabilities and tokens go into the distance, its log sums into the gradient, in the logits' place: captured on
    a stream of its own and replayed over changing logits, against the eager calls, and the last against the oracle."""
    import torch
    q = gpu_lib
    vocab, K, T = 5003, 12, 1.7
    teacher, student, work = (torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    targets = torch.arange(rows, dtype=torch.int32, device="cuda") - 1
    f = lambda *s: torch.zeros(*s, device="cuda")
    chosen, best, tokens, losses, sums, rests, weights = f(rows), f(rows, K), f(rows, K).int(), f(rows), f(rows), f(rows), f(rows) + 0.5
    gradient = torch.zeros_like(student)
    spaces = [torch.empty(max(16, n), dtype=torch.uint8, device="cuda") for n in (q.quamba_token_logprobs_workspace_size(rows, vocab, K),
                                                                                 q.quamba_distill_loss_workspace_size(rows, vocab, K))]

    def step():
        q.quamba_token_logprobs(teacher, targets, chosen, top_logprobs=best, top_tokens=tokens, temperature=T, workspace=spaces[0])
        q.quamba_distill_loss(student, best, tokens, losses, log_sums=sums, log_rests=rests, weights=weights, grad_logits=gradient, rest=True,
                              temperature=T, workspace=spaces[1])
        work.copy_(student)
        q.quamba_distill_backward(work, best, tokens, sums, weights, work, log_rests=rests, rest=True, temperature=T)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    outs = (chosen, best, tokens, losses, sums, rests, gradient, work)
    for seed in range(4):
        teacher.copy_(_logits(rows, vocab, "bf16", seed))
        student.copy_(_logits(rows, vocab, "bf16", seed + 50))
        graph.replay()
        got = [t.clone() for t in outs]
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))
    assert float((gradient.float() - work.float()).abs().max()) <= 2.0 ** -8 * float(gradient.float().abs().max())
    n = min(rows, 20)
    want = oracle.ref_token_logprobs(_host(teacher[:n]), targets[:n].cpu().numpy(), K, T)
    assert np.array_equal(tokens[:n].cpu().numpy(), want["top_tokens"])
    assert np.isneginf(best[0].cpu().numpy()).all() and float(losses[0]) == 0 and not gradient[0].any()
    _check_distill(q, student[:n].clone(), best[:n].cpu().numpy(), tokens[:n].cpu().numpy(), True, np.full(n, 0.5), T)


def test_two_streams_with_a_workspace_each(gpu_lib):
    import torch
    q = gpu_lib
    x = [_logits(4, 60001, "bf16", s) for s in range(2)]
    want = [_run(q, v, [1, 2, 3, 4], 16) for v in x]
    streams = [torch.cuda.Stream() for _ in range(2)]
    size = q.quamba_token_logprobs_workspace_size(4, 60001, 16)
    spaces = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [(torch.empty(4, device="cuda"), torch.empty(4, 16, device="cuda"), torch.empty(4, 16, dtype=torch.int32, device="cuda")) for _ in range(2)]
    targets = _dev([1, 2, 3, 4], np.int32)
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            q.quamba_token_logprobs(x[i], targets, outs[i][0], top_logprobs=outs[i][1], top_tokens=outs[i][2], workspace=spaces[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i][2], want[i]["top_tokens"])
        assert torch.allclose(outs[i][0], want[i]["logprobs"], atol=1e-5, rtol=0) and torch.allclose(outs[i][1], want[i]["top_logprobs"], atol=1e-5, rtol=0)
