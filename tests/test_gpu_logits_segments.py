"""GPU parity of rows of logits that are cut into segments, whose sums and best tokens a second launch joins: masks, ties, order, padding, addresses,
streams and graphs, with a workspace that is not empty; and of sums that are whole numbers, which show every logit that is lost or counted twice, in
every form."""
import numpy as np
import pytest

import oracle
from test_gpu_logits import TYPES, U, _as, _check, _check_distill, _dev, _gradient_close, _host, _logits, _run, _teacher, _torch_type
from test_gpu_logits_far import FORMS, STEPS

pytestmark = pytest.mark.gpu

VOCAB = 120001      # is cut for 10 rows of each type, with alternatives and without (test_logits_plans_of_segments.py)


def _of(x, kind):
    import torch
    return torch.from_numpy(np.asarray(x, np.float32)).cuda().to(_torch_type(kind))


def _is_cut(q, rows, vocab, count):
    assert q.quamba_token_logprobs_workspace_size(rows, vocab, count) > 0


# ---------------------------------------------------------------- what a segment may hold


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("count", [0, 1, 20, 128])
def test_masks(gpu_lib, count, kind):
    """Every logit forbidden, all but those of some segments, all but one, the type's lowest value in part and throughout, NaN and infinity in the first
    and the last segment, logits far below 0, one far above."""
    import torch
    _is_cut(gpu_lib, 10, VOCAB, count)
    x = _logits(10, VOCAB, kind, 8)
    low = torch.finfo(x.dtype).min
    x[0] = -np.inf
    x[1, :60000] = -np.inf
    x[1, 80000:] = -np.inf
    x[2, 3:] = low
    x[3] = low
    x[4, 77] = np.nan
    x[5, VOCAB - 2] = np.inf
    x[6] -= 10000 if kind != "fp16" else 1000
    x[7, VOCAB - 1] = 60000.0
    x[8, :VOCAB - 11] = -np.inf
    x[9] = -np.inf
    x[9, 4321] = low
    targets = [3, 70000, 2, 9000, 5, 8999, 17, 0, 5, 4321]
    _check(gpu_lib, x, targets, count)
    for r in (1, 5, 8, 9):
        _check(gpu_lib, x[r:r + 1], [targets[r]], count)
    _check(gpu_lib, x, targets, count, 0.5)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("count", [1, 9, 128])
def test_ties(gpu_lib, count, kind):
    """Few different logits, one, zeros of both signs, and the best alike on both sides of every segment's border: the lowest tokens first."""
    _is_cut(gpu_lib, 7, VOCAB, count)
    r, v = np.random.default_rng(5), np.arange(VOCAB)
    rows = [r.integers(0, 3, VOCAB), np.zeros(VOCAB), np.full(VOCAB, -3.0), np.where(r.random(VOCAB) < 0.5, 0.0, -0.0),
            np.where(v < VOCAB - 3, -0.0, 0.0), np.where(v % 1000 == 999, 1.0, -2.0), np.where(v % 8 == 7, 2.0, np.where(v % 8 == 0, 2.0, 1.0))]
    _check(gpu_lib, _of(np.stack(rows), kind), [0] * 7, count)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("count", [0, 1, 8, 128])
def test_rows_in_order(gpu_lib, count, kind):
    _is_cut(gpu_lib, 8, VOCAB, count)
    x = _logits(8, VOCAB, kind, 21)
    x[0] = x[0].sort().values
    x[1] = x[1].sort(descending=True).values
    x[2, VOCAB - 101:] += 30
    x[3, :100] += 30
    x[4] = x[4].sort().values * 100
    x[5] = x[5].sort(descending=True).values * 100
    x[6, 35000:] = -np.inf
    x[7] = (x[7] * 4).round()
    _check(gpu_lib, x, [VOCAB - 1, 0, VOCAB - 51, 99, VOCAB - 1, 0, 1, 1], count)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("count", [0, 6])
@pytest.mark.parametrize("left", [0, 1, 5])
def test_padding_among_rows_at_odd_addresses(gpu_lib, left, count, kind):
    """Padding holds NaN, and what lies between the rows is infinite; the last logits of a row stand in a vector of their own."""
    import torch
    for vocab in (VOCAB, VOCAB + 7):
        _is_cut(gpu_lib, 9, vocab, count)
        wide = torch.full((9, vocab + 13), float("inf"), dtype=_torch_type(kind), device="cuda")
        x = wide[:, left:left + vocab]
        x.copy_(_logits(9, vocab, kind, 9))
        targets = [0, vocab - 1, -1, vocab // 2, vocab, 1, -2 ** 31, 2, 2 ** 31 - 1]
        x[2::2] = float("nan")
        x[3:9:2, vocab - 1] = 25.0
        _check(gpu_lib, x, targets, count)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rest", [False, True])
def test_distill_masks_and_rows_without_a_teacher(gpu_lib, rest, kind):
    import torch
    q, vocab, K = gpu_lib, VOCAB + 2, 6
    assert q.quamba_distill_loss_workspace_size(10, vocab, K) > 16 * 10
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
    x[7, tokens[7].tolist()] += 18.0
    x[8] = torch.finfo(x.dtype).min
    x[9, tokens[9].tolist()] = 0.0
    x[9, 0] = np.inf
    _check_distill(q, x, teacher, tokens, rest)
    _check_distill(q, x, teacher, tokens, rest, np.linspace(-1, 1, 10), out=x)
    for r in (1, 6, 7):
        _check_distill(q, x[r:r + 1].clone(), teacher[r:r + 1], tokens[r:r + 1], rest)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rest", [False, True])
def test_distill_padding_at_odd_addresses(gpu_lib, rest, kind):
    """A teacher's tokens at the row's ends and on both sides of every multiple of 512 vectors, some of them twice."""
    import torch
    vocab, K = VOCAB + 4, 128
    per = 4 if kind == "fp32" else 8
    teacher, tokens = _teacher(6, vocab, K, rest, 12)
    edges = np.arange(1, vocab // (512 * per)) * 512 * per
    at = np.concatenate([[0, 1, vocab - 1, vocab - 2], edges - 4, edges - 3, edges - 1, edges])[:100]
    tokens[1::2, :len(at)] = at
    tokens[3, len(at)] = at[0]
    wide = torch.full((6, vocab + 9), float("nan"), dtype=_torch_type(kind), device="cuda")
    x = wide[:, 3:3 + vocab]
    x.copy_(_logits(6, vocab, kind, 13))
    w = [1.0, -1.0, 0.0, 0.5, 2.0, 1.0]
    x[2] = float("nan")
    _check_distill(gpu_lib, x[:], teacher, tokens, rest, w)


# ---------------------------------------------------------------- sums that are whole numbers


def _allowed(vocab, kind):
    """Eight rows of tokens that may come: all, every second by chance, one in a hundred, those at borders of threads, waves and segments wherever the row
    begins, every other vector, the last, the first, a middle part."""
    r, v, per = np.random.default_rng(vocab), np.arange(vocab), 4 if kind == "fp32" else 8
    vector = v // per
    return np.stack([v >= 0, r.random(vocab) < 0.5, (r.random(vocab) < 0.01) | (v == 7), np.isin(vector % 64, (0, 1, 63)) & (v % 3 == 0),
                     vector % 2 == 0, v == vocab - 1, v == 0, (v >= vocab // 3) & (v < vocab // 2)])


def _equal_logits(rows, vocab, kind, left):
    """0 where a token may come and -infinity elsewhere, at addresses `left` logits behind a multiple of 16 bytes."""
    import torch
    ok = _allowed(vocab, kind)
    wide = torch.full((rows, (vocab + left + 15) // 8 * 8), float("nan"), dtype=_torch_type(kind), device="cuda")
    x = wide[:, left:left + vocab]
    x.copy_(torch.from_numpy(np.where(ok, 0.0, -np.inf).astype(np.float32)).cuda().to(x.dtype).repeat((rows + 7) // 8, 1)[:rows])
    return x, ok


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("count", [0, 9])
@pytest.mark.parametrize("rows,vocab", FORMS + [(600, 2049), (520, 9001)])
def test_no_logit_is_lost_or_counted_twice(gpu_lib, rows, vocab, count, kind):
    """Every exponential is 1 and their sum a whole number below 2^24, so exact in any order; its logarithm is good to two units (four half steps) and is what
    all values are, but for the sign."""
    for left in (0, 3):
        x, ok = _equal_logits(rows, vocab, kind, left)
        n, targets = ok.sum(1), np.resize(ok.argmax(1), rows)
        most = 4 * U * np.log(n)
        for workspace in (True, False):
            for everything in (True, False):
                got = {k: v[:8].cpu().numpy() for k, v in _run(gpu_lib, x, targets, count, 1.0, workspace, everything).items()}
                assert (np.abs(got["logprobs"] + np.log(n)) <= most).all()
                if everything:
                    for name in ("log_sums", "entropies"):
                        assert (np.abs(got[name] - np.log(n)) <= most).all(), name
                for r in range(8 if count else 0):
                    best = np.nonzero(ok[r])[0][:count]
                    assert got["top_tokens"][r].tolist() == best.tolist() + [-1] * (count - len(best))
                    assert (np.abs(got["top_logprobs"][r, :len(best)] + np.log(n[r])) <= most[r]).all()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab", STEPS + [(1100, 2003), (33, 270001)])
def test_no_logit_is_lost_or_counted_twice_by_the_distance(gpu_lib, rows, vocab, rest, kind):
    """As above, with four tokens of a teacher (one that may not come counts 0 of the sums) and their rest; the gradient of p = 1 / n."""
    import torch
    q = gpu_lib
    vocab = vocab // 2 if kind == "fp32" else vocab
    for left in (0, 3):
        x, ok = _equal_logits(rows, vocab, kind, left)
        first, last = ok.argmax(1), vocab - 1 - ok[:, ::-1].argmax(1)
        # two that may come, where there are two, an empty place, and one of the first's once more
        tokens = np.stack([first, last, np.full(8, -1), first], 1).astype(np.int32)
        log_q = np.log(np.tile([0.25, 0.25, 0.5, 0.125], (8, 1))).astype(np.float32)
        named = 1 + (first != last)
        n = ok.sum(1)
        Q = _as(np.float64, [0.25, 0.25, 0.0, 0.125]) / (1.0 if rest else 0.625)
        others = n - named
        left_ = np.where(others > 0, 0.375, 0.0) if rest else np.zeros(8)
        with np.errstate(divide="ignore"):
            log_rest = np.log(others)
        losses = (Q * np.log(np.where(Q > 0, Q, 1))).sum() + Q.sum() * np.log(n) + np.where(left_ > 0, left_ * (np.log(0.375) - np.where(others > 0, log_rest, 0) + np.log(n)), 0)
        at, t = (_dev(np.tile(v, ((rows + 7) // 8, 1))[:rows], d) for v, d in ((tokens, np.int32), (log_q, np.float32)))
        dx_want = np.where(ok, ((1.0 * (Q.sum() + left_)) / n)[:, None], 0.0)
        for r in range(8):
            is_named = np.isin(np.arange(vocab), (first[r], last[r]))
            np.add.at(dx_want[r], [first[r], last[r], first[r]], -Q[[0, 1, 3]])
            if left_[r] > 0:
                dx_want[r] -= np.where(ok[r] & ~is_named, left_[r] / others[r], 0)
        # q to 16 half steps, p to 8; values that cancel are a sum of terms of that size
        arithmetic = U * 40 * (np.where(ok, 1 / n[:, None], 0) + np.where(ok & (others > 0)[:, None], 1 / np.maximum(others, 1)[:, None], 0))
        for r in range(8):
            arithmetic[r, [first[r], last[r]]] += U * 40
        size = q.quamba_distill_loss_workspace_size(rows, vocab, 4)
        for workspace in (True, False):
            space = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if workspace else None
            for step in (False, True):
                got, sums, rests = (torch.full((rows,), 7.0, device="cuda") for _ in range(3))
                dx = torch.full_like(x, 3.0) if step else None
                q.quamba_distill_loss(x, t, at, got, log_sums=sums, log_rests=rests, grad_logits=dx, rest=rest, workspace=space)
                assert (np.abs(_host(sums)[:8] - np.log(n)) <= 4 * U * np.log(n)).all()
                if rest:
                    assert np.array_equal(np.isneginf(_host(rests)[:8]), others == 0)
                    some = others > 0
                    assert (np.abs(_host(rests)[:8][some] - log_rest[some]) <= 4 * U * log_rest[some]).all()
                # q (ln q - ln p) of four places and the rest: eight roundings each of values up to ln n
                assert (np.abs(_host(got)[:8] - losses) <= U * 16 * (np.log(n) + 3)).all(), np.abs(_host(got)[:8] - losses).max()
                if step:
                    _gradient_close(_host(dx[:8]), dx_want, kind, arithmetic)
        dx = torch.full_like(x, 3.0)
        q.quamba_distill_backward(x, t, at, sums, _dev(np.ones(rows)), dx, log_rests=rests if rest else None, rest=rest)
        # the log sums' rounding is a factor of p
        _gradient_close(_host(dx[:8]), dx_want, kind, arithmetic * (1 + np.log(n))[:, None])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,vocab", [(8, 403), (8, 9001), (8, 130001), (320, 120001)])
def test_no_logit_is_lost_or_counted_twice_by_the_gradient(gpu_lib, rows, vocab, kind):
    """Of the log probability and, 0 for equal logits, the entropy."""
    import torch
    for left in (0, 3):
        x, ok = _equal_logits(rows, vocab, kind, left)
        n, target = ok.sum(1), ok.argmax(1)
        log_n = np.resize(np.log(n), rows).astype(np.float32)
        for h in (None, np.ones(rows, np.float32)):
            dx = torch.full_like(x, 3.0)
            gpu_lib.quamba_token_logprobs_backward(x, _dev(np.resize(target, rows), np.int32), _dev(log_n), _dev(np.ones(rows)), dx,
                                                   entropies=None if h is None else _dev(log_n), grad_entropies=_dev(h))
            want = np.where(ok, -1 / n[:, None], 0.0)
            want[np.arange(8), target] += 1
            # p from a log sum that is rounded, ln p + entropy from two; 1 - p
            arithmetic = U * 16 * (np.where(ok, 1 / n[:, None], 0) * (1 + np.log(n))[:, None] + (np.arange(vocab) == target[:, None]))
            _gradient_close(_host(dx[:8]), want, kind, arithmetic)


# ---------------------------------------------------------------- in graphs and on streams


def test_two_streams_with_a_workspace_each(gpu_lib):
    """Of two launches a call, whose workspaces hold what the first leaves to the second."""
    import torch
    q, vocab, K = gpu_lib, 130001, 16
    x = [_logits(4, vocab, "bf16", s) for s in range(2)]
    targets = _dev([1, 2, 3, 4], np.int32)
    teacher, tokens = (_dev(v, d) for v, d in zip(_teacher(4, vocab, K, True, 3), (np.float32, np.int32)))
    sizes = q.quamba_token_logprobs_workspace_size(4, vocab, K), q.quamba_distill_loss_workspace_size(4, vocab, K)
    assert sizes[0] > 0 and sizes[1] > 16 * 4
    f = lambda *s: torch.zeros(*s, device="cuda")

    def outputs():
        return dict(p=f(4), best=f(4, K), at=f(4, K).int(), losses=f(4), sums=f(4), rests=f(4), gradient=torch.zeros_like(x[0]))

    def step(i, o, spaces, stream):
        q.quamba_token_logprobs(x[i], targets, o["p"], top_logprobs=o["best"], top_tokens=o["at"], workspace=spaces[0], stream=stream)
        q.quamba_distill_loss(x[i], teacher, tokens, o["losses"], log_sums=o["sums"], log_rests=o["rests"], grad_logits=o["gradient"], rest=True,
                              workspace=spaces[1], stream=stream)
    space = lambda: [torch.full((s,), 0xFF, dtype=torch.uint8, device="cuda") for s in sizes]
    want, spaces = [outputs() for _ in range(2)], space()
    for i in range(2):
        step(i, want[i], spaces, None)
    streams, mine, got = [torch.cuda.Stream() for _ in range(2)], [space() for _ in range(2)], [outputs() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            step(i, got[i], mine[i], streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(got[i][k], want[i][k]) for k in want[i])
        h = oracle.ref_token_logprobs(_host(x[i]), [1, 2, 3, 4], K)
        assert np.array_equal(want[i]["at"].cpu().numpy(), h["top_tokens"])


def test_two_graphs_that_share_a_workspace(gpu_lib):
    """A teacher's answers into a student's gradient, each call in two launches, captured twice over one workspace and replayed in turn on a stream, with
    eager calls between; every replay against the eager result, bit for bit."""
    import torch
    q, rows, vocab, K, T = gpu_lib, 3, 130001, 12, 1.7
    sizes = q.quamba_token_logprobs_workspace_size(rows, vocab, K), q.quamba_distill_loss_workspace_size(rows, vocab, K)
    assert sizes[0] > 0 and sizes[1] > 16 * rows
    spaces = [torch.full((s,), 0xFF, dtype=torch.uint8, device="cuda") for s in sizes]
    f = lambda *s: torch.zeros(*s, device="cuda")
    targets = torch.arange(rows, dtype=torch.int32, device="cuda") - 1
    weights = f(rows) + 0.5

    class Chain:
        def __init__(self):
            self.teacher, self.student, self.work = (torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda") for _ in range(3))
            self.gradient = torch.zeros_like(self.student)
            self.p, self.best, self.at, self.losses, self.sums, self.rests = f(rows), f(rows, K), f(rows, K).int(), f(rows), f(rows), f(rows)
            self.in_place = f(rows)

        def step(self):
            q.quamba_token_logprobs(self.teacher, targets, self.p, top_logprobs=self.best, top_tokens=self.at, temperature=T, workspace=spaces[0])
            q.quamba_distill_loss(self.student, self.best, self.at, self.losses, log_sums=self.sums, log_rests=self.rests, weights=weights,
                                  grad_logits=self.gradient, rest=True, temperature=T, workspace=spaces[1])
            self.work.copy_(self.student)
            q.quamba_distill_loss(self.work, self.best, self.at, self.in_place, weights=weights, grad_logits=self.work, rest=True, temperature=T,
                                  workspace=spaces[1])

        def outs(self):
            return self.p, self.best, self.at, self.losses, self.sums, self.rests, self.gradient, self.work, self.in_place
    side, chains, graphs = torch.cuda.Stream(), [Chain(), Chain()], []
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for c in chains:
            c.step()
    torch.cuda.synchronize()
    for c in chains:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.step()
        graphs.append(graph)
    for seed in range(4):
        for i, c in enumerate(chains):
            c.teacher.copy_(_logits(rows, vocab, "bf16", seed + 10 * i))
            c.student.copy_(_logits(rows, vocab, "bf16", seed + 50 + 10 * i))
        for g in graphs:
            g.replay()
        got = [[t.clone() for t in c.outs()] for c in chains]
        torch.cuda.synchronize()
        for c in chains:
            c.step()
        torch.cuda.synchronize()
        for c, mine in zip(chains, got):
            assert all(torch.equal(a, b) for a, b in zip(mine, c.outs()))
    for c in chains:
        want = oracle.ref_token_logprobs(_host(c.teacher), targets.cpu().numpy(), K, T)
        assert np.array_equal(c.at.cpu().numpy(), want["top_tokens"])
        assert float(c.losses[0]) == 0 and not c.gradient[0].any() and not c.work[0].any()
        _check_distill(q, c.student.clone(), c.best.cpu().numpy(), c.at.cpu().numpy(), True, np.full(rows, 0.5), T)
