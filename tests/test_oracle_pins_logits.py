"""Pins of oracle/logits.py: torch's own log softmax, entropy and divergence in float64, gradients by autograd and by differences, closed
forms, and the rows that have no distribution."""
import numpy as np
import pytest
import torch

import oracle


def _rows(rows, vocab, seed, spread=2.0):
    return np.random.default_rng(seed).standard_normal((rows, vocab)) * spread


@pytest.mark.parametrize("temperature", [1.0, 0.4, 3.0])
def test_logprobs_against_torch(temperature):
    x = _rows(5, 40, 0)
    x[1, 3:9] = -np.inf
    targets = np.array([0, 3, 39, 7, 12])
    got = oracle.ref_token_logprobs(x, targets, 6, temperature)
    t = torch.from_numpy(x) / temperature
    log_p = torch.log_softmax(t, 1)
    assert np.array_equal(np.isneginf(got["logprobs"]), [False, True, False, False, False])
    fin = [0, 2, 3, 4]
    assert np.abs(got["logprobs"][fin] - log_p[fin, targets[fin]].numpy()).max() < 1e-13
    assert np.abs(got["log_sums"] - torch.logsumexp(t, 1).numpy()).max() < 1e-13
    assert np.abs(got["entropies"] - torch.distributions.Categorical(logits=t.clamp(min=-1e30)).entropy().numpy()).max() < 1e-12
    best, tokens = torch.topk(log_p, 6, dim=1)
    assert np.abs(got["top_logprobs"] - best.numpy()).max() < 1e-13 and np.array_equal(got["top_tokens"], tokens.numpy())


def test_uniform_rows_ties_and_short_lists():
    x = np.zeros((2, 8))
    x[1, 3:] = -np.inf
    got = oracle.ref_token_logprobs(x, [2, 0], 5)
    assert np.allclose(got["entropies"], [np.log(8), np.log(3)]) and np.allclose(got["logprobs"], [-np.log(8), -np.log(3)])
    assert got["top_tokens"].tolist() == [[0, 1, 2, 3, 4], [0, 1, 2, -1, -1]] and np.isneginf(got["top_logprobs"][1, 3:]).all()


def test_rows_without_a_distribution_and_padding():
    x = _rows(5, 9, 1)
    x[0], x[1, 4], x[2, 4] = -np.inf, np.nan, np.inf
    got = oracle.ref_token_logprobs(x, [1, 1, 1, -1, 9], 2)
    for k in ("logprobs", "log_sums", "entropies"):
        assert np.isnan(got[k][:3]).all() and (got[k][3:] == 0).all()
    assert (got["top_tokens"] == -1).all() and np.isneginf(got["top_logprobs"]).all()


@pytest.mark.parametrize("temperature", [1.0, 0.4, 3.0])
def test_gradient_of_logprobs_and_entropy(temperature):
    x, targets = _rows(4, 30, 2), np.array([5, -1, 0, 29])
    r = np.random.default_rng(3)
    g, h = r.standard_normal(4), r.standard_normal(4)
    f = oracle.ref_token_logprobs(x, targets, 0, temperature)
    dx = oracle.ref_token_logprobs_backward(x, targets, f["log_sums"], f["entropies"], g, h, temperature)
    assert (dx[1] == 0).all()
    t = torch.from_numpy(x).requires_grad_()
    log_p = torch.log_softmax(t / temperature, 1)
    live = torch.tensor([0, 2, 3])
    value = (torch.from_numpy(g)[live] * log_p[live, torch.from_numpy(targets)[live]] - torch.from_numpy(h)[live] * (log_p.exp() * log_p).sum(1)[live]).sum()
    value.backward()
    assert np.abs(dx - t.grad.numpy()).max() < 1e-13

    def total(v):
        o = oracle.ref_token_logprobs(v, targets, 0, temperature)
        return (g * o["logprobs"] + h * o["entropies"]).sum()
    for r, v in ((0, 5), (0, 6), (2, 0), (3, 11)):
        d = np.zeros_like(x)
        d[r, v] = 1e-5
        assert abs((total(x + d) - total(x - d)) / 2e-5 - dx[r, v]) < 1e-8


@pytest.mark.parametrize("temperature", [1.0, 2.5])
def test_distance_over_the_whole_vocabulary_is_the_divergence(temperature):
    x, t = _rows(3, 17, 4), _rows(3, 17, 5)
    tokens = np.stack([np.random.default_rng(i).permutation(17) for i in range(3)])
    teacher = np.take_along_axis(t, tokens, 1)
    log_q = torch.log_softmax(torch.from_numpy(t) / temperature, 1)
    log_p = torch.log_softmax(torch.from_numpy(x) / temperature, 1)
    want = torch.nn.functional.kl_div(log_p, log_q, log_target=True, reduction="none").sum(1).numpy()
    assert np.abs(oracle.ref_distill(x, teacher, tokens, False, None, temperature)["losses"] - want).max() < 1e-12
    # with nothing left to a rest
    teacher = np.take_along_axis(log_q.numpy(), tokens, 1)
    assert np.abs(oracle.ref_distill(x, teacher, tokens, True, None, temperature)["losses"] - want).max() < 1e-12


@pytest.mark.parametrize("rest", [False, True])
def test_distance_zero_cross_entropy_and_weights(rest):
    x = _rows(4, 20, 6)
    log_p = torch.log_softmax(torch.from_numpy(x), 1).numpy()
    tokens = np.tile(np.arange(5), (4, 1))
    out = oracle.ref_distill(x, log_p[:, :5], tokens, rest, [1, 0, 1, 1])
    if rest:  # the teacher is the model
        assert np.abs(out["losses"]).max() < 1e-14 and np.abs(out["gradient"]).max() < 1e-15
    assert out["losses"][1] == 0 and (out["gradient"][1] == 0).all()
    one = oracle.ref_distill(x, np.zeros((4, 1)), np.full((4, 1), 3), rest)
    want = -log_p[:, 3]
    assert np.abs(one["losses"] - want).max() < 1e-13
    assert np.abs(one["gradient"] - (np.exp(log_p) - np.eye(20)[3])).max() < 1e-13


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("temperature", [1.0, 0.6])
def test_gradient_of_the_distance(rest, temperature):
    """By differences, with empty places and a token that stands in two of them."""
    r = np.random.default_rng(7)
    x = _rows(3, 15, 8)
    tokens = np.array([[3, 4, 4, 9, -1], [0, 14, 5, 15, 6], [1, 2, 3, 4, 5]])
    teacher = np.log(r.dirichlet(np.ones(7), 3)[:, :5])
    teacher[2, 1] = -np.inf
    w = np.array([1.0, 0.3, -2.0])
    out = oracle.ref_distill(x, teacher, tokens, rest, w, temperature)

    def total(v):
        return (w * oracle.ref_distill(v, teacher, tokens, rest, w, temperature)["losses"]).sum()
    for i in range(3):
        for v in range(15):
            d = np.zeros_like(x)
            d[i, v] = 1e-5
            assert abs((total(x + d) - total(x - d)) / 2e-5 - out["gradient"][i, v]) < 1e-8


def test_rows_without_places_and_without_a_distribution():
    x = _rows(5, 9, 9)
    x[2, 1] = np.nan
    tokens = np.array([[-1, 9], [1, 2], [1, 2], [1, 2], [1, 2]])
    teacher = np.zeros((5, 2))
    teacher[1] = -np.inf
    teacher[3, 0] = np.nan
    x[4, 1] = -np.inf
    out = oracle.ref_distill(x, teacher, tokens)
    assert (out["losses"][:2] == 0).all() and (out["gradient"][:2] == 0).all()
    assert np.isnan(out["losses"][2:4]).all() and np.isnan(out["gradient"][2:4]).all()
    assert out["losses"][4] == np.inf and np.isfinite(out["gradient"][4]).all()
