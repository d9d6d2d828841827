"""The beam search of examples/beam_search.py: its choices against float64, its hypotheses against the same tokens run without a
selection or a move of states, and the recorded step against the eager one."""
import os
import sys

import numpy as np
import pytest

import workloads as W

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

SHAPES = [(W.CONFIGS["tiny"], 2, 3, 5, 1003, 33), (W.CONFIGS["m2_130m"], 2, 2, 4, 4099, 130), (W.CONFIGS["tiny"], 1, 24, 4, 515, 1)]


def _search(s, layers, batch, beams, vocab, seed=3):
    from beam_search import BeamSearch
    return BeamSearch(s, layers, batch, beams, vocab, end_token=1, seed=seed)


def _prompts(batch, length, vocab):
    import torch
    return torch.from_numpy(np.random.default_rng(length).integers(2, vocab, (batch, length))).cuda()


@pytest.mark.parametrize("s,layers,batch,beams,vocab,length", SHAPES)
def test_choices_and_hypotheses(gpu_lib, s, layers, batch, beams, vocab, length):
    """Every step's scores are the best sums of the step before and the log-probabilities of the logits, within fp32's rounding of the
    sums (a few units of 2^-24 of up to 60, and the sum of exponentials to some 2^-20).  A hypothesis' tokens, run from the prompt in
    the place that its states ended in, give the logits that it was scored by, bit for bit, wherever it came from."""
    import torch
    steps = 6
    search = _search(s, layers, batch, beams, vocab)
    prompts = _prompts(batch, length, vocab)
    search.prompt(prompts)
    history = [(search.parents.cpu().numpy(), search.tokens.cpu().numpy(), None)]
    for _ in range(steps):
        scores, finished = search.scores.double().cpu(), search.finished.cpu()
        search.eager_step()
        logp = torch.log_softmax(search.logits.double().cpu(), -1) + scores[..., None]
        ended = torch.full_like(logp, -np.inf)
        ended[..., 1] = scores
        total = torch.where(finished[..., None], ended, logp)
        best = total.view(batch, -1).topk(beams).values
        parents, tokens = search.parents.long().cpu(), search.tokens.long().cpu()
        got = search.scores.double().cpu()
        chosen = total[torch.arange(batch)[:, None], parents, tokens]
        assert (got - best).abs().max() < 5e-5 and (got - chosen).abs().max() < 5e-5
        assert all(len(set(zip(p.tolist(), t.tolist()))) == beams for p, t in zip(parents, tokens))
        history.append((parents.numpy(), tokens.numpy(), search.logits.cpu().numpy()))
    assert any((p != np.arange(beams)).any() for p, _, _ in history[1:])              # states did move
    # each place's own past
    at = np.tile(np.arange(beams), (batch, 1))
    forced, rows = [None] * (steps + 1), [None] * (steps + 1)
    for t in reversed(range(steps + 1)):
        forced[t] = np.take_along_axis(history[t][1], at, 1)
        at = np.take_along_axis(history[t][0], at, 1)
        rows[t] = at
    search.prompt(prompts)
    for t in range(1, steps + 1):
        search.tokens.copy_(torch.from_numpy(forced[t - 1]))
        logits = search.advance().cpu().numpy()
        for b in range(batch):
            for k in range(beams):
                assert np.array_equal(logits[b, k], history[t][2][b, rows[t][b, k]]), (t, b, k)


@pytest.mark.parametrize("s,layers,batch,beams,vocab,length", SHAPES)
def test_recorded_step(gpu_lib, s, layers, batch, beams, vocab, length):
    """Replays of the graph, with eager work between them, leave what eager steps leave, bit for bit; a second prompt as well."""
    import torch
    eager, recorded = (_search(s, layers, batch, beams, vocab) for _ in range(2))
    for prompts in (_prompts(batch, length, vocab), _prompts(batch, length + 3, vocab)):
        eager.prompt(prompts)
        recorded.prompt(prompts)
        if recorded.graph is None:
            recorded.record()
        for t in range(5):
            eager.eager_step()
            recorded.step()
            torch.cuda.synchronize()
            for name in ("scores", "parents", "tokens", "finished"):
                assert torch.equal(getattr(eager, name), getattr(recorded, name)), (t, name)
            for a, b in zip(eager.states + eager.windows, recorded.states + recorded.windows):
                assert torch.equal(a, b), t


def test_generate(gpu_lib):
    """The hypotheses that are read back: best first, and none twice."""
    search = _search(W.CONFIGS["tiny"], 2, 4, 6, 777)
    tokens, scores = search.generate(_prompts(4, 20, 777), 9)
    assert tokens.shape == (4, 6, 9) and (scores[:, :-1] >= scores[:, 1:]).all()
    assert all(len({tuple(h) for h in sequence.tolist()}) == 6 for sequence in tokens)
