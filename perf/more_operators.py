"""The operators on what a model answers, its logits, as measurable cases: log probabilities of given tokens with the entropy and the
most likely alternatives, their gradients, and the distance from a teacher that is known by its most likely tokens, with its
gradient.  A quantized model is scored, served and brought back towards the model it was made from with them.

Vocabularies are generic sizes; rows are the tokens of a step (1 to some hundred sequences) or of prompts and training batches.

Plain forms, with z = x / T and log_sum = max z + log sum exp(z - max z) of a row of logits x:
  logprob = z[target] - log_sum        entropy = -sum p log p, p = exp(z - log_sum)
  top: the largest logits, ties to the lowest token, as z - log_sum
  their gradient: dx = (g ([v = target] - p) - h p (log p + entropy)) / T
  loss = sum over the teacher's places of q (log q - log p[token]), q its probabilities, made to sum to 1 or with the rest of both
  distributions as one more outcome: + q_rest (log q_rest - log p_rest), p_rest the sum over all other tokens
  its gradient: dx = w (p sum q - q [token] - q_rest p / p_rest [other token]) / T
A row whose target is no token, or whose weight is 0, is padding: zeros, and no alternatives (-inf, -1).
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}
PADDING = 1 / 16                # share of the rows that are padding, from 16 rows on
MAX_READ = 8192 * 128000        # logits of the largest listed call that only reads them
MAX_WRITTEN = 4096 * 128000     # of the largest that also writes a gradient


def listed():
    return [
        # What a server returns beside one sequence's next token: a call that is mostly launch, ...
        dict(name="logprobs 1x50021 top 8", kind="logprobs", rows=1, vocab=50021, type="bf16", top=8, entropy=False, masked=False, temperature=1.0),
        # ... beside those of a serving batch whose tokens are constrained, from fp32 logits, with the entropy, ...
        dict(name="logprobs 64x128000 top 20", kind="logprobs", rows=64, vocab=128000, type="fp32", top=20, entropy=True, masked=True, temperature=0.7),
        # ... the score of a prompt batch (perplexity, multiple choice): log probabilities alone, an odd vocabulary, ...
        dict(name="score 2048x50021", kind="logprobs", rows=2048, vocab=50021, type="bf16", top=0, entropy=False, masked=False, temperature=1.0),
        # ... and a corpus' tokens with everything, which is also how a teacher's answers are kept.
        dict(name="logprobs 8192x128000 top 5", kind="logprobs", rows=8192, vocab=128000, type="bf16", top=5, entropy=True, masked=False, temperature=1.0),
        # Gradients of chosen tokens' log probabilities and of the entropy (a policy's update) of a few sequences, ...
        dict(name="backward 300x50021 entropy", kind="logprobs_backward", rows=300, vocab=50021, type="fp16", entropy=True, temperature=1.0),
        # ... and of a training batch.
        dict(name="backward 4096x128000", kind="logprobs_backward", rows=4096, vocab=128000, type="bf16", entropy=False, temperature=1.0),
        # How far a quantized model is from its teacher: at the tokens of one step, ...
        dict(name="distill 16x50021 of 16", kind="distill", rows=16, vocab=50021, type="fp32", places=16, rest=False, temperature=1.0),
        # ... and over prompts, by the true probabilities of the teacher's most likely tokens and the rest of them.
        dict(name="distill 2048x128000 of 64 rest", kind="distill", rows=2048, vocab=128000, type="bf16", places=64, rest=True, temperature=1.0),
        # Loss and gradient in one step of a training: a small vocabulary's, ...
        dict(name="distill step 24x8192 of 8", kind="distill_step", rows=24, vocab=8192, type="fp32", places=8, rest=False, temperature=1.0),
        # ... an odd one's at a softened temperature, ...
        dict(name="distill step 512x50021 of 32", kind="distill_step", rows=512, vocab=50021, type="fp16", places=32, rest=False, temperature=2.0),
        # ... a large batch's, ...
        dict(name="distill step 4096x128000 of 64", kind="distill_step", rows=4096, vocab=128000, type="bf16", places=64, rest=True, temperature=1.0),
        # ... and the gradient alone, where the loss goes on into something else first.
        dict(name="distill backward 1000x50021", kind="distill_backward", rows=1000, vocab=50021, type="bf16", places=20, rest=True, temperature=1.0),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["logprobs", "logprobs", "logprobs_backward", "distill", "distill_step", "distill_step", "distill_backward"])
    vocab = _log(rng, 500, 200000)
    if rng.random() < 0.5:
        vocab = (vocab + 7) // 8 * 8
    most = MAX_READ if kind in ("logprobs", "distill") else MAX_WRITTEN
    case = dict(kind=kind, rows=_log(rng, 1, min(16384, most // vocab)), vocab=vocab, type=rng.choice(sorted(TYPES)),
                temperature=rng.choice([1.0, 1.0, 0.7, 2.0]))
    if kind == "logprobs":
        case.update(top=rng.choice([0, 1, 5, 20, 64]), entropy=rng.random() < 0.5, masked=rng.random() < 0.3)
    elif kind == "logprobs_backward":
        case.update(entropy=rng.random() < 0.5)
    else:
        case.update(places=_log(rng, 1, 128), rest=rng.random() < 0.5)
    return case


# ---------------------------------------------------------------- inputs


class _Draw:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda")

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda")

    def below(self, n, *shape):
        return torch.randint(n, shape, generator=self.g, device="cuda")


def _logits(d, case, places):
    """Sharp next-token distributions: a normal field, and `places` likely tokens of each row above it.  Their tokens and their
    values in falling order come as well."""
    rows, vocab = case["rows"], case["vocab"]
    x = d.normal(rows, vocab).mul_(2.0)
    each = vocab // places
    tokens = each * torch.arange(places, device="cuda") + d.below(each, rows, places)
    tokens = tokens.gather(1, d.uniform(rows, places).argsort(1))
    values = (7.0 + 3.0 * d.normal(rows, places)).sort(1, descending=True).values
    x.scatter_(1, tokens, values + 0.5 * d.normal(rows, places))
    return x, tokens, values


def _padding(d, rows):
    """Which rows are padding."""
    return (d.uniform(rows) < PADDING) & torch.tensor(rows >= 16, device="cuda")


def _library():
    """This repository's package, where its operators are to be run."""
    if not own:
        return None
    import paper_2503_22879_amd as q
    return q


def _space(size):
    return torch.empty(size, dtype=torch.uint8, device="cuda") if size else None


def _log_sums(x, temperature):
    return torch.logsumexp(x.double() / temperature, 1)


def _prepare_logprobs(case, d):
    rows, vocab = case["rows"], case["vocab"]
    x, likely, _ = _logits(d, case, 8)
    targets = torch.where(d.uniform(rows) < 0.8, likely.gather(1, d.below(8, rows, 1))[:, 0], d.below(vocab, rows))
    if case.get("masked"):  # tokens that a grammar forbids; the chosen one is allowed
        allowed = x.gather(1, targets[:, None])
        x = torch.where(d.uniform(rows, vocab) < 0.3, -math.inf, x).scatter_(1, targets[:, None], allowed)
    x = x.to(TYPES[case["type"]])
    padding = _padding(d, rows)
    state = dict(logits=x, targets=torch.where(padding, -1, targets).to(torch.int32))
    if case["kind"] == "logprobs":
        top = case["top"]
        state.update(logprobs=torch.empty(rows, device="cuda"), log_sums=torch.empty(rows, device="cuda"),
                     entropies=torch.empty(rows, device="cuda") if case["entropy"] else None,
                     top_logprobs=torch.empty((rows, top), device="cuda") if top else None,
                     top_tokens=torch.empty((rows, top), dtype=torch.int32, device="cuda") if top else None, workspace=None)
        lib = _library()
        if lib is not None:  # what a program that calls the library keeps for it
            state["workspace"] = _space(lib.quamba_token_logprobs_workspace_size(rows, vocab, top))
        return state
    log_sums = _log_sums(x, case["temperature"])
    z = x.double() / case["temperature"] - log_sums[:, None]
    state.update(log_sums=torch.where(padding, 0.0, log_sums).float(), grad_logprobs=d.normal(rows), grad_logits=torch.empty_like(x),
                 entropies=None, grad_entropies=None)
    if case["entropy"]:
        entropies = -(torch.exp(z) * z).sum(1)
        state.update(entropies=torch.where(padding, 0.0, entropies).float(), grad_entropies=0.1 * d.normal(rows))
    return state


def _prepare_distill(case, d):
    rows, vocab, K, T = case["rows"], case["vocab"], case["places"], case["temperature"]
    x, tokens, values = _logits(d, case, K)
    if case["rest"]:  # log probabilities at the temperature: what the teacher leaves to other tokens is one to thirty per cent
        left = torch.exp(math.log(0.01) + math.log(30.0) * d.uniform(rows, 1))
        values = torch.log_softmax(values.double() / T, 1).float() + torch.log1p(-left)
    # some of the teacher's lists are shorter
    ends = torch.where(d.uniform(rows) < 0.1, 1 + d.below(K, rows), K)
    empty = torch.arange(K, device="cuda") >= ends[:, None]
    weights = torch.where(_padding(d, rows), 0.0, 0.5 + d.uniform(rows))
    x = x.to(TYPES[case["type"]])
    state = dict(logits=x, teacher=torch.where(empty, -math.inf, values), tokens=torch.where(empty, -1, tokens).to(torch.int32), weights=weights,
                 rest=case["rest"], workspace=None, grad_logits=None)
    if case["kind"] == "distill_backward":
        inside = torch.zeros_like(x, dtype=torch.bool).scatter_(1, tokens, True)
        inside &= ~torch.zeros_like(inside).scatter_(1, tokens, empty)
        state.update(log_sums=_log_sums(x, T).float(), log_rests=None, grad_logits=torch.empty_like(x))
        if case["rest"]:
            state["log_rests"] = _log_sums(torch.where(inside, -math.inf, x.float()), T).float()
        return state
    state.update(losses=torch.empty(rows, device="cuda"), log_sums=None)
    if case["kind"] == "distill_step":
        state["grad_logits"] = torch.empty_like(x)
    lib = _library()
    if lib is not None:
        state["workspace"] = _space(lib.quamba_distill_loss_workspace_size(rows, vocab, K))
    return state


def prepare(case, seed):
    d = _Draw(seed)
    state = (_prepare_logprobs if case["kind"].startswith("logprobs") else _prepare_distill)(case, d)
    state.update(kind=case["kind"], temperature=case["temperature"])
    return state


# ---------------------------------------------------------------- one pass


def _softmax_parts(z):
    """(max, exp(z - max), its sum), of rows."""
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    return top, e, e.sum(1, keepdim=True)


def _largest(x, count):
    """Tokens of the `count` largest values of rows x, ties to the lowest token."""
    bits = x.view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7fffffff, bits).to(torch.int64)
    key = order * (1 << 32) + (x.shape[1] - 1 - torch.arange(x.shape[1], device=x.device))
    return x.shape[1] - 1 - (torch.topk(key, count, dim=1).values & 0xffffffff)


def _plain_logprobs(s):
    x = s["logits"].float() + 0.0
    z = x / s["temperature"]
    padding = s["targets"] < 0
    top, e, total = _softmax_parts(z)
    log_total = torch.log(total)
    target = s["targets"].clamp(min=0).long()[:, None]
    out = dict(logprobs=torch.where(padding, 0.0, ((z.gather(1, target) - top) - log_total)[:, 0]),
               log_sums=torch.where(padding, 0.0, (top + log_total)[:, 0]))
    if s["entropies"] is not None:
        weighted = torch.where(e > 0, e * (z - top), 0.0).sum(1, keepdim=True)
        out["entropies"] = torch.where(padding, 0.0, (log_total - weighted / total)[:, 0])
    if s["top_tokens"] is not None:
        tokens = _largest(x, s["top_tokens"].shape[1])
        out["top_logprobs"] = torch.where(padding[:, None], -math.inf, (z.gather(1, tokens) - top) - log_total)
        out["top_tokens"] = torch.where(padding[:, None], -1, tokens).to(torch.int32)
    return out


def _plain_logprobs_backward(s):
    z = s["logits"].float() / s["temperature"]
    log_p = z - s["log_sums"][:, None]
    p = torch.exp(log_p)
    padding = (s["targets"] < 0)[:, None]
    g = s["grad_logprobs"][:, None]
    dx = -g * p
    dx.scatter_add_(1, s["targets"].clamp(min=0).long()[:, None], g)
    if s["entropies"] is not None:
        dx -= s["grad_entropies"][:, None] * torch.where(p > 0, p * (log_p + s["entropies"][:, None]), 0.0)
    return torch.where(padding, 0.0, dx / s["temperature"]).to(s["logits"].dtype)


def _teacher(s):
    """Probabilities of the teacher's places, their tokens (of empty places: 0, at probability 0) and which places are none."""
    t = s["teacher"]
    valid = (s["tokens"] >= 0) & (t > -math.inf)
    if s["rest"]:
        q = torch.exp(t)
    else:
        q = torch.exp((t - t.amax(1, keepdim=True)) / s["temperature"])
        q = q / q.sum(1, keepdim=True)
    return torch.where(valid, q, 0.0), s["tokens"].clamp(min=0).long(), valid


def _plain_distill(s):
    """(losses, gradient)"""
    z = s["logits"].float() / s["temperature"]
    q, tokens, valid = _teacher(s)
    counted = s["weights"][:, None] != 0
    if s["kind"] == "distill_backward":
        log_sum = s["log_sums"][:, None]
        p = torch.exp(z - log_sum)
    else:
        top, e, total = _softmax_parts(z)
        p = e / total
    whole = q.sum(1, keepdim=True)
    inside = torch.zeros_like(z).scatter_add_(1, tokens, valid.float()) > 0
    left, share = torch.zeros_like(whole), None
    if s["rest"]:
        left = (1.0 - whole).clamp(min=0)
        if s["kind"] == "distill_backward":
            share = torch.where(inside, 0.0, torch.exp(z - s["log_rests"][:, None]))
        else:
            outside = torch.where(inside, 0.0, e)
            other = outside.sum(1, keepdim=True)
            share = outside / other
        whole = whole + left
    losses = None
    if s["kind"] != "distill_backward":
        log_p = (z.gather(1, tokens) - top) - torch.log(total)
        losses = torch.where(q > 0, q * (torch.log(q) - log_p), 0.0).sum(1, keepdim=True)
        if s["rest"]:
            losses = losses + torch.where(left > 0, left * (torch.log(left) - (torch.log(other) - torch.log(total))), 0.0)
        losses = torch.where(counted, losses, 0.0)[:, 0]
    if s["grad_logits"] is None:
        return losses
    dx = (p * whole).scatter_add_(1, tokens, -q)
    if s["rest"]:
        dx -= left * share
    dx = torch.where(counted, dx * (s["weights"][:, None] / s["temperature"]), 0.0).to(s["logits"].dtype)
    return dx if losses is None else (losses, dx)


def _plain(s):
    if s["kind"] == "logprobs":
        return _plain_logprobs(s)
    if s["kind"] == "logprobs_backward":
        return _plain_logprobs_backward(s)
    return _plain_distill(s)


def _call(s):
    import paper_2503_22879_amd as q
    T = s["temperature"]
    if s["kind"] == "logprobs":
        q.quamba_token_logprobs(s["logits"], s["targets"], s["logprobs"], log_sums=s["log_sums"], entropies=s["entropies"],
                                top_logprobs=s["top_logprobs"], top_tokens=s["top_tokens"], temperature=T, workspace=s["workspace"])
        return {k: s[k] for k in ("logprobs", "log_sums", "entropies", "top_logprobs", "top_tokens") if s[k] is not None}
    if s["kind"] == "logprobs_backward":
        q.quamba_token_logprobs_backward(s["logits"], s["targets"], s["log_sums"], s["grad_logprobs"], s["grad_logits"],
                                         entropies=s["entropies"], grad_entropies=s["grad_entropies"], temperature=T)
        return s["grad_logits"]
    if s["kind"] == "distill_backward":
        q.quamba_distill_backward(s["logits"], s["teacher"], s["tokens"], s["log_sums"], s["weights"], s["grad_logits"],
                                  log_rests=s["log_rests"], rest=s["rest"], temperature=T)
        return s["grad_logits"]
    q.quamba_distill_loss(s["logits"], s["teacher"], s["tokens"], s["losses"], weights=s["weights"], grad_logits=s["grad_logits"],
                          rest=s["rest"], temperature=T, workspace=s["workspace"])
    return s["losses"] if s["grad_logits"] is None else (s["losses"], s["grad_logits"])


def run(state):
    return _call(state) if own else _plain(state)


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    rows, n = case["rows"], case["rows"] * case["vocab"]
    kept = 1.0 - PADDING if rows >= 16 else 1.0
    read = n * BYTES[case["type"]] * kept
    if case["kind"] == "logprobs":
        return {"bytes": read + rows * (12 + 4 * case["entropy"] + 8 * case["top"]), "flops": n * (4 + 2 * case["entropy"])}
    if case["kind"] == "logprobs_backward":
        return {"bytes": read + n * BYTES[case["type"]] + rows * (12 + 8 * case["entropy"]), "flops": n * (4 + 3 * case["entropy"])}
    teacher = rows * (8 * case["places"] + 8)
    if case["kind"] == "distill":
        return {"bytes": read + teacher, "flops": 4 * n}
    return {"bytes": read + n * BYTES[case["type"]] + teacher, "flops": n * (4 if case["kind"] == "distill_backward" else 7)}


# ---------------------------------------------------------------- the definitions in 64 bits


def _exact_logprobs(s):
    log_p = torch.log_softmax(s["logits"].double() / s["temperature"], 1)
    live = s["targets"] >= 0
    row = torch.arange(live.numel(), device=live.device)
    chosen = log_p[row, s["targets"].long() * live]
    out = dict(logprobs=chosen * live, log_sums=_log_sums(s["logits"], s["temperature"]) * live)
    if s["entropies"] is not None:
        out["entropies"] = -torch.xlogy(torch.exp(log_p), torch.exp(log_p)).sum(1) * live
    if s["top_tokens"] is not None:
        out["top_logprobs"] = torch.topk(log_p, s["top_tokens"].shape[1], dim=1).values.masked_fill(~live[:, None], -math.inf)
        out["top_tokens"] = None
    return out


def _exact_logprobs_backward(s):
    T, live = s["temperature"], s["targets"] >= 0
    log_p = s["logits"].double().div_(T).sub_(s["log_sums"].double()[:, None])
    slope = -s["grad_logprobs"].double()[:, None].expand_as(log_p)
    if s["entropies"] is not None:
        slope = slope - s["grad_entropies"].double()[:, None] * (log_p + s["entropies"].double()[:, None])
    dx = torch.exp(log_p).mul_(slope)
    rows = torch.nonzero(live)[:, 0]
    dx[rows, s["targets"].long()[rows]] += s["grad_logprobs"].double()[rows]
    return dx.mul_(live[:, None] / T)


def _exact_distill(s):
    T, rest = s["temperature"], s["rest"]
    z = s["logits"].double() / T
    rows, K = s["tokens"].shape
    live = (s["weights"] != 0).double()
    t = s["teacher"].double()
    q = torch.exp(t) if rest else torch.softmax(t / T, 1)
    # one outcome more than tokens holds what belongs to no place
    tokens = torch.where(s["tokens"] < 0, z.shape[1], s["tokens"].long())
    full = torch.zeros((rows, z.shape[1] + 1), dtype=torch.float64, device=z.device)
    target = full.clone().scatter_(1, tokens, q)[:, :-1]
    named = full.scatter_(1, tokens, 1.0)[:, :-1] > 0
    given = s["kind"] == "distill_backward"
    log_sum = s["log_sums"].double() if given else torch.logsumexp(z, 1)
    p = torch.exp(z - log_sum[:, None])
    left = torch.clamp(1.0 - q.sum(1), min=0.0) if rest else torch.zeros_like(live)
    if rest:
        log_rest = s["log_rests"].double() if given else torch.logsumexp(z.masked_fill(named, -math.inf), 1)
    losses = None
    if not given:
        losses = torch.special.xlogy(target, target).sum(1) - (target * torch.where(named, z - log_sum[:, None], 0.0)).sum(1)
        if rest:
            losses = losses + torch.special.xlogy(left, left) - left * (log_rest - log_sum)
        losses = losses * live
    if s["grad_logits"] is None:
        return losses
    dx = p * (q.sum(1) + left)[:, None] - target
    if rest:
        dx = dx - left[:, None] * torch.exp(z - log_rest[:, None]).masked_fill(named, 0.0)
    dx = dx * (live * s["weights"].double() / T)[:, None]
    return dx if given else (losses, dx)


def exact(case, seed):
    state = prepare(case, seed)
    return {"logprobs": _exact_logprobs, "logprobs_backward": _exact_logprobs_backward}.get(case["kind"], _exact_distill)(state)
