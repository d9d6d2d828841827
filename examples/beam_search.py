"""Beam search with a Mamba2-shaped language model of random weights: projections in 8-bit floating point, the scan, its states and
the convolution in int8.

    python examples/beam_search.py --config m2_130m --layers 24 --batch 8 --beams 4 --tokens 64

The prompts go through the model once, whole (projections with many rows, the chunked scan).  Then every sequence holds `beams`
hypotheses, and a step of all of them is: projections with batch x beams rows, convolution and scan for a single token on their
cached states, the vocabulary's logits, the selection of the best continuations, and the move of the cached states to the
hypotheses that go on.  The step is recorded into a HIP graph once and replayed for every token."""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2503_22879_amd as q
import workloads as W

IN_SCALE, Z_SCALE = 4.5 / 127, 6.0 / 127  # of the convolution's input and of the gate's branch


class Weight:
    """A projection [n, k] as e4m3 codes with a scale for each square of 128 x 128."""

    def __init__(self, w):
        n, k = w.shape
        self.n, self.k = n, k
        self.codes = torch.empty(n, k, dtype=torch.float8_e4m3fn, device=w.device)
        self.scales = torch.empty(-(-n // 128), -(-k // 128), device=w.device)
        q.quamba_fp8_quantize(w, self.codes, self.scales, block_rows=128)

    def __call__(self, x, dtype):
        rows = x.shape[0]
        codes = torch.empty(rows, self.k, dtype=torch.float8_e4m3fn, device=x.device)
        scales = torch.empty(rows, -(-self.k // 128), device=x.device)
        q.quamba_fp8_quantize(x, codes, scales)
        y = torch.empty(rows, self.n, dtype=dtype, device=x.device)
        size = q.quamba_fp8_matmul_workspace_size(rows, self.n, self.k)
        space = torch.empty(size, dtype=torch.uint8, device=x.device) if size else None
        q.quamba_fp8_matmul(codes, scales, self.codes, self.scales, y, workspace=space)
        return y


def normed(x):
    x = x.float()
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5)


def codes(x, scale):
    return (x.float() * (1 / scale)).round().clamp(-128, 127).to(torch.int8)


class Layer:
    def __init__(self, s, d_model, draw):
        inner, states = s.nheads * s.headdim, s.ngroups * s.d_state
        self.split = [inner, inner + 2 * states, s.nheads]
        self.project_in = Weight(draw(sum(self.split), d_model) * d_model ** -0.5)
        self.project_out = Weight(draw(d_model, inner) * inner ** -0.5)
        weight = draw(self.split[1], 4) * 0.5
        w_scale = float(weight.abs().max()) / 127
        self.conv, self.conv_bias, self.conv_scale = codes(weight, w_scale), draw(self.split[1]) * 0.3, IN_SCALE * w_scale
        self.A, self.D = -torch.exp(draw(s.nheads)), draw(s.nheads)
        self.dt_bias = draw(s.nheads) * 0.5 - 3
        self.state_scales = None
        # static scales from maxima that a calibration would give; random weights are in any order, so in the sorted one as well
        x_max = 3 * torch.exp(0.3 * draw(s.nheads, s.headdim))
        b_max, c_max = (3 * torch.exp(0.3 * draw(s.ngroups, s.d_state)) for _ in range(2))
        self.host = q.quamba_reorder_params(s.nheads, s.headdim, s.ngroups, s.m, s.n, s.d_state,
                                            *(v.cpu().numpy() for v in (x_max, b_max, c_max)))[2]
        self.scales = q.DeviceScales(self.host)


class BeamSearch:
    """`tokens`, `scores`, `finished` [batch, beams] are the hypotheses' last tokens, their log-probabilities and whether they have
    ended; `parents` which hypotheses of the step before they go on from."""

    def __init__(self, s: W.LayerShape, layers: int, batch: int, beams: int, vocab: int, end_token: int = 0, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda *size: torch.randn(*size, generator=g, device="cuda")
        self.s, self.batch, self.beams, self.vocab, self.end_token = s, batch, beams, vocab, end_token
        self.d_model = s.nheads * s.headdim // 2
        self.embedding = draw(vocab, self.d_model).bfloat16()
        self.head = Weight(draw(vocab, self.d_model) * (4 * self.d_model ** -0.5))
        self.layers = [Layer(s, self.d_model, draw) for _ in range(layers)]
        channels = self.layers[0].split[1]
        self.states = [torch.empty(batch, beams, s.nheads, s.headdim, s.d_state, dtype=torch.int8, device="cuda") for _ in range(layers)]
        self.windows = [torch.empty(batch, beams, 3, channels, dtype=torch.int8, device="cuda") for _ in range(layers)]
        self.scores = torch.zeros(batch, beams, device="cuda")
        self.tokens, self.parents = (torch.zeros(batch, beams, dtype=torch.int32, device="cuda") for _ in range(2))
        self.finished = torch.zeros(batch, beams, dtype=torch.bool, device="cuda")
        self.logits, self.graph = None, None

    def shape(self, rows, length):
        s = self.s
        return q.Shape(batch=rows, seqlen=length, nheads=s.nheads, headdim=s.headdim, d_state=s.d_state, ngroups=s.ngroups, chunk=s.chunk,
                       n_head_clusters=s.m, n_chan_clusters=s.n, flags=0)

    def block(self, layer, h, rows, length, before, window, scan):
        """One layer on h [rows * length, d_model]; scan(x, B, C, dt, gate, y) enqueues the recurrence.  `before`: the convolution's
        last inputs, None at a sequence's start; `window` receives them."""
        s = self.s
        z, xBC, dt = layer.project_in(normed(h), torch.float16).split(layer.split, dim=-1)
        dt = F.softplus(dt.float() + layer.dt_bias).view(rows, length, s.nheads)
        heads, groups = (rows, length, s.nheads, s.headdim), (rows, length, s.ngroups, s.d_state)
        x, B, C = (torch.empty(size, dtype=torch.int8, device="cuda") for size in (heads, groups, groups))
        q.quamba_conv1d_q8(self.shape(rows, length), layer.scales, codes(xBC, IN_SCALE).view(rows, length, -1), layer.conv, layer.conv_bias,
                           layer.conv_scale, x, B, C, conv_state_in=before, conv_state_out=window)
        y = torch.empty(heads, dtype=torch.float16, device="cuda")
        scan(x, B, C, dt, q.Gate(z=codes(z, Z_SCALE).view(heads), z_scale=Z_SCALE), y)
        return h + layer.project_out(normed(y.view(rows * length, -1)), torch.bfloat16)

    def prompt(self, prompts):
        """prompts [batch, length]: fills the states and selects every sequence's first tokens."""
        (batch, length), s = prompts.shape, self.s
        shape = self.shape(batch, length)
        space = torch.empty(max(16, q.quamba_ssd_prefill_workspace_size(shape)), dtype=torch.uint8, device="cuda")
        h = F.embedding(prompts, self.embedding).view(batch * length, -1)
        for layer, states, windows in zip(self.layers, self.states, self.windows):
            final = torch.empty(batch, s.nheads, s.headdim, s.d_state, device="cuda")
            window = torch.empty(batch, 3, layer.split[1], dtype=torch.int8, device="cuda")
            h = self.block(layer, h, batch, length, None, window, lambda x, B, C, dt, gate, y: q.quamba_ssd_prefill(
                shape, layer.scales, x, B, C, dt, layer.A, layer.D, None, y, final, workspace=space, gate=gate))
            if layer.state_scales is None:  # of the 8-bit states, with room above what the first prompts leave
                most = 2 * final.abs().amax(0).cpu().numpy() + np.float32(1e-3)
                layer.state_scales = torch.from_numpy(q.quamba_state_scales(
                    s.nheads, s.headdim, s.ngroups, s.m, s.n, s.d_state, layer.host.head_cluster_end, layer.host.chan_cluster_end, most)).cuda()
            quantized = torch.empty(final.shape, dtype=torch.int8, device="cuda")
            q.quamba_ssd_quantize_state(shape, layer.scales, layer.state_scales, final, quantized)
            states.copy_(quantized[:, None].expand_as(states))
            windows.copy_(window[:, None].expand_as(windows))
        logits = self.head(normed(h.view(batch, length, -1)[:, -1]), torch.float32).view(batch, 1, self.vocab)
        self.finished.zero_()
        self.select(logits, torch.zeros(batch, 1, device="cuda"), torch.zeros(batch, 1, dtype=torch.bool, device="cuda"))

    def select(self, logits, scores, finished):
        """The best continuations over hypotheses and vocabulary; they become the hypotheses."""
        batch, beams, vocab = logits.shape
        space = torch.empty(q.quamba_beam_select_workspace_size(batch, beams, vocab, self.beams), dtype=torch.uint8, device="cuda")
        best = torch.empty_like(self.scores)
        q.quamba_beam_select(logits, scores, best, self.parents, self.tokens, space, finished=finished, pad_token=self.end_token)
        self.scores.copy_(best)
        self.finished.copy_(finished.gather(1, self.parents.long()) | (self.tokens == self.end_token))
        self.logits = logits

    def advance(self):
        """The logits [batch, beams, vocab] behind the hypotheses' last tokens; their states go on by these."""
        rows = self.batch * self.beams
        shape = self.shape(rows, 1)
        h = F.embedding(self.tokens.view(rows), self.embedding)
        for layer, states, windows in zip(self.layers, self.states, self.windows):
            window = windows.view(rows, 3, -1)
            h = self.block(layer, h, rows, 1, window, window, lambda x, B, C, dt, gate, y: q.quamba_ssd_decode_step_q8(
                shape, layer.scales, layer.state_scales, x[:, 0], B[:, 0], C[:, 0], dt[:, 0], layer.A, layer.D,
                states.view(rows, *states.shape[2:]), y[:, 0], gate=q.Gate(z=gate.z[:, 0], z_scale=gate.z_scale)))
        return self.head(normed(h), torch.float32).view(self.batch, self.beams, self.vocab)

    def eager_step(self):
        self.select(self.advance(), self.scores, self.finished)
        q.quamba_beam_reorder(self.parents, self.states + self.windows)

    def record(self):
        """Record the step into a graph.  The recording runs nothing; the run in front of it is taken back."""
        kept = [self.scores, self.tokens, self.parents, self.finished, *self.states, *self.windows]
        saved = [t.clone() for t in kept]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.eager_step()
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.eager_step()
        for t, before in zip(kept, saved):
            t.copy_(before)

    def step(self):
        self.graph.replay() if self.graph else self.eager_step()

    def generate(self, prompts, count, use_graph=True):
        """The `count` next tokens [batch, beams, count] of every hypothesis, best first, and their log-probabilities."""
        self.prompt(prompts)
        if use_graph and self.graph is None:
            self.record()
        parents = torch.empty(count, *self.parents.shape, dtype=torch.int64, device="cuda")
        tokens = torch.empty_like(parents)
        for t in range(count):
            if t:
                self.step()
            parents[t], tokens[t] = self.parents, self.tokens
        out, at = torch.empty_like(tokens), torch.arange(self.beams, device="cuda").expand(self.batch, -1)
        for t in reversed(range(count)):
            out[t] = tokens[t].gather(1, at)
            at = parents[t].gather(1, at)
        return out.permute(1, 2, 0).contiguous(), self.scores.clone()


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--config", default="m2_130m", choices=sorted(W.CONFIGS))
    p.add_argument("--layers", type=int, default=24)
    p.add_argument("--batch", type=int, default=8)
    p.add_argument("--beams", type=int, default=4)
    p.add_argument("--prompt", type=int, default=512)
    p.add_argument("--tokens", type=int, default=64)
    p.add_argument("--vocab", type=int, default=50021)
    p.add_argument("--no-graph", action="store_true")
    a = p.parse_args()
    torch.manual_seed(0)
    search = BeamSearch(W.CONFIGS[a.config], a.layers, a.batch, a.beams, a.vocab)
    prompts = torch.randint(1, a.vocab, (a.batch, a.prompt), device="cuda")
    search.generate(prompts, 3, not a.no_graph)  # first launches, recording
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    search.prompt(prompts)
    torch.cuda.synchronize()
    t1 = time.perf_counter()
    for _ in range(a.tokens):
        search.step()
    torch.cuda.synchronize()
    t2 = time.perf_counter()
    tokens, scores = search.generate(prompts, a.tokens, not a.no_graph)
    print(f"{a.config}, {a.layers} layers, {a.batch} prompts of {a.prompt} tokens: {1e3 * (t1 - t0):.2f} ms; "
          f"{a.beams} hypotheses each: {1e6 * (t2 - t1) / a.tokens:.0f} us a token" + ("" if a.no_graph else " (graph)"))
    for b in range(min(2, a.batch)):
        print(f"  sequence {b}: best {scores[b, 0].item():.2f}, tokens {tokens[b, 0, :12].tolist()}")


if __name__ == "__main__":
    main()
