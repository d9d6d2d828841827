"""GPU parity of the beam selection (places exactly, values to fp32 rounding) and of the states' reordering (byte for byte),
through the C ABI, against plain loops in float64."""
import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu

TYPES = ("fp32", "fp16", "bf16")


def _torch_type(name):
    import torch
    return {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}[name]


def _select(q, logits, scores, finished, pad, count):
    import torch
    b, K, V = logits.shape
    out = torch.full((b, count), 5.0, device="cuda")
    parents, tokens = (torch.full((b, count), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    space = torch.full((max(16, q.quamba_beam_select_workspace_size(b, K, V, count)),), 0xFF, dtype=torch.uint8, device="cuda")
    q.quamba_beam_select(logits, torch.from_numpy(np.asarray(scores, np.float32)).cuda(), out, parents, tokens, space,
                         finished=None if finished is None else torch.from_numpy(np.asarray(finished)).cuda(), pad_token=pad)
    return out.double().cpu().numpy(), parents.cpu().numpy(), tokens.cpu().numpy()


def _tolerance(logits, scores, values):
    """fp32: the sum of exponentials is off by some 2^-21 of itself (its terms by about an ulp each, their arguments by half an
    ulp of up to 30), the differences and the final sum by half an ulp of their sizes."""
    size = np.where(np.isfinite(values), np.abs(values), 0)
    s = np.where(np.isfinite(scores), np.abs(scores), 0).max(axis=1, keepdims=True)
    return 2.0 ** -20 + 2.0 ** -22 * (size + 2 * s + 12)


def _check(q, logits, scores, finished=None, pad=0, count=4, gap=True):
    """`gap`: move the scores until different beams' best candidates are told apart by fp32 (ties of one beam stay)."""
    x = logits.float().cpu().numpy()
    scores = np.array(scores, np.float32)
    r = np.random.default_rng(7)
    for _ in range(100 if gap else 0):
        v, p, _ = oracle.ref_beam_select(x, scores, finished, pad, min(count + 1, x.shape[1] * x.shape[2]))
        with np.errstate(invalid="ignore"):
            near = ((v[:, :-1] - v[:, 1:] < 1e-4) & (p[:, :-1] != p[:, 1:]) & (v[:, 1:] > -np.inf)).any(axis=1)
        if not near.any():
            break
        scores[near] += r.uniform(-0.05, 0.05, scores[near].shape).astype(np.float32)
    want = oracle.ref_beam_select(x, scores, finished, pad, count)
    got = _select(q, logits, scores, finished, pad, count)
    assert np.array_equal(got[1], want[1]), (got[1], want[1])
    assert np.array_equal(got[2], want[2]), (got[2], want[2])
    fin = np.isfinite(want[0])
    assert np.array_equal(np.isfinite(got[0]), fin) and (got[0][~fin] == -np.inf).all()
    off = np.abs(got[0] - want[0], where=fin, out=np.zeros_like(want[0]))
    assert (off <= _tolerance(x, scores, want[0])).all(), off.max()
    return got


def _logits(b, K, V, kind, seed, spread=2.0):
    import torch
    r = np.random.default_rng(seed)
    return torch.from_numpy((r.standard_normal((b, K, V)) * spread).astype(np.float32)).cuda().to(_torch_type(kind))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("b,K,V,count", [(1, 1, 1, 1), (1, 1, 5, 3), (2, 3, 7, 40), (1, 4, 2048, 4), (3, 2, 2049, 5), (1, 1, 4097, 1),
                                         (2, 5, 10007, 10), (5, 16, 3001, 32), (1, 64, 515, 128), (2, 8, 50021, 16), (1, 2, 300000, 7)])
def test_select(gpu_lib, b, K, V, count, kind):
    r = np.random.default_rng(V)
    _check(gpu_lib, _logits(b, K, V, kind, V + K), -np.abs(r.standard_normal((b, K)) * 3), count=count)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_select_large_batch(gpu_lib, kind):
    """Long pieces of many rows, and the places of finished beams."""
    r = np.random.default_rng(1)
    b, K, V = 40, 8, 33001
    fin = (r.random((b, K)) < 0.3).astype(np.uint8)
    fin[0] = 1
    fin[1] = 0
    _check(gpu_lib, _logits(b, K, V, kind, 2), -5 - np.abs(r.standard_normal((b, K)) * 3), fin, pad=17, count=16)
    _check(gpu_lib, _logits(b, K, V, kind, 3), -5 - np.abs(r.standard_normal((b, K)) * 3), fin.astype(bool), pad=V - 1, count=8)


@pytest.mark.parametrize("kind", ["fp32", "fp16"])
@pytest.mark.parametrize("K,V,count", [(64, 30011, 128), (20, 70001, 128), (64, 264001, 3), (5, 3000, 128)])
def test_select_of_many_candidates(gpu_lib, K, V, count, kind):
    """Many pieces and many choices of a sequence: the best spread over all beams, all in one beam, all in one piece of one beam, and
    finished beams among the last ones whose candidates are the best."""
    x = _logits(1, K, V, kind, 31)
    r = np.random.default_rng(6)
    even = -3 - r.random((1, K))
    _check(gpu_lib, x, even, count=count)
    fin = np.zeros((1, K), np.uint8)
    fin[0, K - 1] = fin[0, K // 2] = 1
    _check(gpu_lib, x, even + 2 * fin, fin, pad=V - 1, count=count)
    if V > 100000:
        return
    alone = even - 60
    alone[0, K - 2] = -1.0
    _check(gpu_lib, x, alone, count=count)
    x[0, K - 2, V // 2:V // 2 + 200] += 12
    _check(gpu_lib, x, alone, count=count)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("count", [1, 8, 128])
def test_select_from_rows_in_order(gpu_lib, count, kind):
    """Many rows, each in few long pieces: rising logits (every piece better than all before it), falling ones, few different ones,
    one, and rows whose first piece is forbidden or that hold their best, or all that is allowed, at one end."""
    import torch
    b, V = 1024, 17003
    x = _logits(b, 1, V, kind, 21)
    x[::8] = x[::8].sort(dim=-1).values
    x[1::8] = x[1::8].sort(dim=-1, descending=True).values
    x[2::8] = x[2::8].round()
    x[3::8, :, :9000] = -float("inf")
    x[4::8, :, 12:] = -float("inf")
    x[5::8, :, :16990] = torch.finfo(x.dtype).min
    x[6::8] = 0.25
    x[7::8, :, 8000:] += 30
    _check(gpu_lib, x, np.full((b, 1), -1.0), count=count)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("V,count", [(1000, 6), (40000, 128), (2500, 65)])
def test_select_ties(gpu_lib, V, count, kind):
    """Few different logits, or one: the lowest tokens of the best; beams that are alike tie exactly and go by their number."""
    import torch
    r = np.random.default_rng(5)
    for x in (r.integers(0, 3, (2, 2, V)), np.zeros((2, 2, V)), np.full((2, 2, V), -3.0), np.where(r.random((2, 2, V)) < 0.5, 0.0, -0.0)):
        x[:, 1] = x[:, 0]
        t = torch.from_numpy(x.astype(np.float32)).cuda().to(_torch_type(kind))
        _check(gpu_lib, t, [[-1.0, -1.0], [-2.0, -2.5]], count=count, gap=False)


@pytest.mark.parametrize("kind", TYPES)
def test_select_masks(gpu_lib, kind):
    """Rows with every logit forbidden, with few allowed ones, with the type's lowest value for a mask (in part, throughout), NaN and
    infinity in a row, and a row whose largest logits lie far above the rest."""
    import torch
    b, K, V = 1, 8, 9001
    x = _logits(b, K, V, kind, 8)
    low = torch.finfo(x.dtype).min
    x[0, 0] = -np.inf
    x[0, 1, 5:] = -np.inf
    x[0, 2, 3:] = low
    x[0, 3] = low
    x[0, 4, 77] = np.nan
    x[0, 5, 8999] = np.inf
    x[0, 6] -= 10000 if kind != "fp16" else 1000
    x[0, 7, 9000] = 60000.0
    scores = [[-1.0, -2, -3, -4, -5, -6, -7, -30]]
    _check(gpu_lib, x, scores, count=30)
    for k in range(K):                                        # each alone, asked for more than the masks leave
        _check(gpu_lib, x[:, k:k + 1], [[scores[0][k]]], count=9)


def test_select_first_step_and_empty_places(gpu_lib):
    """One beam of a sequence holds a score, the others none; sequences that offer nothing at all."""
    s = np.full((4, 4), -np.inf, np.float32)
    s[0, 0] = 0.0
    s[1, 2] = -1.0
    s[2, 1], s[2, 3] = np.nan, np.inf
    x = _logits(4, 4, 777, "fp32", 4)
    _check(gpu_lib, x, s, count=8, gap=False)
    got = _check(gpu_lib, x, s, np.ones((4, 4), np.uint8), pad=3, count=8, gap=False)
    assert got[1][3].tolist() == [0, 1, 2, 3, 0, 1, 2, 3] and (got[2][3] == 3).all()


@pytest.mark.parametrize("kind", TYPES)
def test_select_from_a_padded_vocabulary(gpu_lib, kind):
    """Rows further apart than they are long, at odd addresses; what lies between is not read as logits."""
    import torch
    b, K, V = 3, 4, 5003
    wide = torch.full((b, K, V + 11), float("inf"), dtype=_torch_type(kind), device="cuda")
    wide[:, :, 7:7 + V] = _logits(b, K, V, kind, 9)
    r = np.random.default_rng(2)
    _check(gpu_lib, wide[:, :, 7:7 + V], -np.abs(r.standard_normal((b, K)) * 2), count=8)


def test_select_offsets_beyond_32_bits(gpu_lib):
    """Rows over 4 GiB from the first."""
    import torch
    far = 3 << 29
    wide = torch.empty(2 * far + 4000, dtype=torch.float16, device="cuda")
    x = wide.as_strided((1, 3, 4000), (3 * far, far, 1))
    x.copy_(_logits(1, 3, 4000, "fp16", 10))
    _check(gpu_lib, x, [[-3.0, -2.0, -1.5]], count=6)


def test_select_in_a_graph(gpu_lib):
    """Captured on a stream of its own and replayed over changing logits, against the eager call."""
    import torch
    b, K, V, count = 2, 4, 20011, 8
    x = torch.zeros(b, K, V, dtype=torch.bfloat16, device="cuda")
    scores = torch.tensor([[-1.0, -2, -3, -4]] * b, device="cuda")
    out, parents, tokens = torch.empty(b, count, device="cuda"), *(torch.empty(b, count, dtype=torch.int32, device="cuda") for _ in range(2))
    space = torch.empty(gpu_lib.quamba_beam_select_workspace_size(b, K, V, count), dtype=torch.uint8, device="cuda")
    call = lambda: gpu_lib.quamba_beam_select(x, scores, out, parents, tokens, space)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for seed in range(5):
        x.copy_(_logits(b, K, V, "bf16", seed))
        graph.replay()
        got = [t.clone() for t in (out, parents, tokens)]
        torch.cuda.synchronize()
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(g, t) for g, t in zip(got, (out, parents, tokens)))


def _parents(b, K, how, seed=0):
    r = np.random.default_rng(seed)
    if how == "same":
        return np.tile(np.arange(K), (b, 1))
    if how == "turn":
        return np.tile((np.arange(K) + 1) % K, (b, 1))
    if how == "first":
        return np.zeros((b, K), np.int64)
    p = r.integers(0, K, (b, K))
    if how == "outside":
        p = np.where(r.random((b, K)) < 0.3, r.choice([-1, K, 2 ** 31 - 1, -2 ** 31], (b, K)), p)
    return p


@pytest.mark.parametrize("how", ["same", "turn", "first", "random", "outside"])
@pytest.mark.parametrize("b,K", [(1, 1), (3, 2), (2, 3), (5, 4), (2, 7), (1, 16), (2, 33), (1, 64)])
def test_reorder(gpu_lib, b, K, how):
    """Caches of several types and lengths in one call, among them odd and empty ones and one at an odd address."""
    import torch
    r = np.random.default_rng(K)
    p = _parents(b, K, how, b + K)
    shapes = [(np.float32, (6, 8, 16)), (np.int8, (3, 1792)), (np.int8, (4099,)), (np.int8, (1,)), (np.float16, (5,)), (np.int8, (0,)),
              (np.int8, (12289,))]
    host = [r.integers(-100, 100, (b, K) + s).astype(t) for t, s in shapes]
    dev = [torch.from_numpy(h).cuda() for h in host]
    room = torch.full((b * K * 1001 + 64,), 3, dtype=torch.int8, device="cuda")      # at an odd address, something around it
    odd = r.integers(-100, 100, (b, K, 1001)).astype(np.int8)
    view = room[17:17 + odd.size].view(b, K, 1001)
    view.copy_(torch.from_numpy(odd))
    gpu_lib.quamba_beam_reorder(torch.from_numpy(p.astype(np.int32)).cuda(), dev + [view])
    for h, d in zip(host + [odd], dev + [view]):
        assert np.array_equal(d.cpu().numpy(), oracle.ref_beam_reorder(h, p))
    assert (room[:17] == 3).all() and (room[17 + odd.size:] == 3).all()


def test_reorder_more_caches_than_a_launch_takes(gpu_lib):
    import torch
    r = np.random.default_rng(3)
    p = _parents(3, 5, "random")
    host = [r.standard_normal((3, 5, 64 + i)).astype(np.float32) for i in range(70)]
    dev = [torch.from_numpy(h).cuda() for h in host]
    gpu_lib.quamba_beam_reorder(torch.from_numpy(p.astype(np.int32)).cuda(), tuple(dev))
    for h, d in zip(host, dev):
        assert np.array_equal(d.cpu().numpy(), oracle.ref_beam_reorder(h, p))
    gpu_lib.quamba_beam_reorder(torch.from_numpy(p.astype(np.int32)).cuda(), [])


def test_reorder_offsets_beyond_32_bits_and_many_sequences(gpu_lib):
    import torch
    n = (1 << 31) + 4099
    cache = torch.empty(1, 3, n, dtype=torch.int8, device="cuda")
    marks = [0, 4095, 1 << 20, (1 << 31) - 1, 1 << 31, n - 1]
    for k in range(3):
        cache[0, k].fill_(k + 1)
        cache[0, k, marks] = torch.tensor([10 * k + i for i in range(6)], dtype=torch.int8, device="cuda")
    gpu_lib.quamba_beam_reorder(torch.tensor([[2, 0, 0]], dtype=torch.int32, device="cuda"), [cache])
    for k, p in enumerate((2, 0, 0)):
        assert cache[0, k, marks].tolist() == [10 * p + i for i in range(6)]
        assert int(cache[0, k, 1 << 30]) == p + 1 and int(cache[0, k, (1 << 31) + 5]) == p + 1
    del cache
    b = 70000
    p = torch.randint(2, (b, 2), dtype=torch.int32, device="cuda")
    small = torch.randn(b, 2, 9, device="cuda")
    want = small[torch.arange(b, device="cuda")[:, None], p.long()].clone()
    gpu_lib.quamba_beam_reorder(p, [small])
    assert torch.equal(small, want)


@pytest.mark.parametrize("count", [1, 2, 3, 16])
@pytest.mark.parametrize("b", [1, 70])
def test_select_tells_candidates_of_a_beam_apart_by_their_logits(gpu_lib, b, count):
    """Logits of a beam that differ while their values round to the same fp32 number: the larger one comes first, in one piece of a row
    and across two, in short pieces (1 sequence) and in long ones (70)."""
    import torch
    V = 9001
    near = [1.0, 1.00001, 1.00002]
    for places in ((5, 77, 4000), (5, 5000, 8999), (8999, 5000, 5), (4095, 4096, 4097), (8191, 8192, 8193), (3, 2, 8500)):
        x = _logits(b, 1, V, "fp32", 41) - 20
        x[..., list(places)] = torch.tensor(near, device="cuda")
        _check(gpu_lib, x, np.full((b, 1), -1000.0), count=count, gap=False)


@pytest.mark.parametrize("b,K,V,count", [(1, 1, 20011, 128), (100, 1, 20011, 128), (1, 1, 20011, 7), (100, 1, 20011, 7), (3, 3, 50, 120),
                                         (1, 1, 4096, 40), (1, 1, 300000, 64)])
def test_select_from_logits_closer_than_the_scores_resolution(gpu_lib, b, K, V, count):
    """Every logit of a beam within some units of the values' last place, beams far apart."""
    x = _logits(b, K, V, "fp32", V + b, spread=1e-3)
    scores = -10000.0 - 100 * np.tile(np.arange(K), (b, 1))
    _check(gpu_lib, x, scores, count=count, gap=False)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("b,K,V,count", [(1, 2, 100, 128), (100, 2, 100, 128), (1, 3, 20011, 128), (64, 3, 20011, 9), (1, 1, 5, 8)])
def test_select_where_all_values_are_equal(gpu_lib, b, K, V, count, kind):
    """Scores so large that every candidate's value is the score: by rising beam, then by falling logit, then by token."""
    x = _logits(b, K, V, kind, V, spread=0.1)
    x = (x.float() * 50).round().div(50).to(x.dtype)                   # some equal ones
    scores = np.full((b, K), -2.0 ** 30, np.float32)
    got = _select(gpu_lib, x, scores, None, 0, count)
    x = x.float().cpu().numpy()
    for i in range(b):
        order = [(k, t) for k in range(K) for t in np.argsort(-x[i, k], kind="stable")][:count]
        n = len(order)
        assert (got[0][i, :n] == -2.0 ** 30).all() and (got[0][i, n:] == -np.inf).all()
        assert [*zip(got[1][i, :n].tolist(), got[2][i, :n].tolist())] == [(k, int(t)) for k, t in order]
