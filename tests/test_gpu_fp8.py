"""GPU parity of the 8-bit floating-point quantizer (codes and scales bit for bit) and of the product of its operands
(against float64), through the C ABI."""
import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu

TYPES = ("fp32", "fp16", "bf16")


def _torch_type(name):
    import torch
    return {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}[name]


def _values(rows, cols, seed, scale=1.0):
    r = np.random.default_rng(seed)
    return (r.standard_normal((rows, cols)) * np.exp(0.5 * r.standard_normal(cols)) * scale).astype(np.float32)


def _quantize(q, x, block_rows):
    """Codes and scales of a torch matrix, and that nothing beside them was written."""
    import torch
    rows, cols = x.shape
    nr, nb = -(-rows // block_rows), -(-cols // 128)
    room = torch.full((rows * cols + 32,), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((nr * nb + 2,), -7.0, device="cuda")
    q.quamba_fp8_quantize(x, room[16:16 + rows * cols].view(rows, cols), scales[1:1 + nr * nb].view(nr, nb), block_rows=block_rows)
    room, scales = room.cpu().numpy(), scales.cpu().numpy()
    assert (room[:16] == 0xA5).all() and (room[16 + rows * cols:] == 0xA5).all()
    assert scales[0] == -7.0 and scales[-1] == -7.0
    return room[16:16 + rows * cols].reshape(rows, cols), scales[1:-1].reshape(nr, nb)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 129), (7, 640), (128, 128), (129, 255), (300, 1031), (130, 4096)])
def test_quantizer_bit_exact(gpu_lib, rows, cols, kind, block_rows):
    import torch
    x = torch.from_numpy(_values(rows, cols, rows * 7 + cols)).to(_torch_type(kind))
    codes, scales = _quantize(gpu_lib, x.cuda(), block_rows)
    want, ws = oracle.quantize_fp8(x.float().numpy(), block_rows)
    assert np.array_equal(scales, ws) and np.array_equal(codes, want)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantizer_extremes(gpu_lib, block_rows):
    """Zeros, values whose scale would be subnormal, the largest and the smallest floats, NaN and infinity: each in a block of its own."""
    import torch
    x = _values(130, 128 * 9, 5)
    x[:, 0:128] = 0.0
    x[:, 0] = -0.0
    x[:, 128:256] *= 1e-40
    x[:, 256:384] *= 1e37 / np.abs(x[:, 256:384]).max()
    x[:, 384:512] = 1.4e-45
    x[0, 512], x[1, 640], x[2, 768] = np.nan, np.inf, -np.inf
    x[:, 896] = 3.4028235e38
    x[:, 1024:] *= 2.0 ** -118 / np.abs(x[:, 1024:]).max()     # a scale at the border of the normal numbers
    codes, scales = _quantize(gpu_lib, torch.from_numpy(x).cuda(), block_rows)
    want, ws = oracle.quantize_fp8(x, block_rows)
    assert np.array_equal(scales, ws, equal_nan=True) and np.array_equal(codes, want)


def test_quantizer_strides_and_alignment(gpu_lib):
    """Rows cut out of a wider tensor at odd places, codes into one."""
    import torch
    wide = torch.from_numpy(_values(41, 700, 6)).to(torch.float16).cuda()
    for lo, hi in ((0, 256), (1, 300), (3, 516), (400, 700)):
        x = wide[:, lo:hi]
        out = torch.full((41, 711), 0x11, dtype=torch.uint8, device="cuda")
        scales = torch.empty(41, -(-(hi - lo) // 128), device="cuda")
        gpu_lib.quamba_fp8_quantize(x, out[:, 5:5 + hi - lo], scales)
        want, ws = oracle.quantize_fp8(x.float().cpu().numpy(), 1)
        got = out.cpu().numpy()
        assert np.array_equal(got[:, 5:5 + hi - lo], want) and np.array_equal(scales.cpu().numpy(), ws)
        assert (got[:, :5] == 0x11).all() and (got[:, 5 + hi - lo:] == 0x11).all()


def test_quantizer_of_nothing(gpu_lib):
    import torch
    gpu_lib.quamba_fp8_quantize(torch.empty(0, 128, device="cuda"), torch.empty(0, 128, dtype=torch.uint8, device="cuda"),
                                torch.empty(0, 1, device="cuda"))


def _operands(m, n, k, seed):
    x, w = _values(m, k, seed), _values(n, k, seed + 1, 0.05)
    return oracle.quantize_fp8(x, 1) + oracle.quantize_fp8(w, 128)


def _bound(y, top, k, kind):
    """The rounding of the sums and of the output.  Products of two 4-bit significands are exact; the sum of n of them loses at
    most n 2^-23 of the sum of their magnitudes (2^-23: also where an addition cuts), the scale two roundings, the sum over
    the blocks one each."""
    err = (128 + 2 + 2 * (-(-k // 128))) * 2.0 ** -23 * top
    half = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}[kind]
    tiny = {"fp32": 2.0 ** -149, "fp16": 2.0 ** -25, "bf16": 2.0 ** -134}[kind]
    return err + half * (np.abs(y) + err) + tiny


def _matmul(q, ops, kind, workspace=True, pad=0):
    """y of the operands, into a tensor with `pad` more columns that stay as they are."""
    import torch
    x, xs, w, ws = (torch.from_numpy(a).cuda() for a in ops)
    m, k = x.shape
    n = w.shape[0]
    y = torch.full((m, n + pad), 77.0, dtype=_torch_type(kind), device="cuda")
    size = q.quamba_fp8_matmul_workspace_size(m, n, k) if workspace else 0
    space = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if size else None
    q.quamba_fp8_matmul(x, xs, w, ws, y[:, :n], workspace=space)
    if pad:
        assert (y[:, n:] == 77.0).all()
    return y[:, :n].double().cpu().numpy()


SIZES = [(1, 1, 1), (1, 16, 128), (1, 130, 257), (1, 333, 4096), (2, 257, 640), (5, 100, 1537), (15, 64, 96), (16, 512, 2048),
         (17, 129, 384), (33, 300, 250), (50, 256, 8192), (64, 128, 128), (65, 1000, 768), (100, 77, 129), (128, 128, 1024),
         (129, 515, 511), (200, 640, 1280), (256, 256, 256), (300, 700, 900), (513, 257, 272)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_matmul(gpu_lib, m, n, k):
    ops = _operands(m, n, k, m + n + k)
    y, top = oracle.ref_fp8_matmul(*ops)
    for kind in TYPES:
        got = _matmul(gpu_lib, ops, kind, pad=3 if kind == "fp16" else 0)
        off = np.abs(got - y) / _bound(y, top, k, kind)
        assert off.max() <= 1.0, (kind, off.max(), np.argwhere(off > 1)[:5])
    # without scratch memory: the same to rounding, and the same again
    a = _matmul(gpu_lib, ops, "fp32", workspace=False)
    assert (np.abs(a - y) <= _bound(y, top, k, "fp32")).all()
    assert np.array_equal(a, _matmul(gpu_lib, ops, "fp32", workspace=False))
    assert np.array_equal(_matmul(gpu_lib, ops, "fp32"), _matmul(gpu_lib, ops, "fp32"))


# A size of each form of the product (test_operator_refusals.py checks which), with a depth of whole blocks, of a partial one, and of one
# whose rows lie at odd addresses; ragged in rows and columns.
FORMS = {"rows": [(5, 300, 2048), (30, 300, 2064), (60, 300, 400)], "tiles64": [(100, 500, 4112), (130, 4000, 1024)],
         "tiles64x128": [(500, 4001, 1040)], "tiles128_one": [(600, 4095, 400), (1000, 3901, 768)], "tiles128_two": [(2000, 2501, 400)],
         "tiles256": [(4090, 4003, 1296)]}


@pytest.mark.parametrize("m,n,k", [s for sizes in FORMS.values() for s in sizes])
def test_matmul_of_every_form(gpu_lib, m, n, k):
    for depth in (k, k // 128 * 128, k + 3):
        ops = _operands(m, n, depth, m + depth)
        y, top = oracle.ref_fp8_matmul(*ops)
        for kind in ("fp32", "bf16"):
            off = np.abs(_matmul(gpu_lib, ops, kind, pad=5) - y) / _bound(y, top, depth, kind)
            assert off.max() <= 1.0, (depth, kind, off.max(), np.argwhere(off > 1)[:5])


UNALIGNED = {"rows": [(9, 300, 517)], "tiles64": [(20, 300, 2101), (100, 500, 4113), (333, 4001, 90)], "tiles128_two": [(2000, 2501, 401)]}


@pytest.mark.parametrize("m,n,k", [s for sizes in UNALIGNED.values() for s in sizes])
def test_matmul_of_unaligned_rows(gpu_lib, m, n, k):
    """A depth that no alignment fits, and a whole number of pieces in rows at odd distances (whose workspace is that of aligned
    rows); with the workspace and without."""
    import torch
    for depth, pad in ((k, 0), (k // 16 * 16, 3)):
        ops = _operands(m, n, depth, m + depth)
        y, top = oracle.ref_fp8_matmul(*ops)
        x, xs, w, ws = (torch.from_numpy(a).cuda() for a in ops)
        xb, wb = (torch.full((a.shape[0], depth + pad), 0x7f, dtype=torch.uint8, device="cuda") for a in (x, w))  # NaN between the rows
        xb[:, :depth], wb[:, :depth] = x, w
        size = gpu_lib.quamba_fp8_matmul_workspace_size(m, n, depth)
        for space in [None] + [torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")] * (size > 0):
            out = torch.full((m, n), float("nan"), device="cuda")
            gpu_lib.quamba_fp8_matmul(xb[:, :depth], xs, wb[:, :depth], ws, out, workspace=space)
            assert (np.abs(out.double().cpu().numpy() - y) <= _bound(y, top, depth, "fp32")).all(), (depth, size)


@pytest.mark.parametrize("m,n,k", [(1, 200, 512), (20, 200, 512), (70, 300, 640), (300, 520, 384)])
def test_matmul_strides_and_alignment(gpu_lib, m, n, k):
    """Operands cut out of wider tensors: rows at multiples of 16 bytes, of 4 and at odd places, and of another width."""
    import torch
    ops = _operands(m, n, k, 3)
    y, top = oracle.ref_fp8_matmul(*ops)
    x, xs, w, ws = (torch.from_numpy(a).cuda() for a in ops)
    for dx, sx, dw, sw in ((0, 16, 0, 32), (16, 48, 0, 0), (4, 12, 0, 0), (0, 0, 1, 7), (3, 5, 8, 24)):
        xb = torch.full((m, k + sx), 0x7f, dtype=torch.uint8, device="cuda")      # NaN around the operands
        wb = torch.full((n, k + sw), 0x7f, dtype=torch.uint8, device="cuda")
        dx, dw = min(dx, sx), min(dw, sw)
        xb[:, dx:dx + k], wb[:, dw:dw + k] = x, w
        out = torch.empty(m, n, device="cuda")
        space = torch.empty(max(16, gpu_lib.quamba_fp8_matmul_workspace_size(m, n, k)), dtype=torch.uint8, device="cuda")
        gpu_lib.quamba_fp8_matmul(xb[:, dx:dx + k], xs, wb[:, dw:dw + k], ws, out, workspace=space)
        got = out.double().cpu().numpy()
        assert (np.abs(got - y) <= _bound(y, top, k, "fp32")).all(), (dx, sx, dw, sw)


@pytest.mark.parametrize("m,n,k", [(3, 150, 300), (40, 150, 300), (150, 260, 300), (300, 600, 520)])
def test_matmul_numbers_that_are_none(gpu_lib, m, n, k):
    """A NaN code reaches the outputs of its row of x, or of its column w, and no others; so do the scales of a block, an infinity among
    them; the rows behind the last one and the columns behind the depth reach nothing."""
    x, xs, w, ws = _operands(m, n, k, 9)
    y, top = oracle.ref_fp8_matmul(x, xs, w, ws)
    x, xs, w, ws = x.copy(), xs.copy(), w.copy(), ws.copy()
    x[m - 1, k - 1] = 0x7f
    xs[0, 1] = np.inf
    w[n - 1, 0] = 0xff
    ws[0, 0] = np.nan
    hit = np.zeros((m, n), bool)
    hit[m - 1], hit[0], hit[:, n - 1], hit[:, :128] = True, True, True, True
    got = _matmul(gpu_lib, (x, xs, w, ws), "fp32")
    assert not np.isfinite(got[hit]).any()
    assert (np.abs(got - y) <= _bound(y, top, k, "fp32"))[~hit].all()


def test_matmul_saturates_like_its_type(gpu_lib):
    """Sums beyond fp16 become infinities, in fp32 and bf16 they stay."""
    x = np.full((2, 256), 0x7e, np.uint8)
    w = np.full((3, 256), 0x7e, np.uint8)
    ops = (x, np.ones((2, 2), np.float32), w, np.ones((1, 2), np.float32))
    assert np.isinf(_matmul(gpu_lib, ops, "fp16")).all()
    for kind in ("fp32", "bf16"):
        assert (np.abs(_matmul(gpu_lib, ops, kind) / (256 * 448.0 ** 2) - 1) < 2.0 ** -8).all()


def test_matmul_offsets_beyond_32_bits(gpu_lib):
    """Rows of x, w and y over 4 GiB apart from the first ones."""
    import torch
    m, n, k, far = 5, 20, 256, 1 << 30
    ops = _operands(m, n, k, 12)
    y, top = oracle.ref_fp8_matmul(*ops)
    x, xs, w, ws = (torch.from_numpy(a).cuda() for a in ops)
    wide = torch.empty(20 * (far // 4), dtype=torch.uint8, device="cuda")
    xv = wide.as_strided((m, k), (far, 1))
    wv = wide.as_strided((n, k), (far // 4, 1), k)
    xv.copy_(x)
    wv.copy_(w)
    out = torch.empty(4 * far // 2 + n, dtype=torch.float32, device="cuda")
    yv = out.as_strided((m, n), (far // 2, 1))
    gpu_lib.quamba_fp8_matmul(xv, xs, wv, ws, yv)
    assert (np.abs(yv.double().cpu().numpy() - y) <= _bound(y, top, k, "fp32")).all()


def test_matmul_of_many_rows_and_no_rows(gpu_lib):
    """More rows than a launch has workgroups along one axis, checked on some; and none at all."""
    import torch
    m, n, k = 70000 * 16, 16, 128
    x, xs, w, ws = _operands(16, n, k, 13)
    y, top = oracle.ref_fp8_matmul(x, xs, w, ws)
    xt = torch.from_numpy(x).cuda().repeat(m // 16, 1)
    st = torch.from_numpy(xs).cuda().repeat(m // 16, 1)
    out = torch.empty(m, n, device="cuda")
    gpu_lib.quamba_fp8_matmul(xt, st, torch.from_numpy(w).cuda(), torch.from_numpy(ws).cuda(), out)
    got = out.view(-1, 16, n)
    assert (got == got[0]).all()
    assert (np.abs(got[0].double().cpu().numpy() - y) <= _bound(y, top, k, "fp32")).all()
    gpu_lib.quamba_fp8_matmul(xt[:0], st[:0], torch.from_numpy(w).cuda(), torch.from_numpy(ws).cuda(), out[:0])


def test_quantize_and_multiply_on_another_stream(gpu_lib):
    """Both calls on a stream that is not the tensors' own, captured into a graph and replayed over changing inputs."""
    import torch
    m, n, k = 40, 384, 1024
    side = torch.cuda.Stream()
    x = torch.zeros(m, k, dtype=torch.bfloat16, device="cuda")
    w = torch.from_numpy(_values(n, k, 21, 0.05)).cuda()
    wq, ws = torch.empty(n, k, dtype=torch.uint8, device="cuda"), torch.empty(3, 8, device="cuda")
    gpu_lib.quamba_fp8_quantize(w, wq, ws, block_rows=128)
    xq, xs, y = torch.empty(m, k, dtype=torch.uint8, device="cuda"), torch.empty(m, 8, device="cuda"), torch.empty(m, n, device="cuda")
    space = torch.empty(max(16, gpu_lib.quamba_fp8_matmul_workspace_size(m, n, k)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()

    def step():
        gpu_lib.quamba_fp8_quantize(x, xq, xs)
        gpu_lib.quamba_fp8_matmul(xq, xs, wq, ws, y, workspace=space)

    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for seed in range(4):
        x.copy_(torch.from_numpy(_values(m, k, seed)))
        graph.replay()
        got = y.clone()
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, y)
        ops = oracle.quantize_fp8(x.float().cpu().numpy(), 1) + (wq.cpu().numpy(), ws.cpu().numpy())
        want, top = oracle.ref_fp8_matmul(*ops)
        assert (np.abs(got.double().cpu().numpy() - want) <= _bound(want, top, k, "fp32")).all()


# 256 x 256 tiles whose last ones hold 1 to 128 columns, in one block of w's scales (test_fp8_plans.py checks the form).
HALF_FILLED = [(3321, 4137, 640), (3840, 4200, 1296)]


@pytest.mark.parametrize("m,n,k", HALF_FILLED)
def test_matmul_of_half_filled_large_tiles(gpu_lib, m, n, k):
    ops = _operands(m, n, k, m + k)
    y, top = oracle.ref_fp8_matmul(*ops)
    assert (np.abs(_matmul(gpu_lib, ops, "fp32", pad=5) - y) <= _bound(y, top, k, "fp32")).all()


# More rows than a launch has workgroups along an axis, and a depth in parts (test_fp8_plans.py checks that): aligned rows, and others.
TALL_SPLIT = [(16 * 4131, 3, 10240), (16 * 4131, 3, 5117)]


@pytest.mark.parametrize("m,n,k", TALL_SPLIT)
def test_matmul_of_many_rows_in_parts(gpu_lib, m, n, k):
    import torch
    x, xs, w, ws = _operands(16, n, k, 14)
    y, top = oracle.ref_fp8_matmul(x, xs, w, ws)
    xt, st = (torch.from_numpy(v).cuda().repeat(m // 16, 1) for v in (x, xs))
    out = torch.full((m, n), float("nan"), device="cuda")
    space = torch.full((gpu_lib.quamba_fp8_matmul_workspace_size(m, n, k),), 0xFF, dtype=torch.uint8, device="cuda")
    gpu_lib.quamba_fp8_matmul(xt, st, torch.from_numpy(w).cuda(), torch.from_numpy(ws).cuda(), out, workspace=space)
    got = out.view(-1, 16, n)
    assert (got == got[0]).all()
    assert (np.abs(got[0].double().cpu().numpy() - y) <= _bound(y, top, k, "fp32")).all()


@pytest.mark.parametrize("rows,cols", [(1 << 30, 1), (1, 1 << 30)])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantizer_of_more_blocks_than_a_launch_takes(gpu_lib, rows, cols, block_rows):
    """As many rows, or columns, as fit: the same 2^17 values again and again, the first against the oracle."""
    import torch
    period = 1 << 17
    shape = (period, 1) if cols == 1 else (1, period)
    x = torch.from_numpy(_values(1, period, 22).reshape(shape)).half()
    want, ws = oracle.quantize_fp8(x.float().numpy(), block_rows)
    xt = x.cuda().view(-1).repeat((rows * cols) // period).view(rows, cols)
    codes = torch.full((rows, cols), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((-(-rows // block_rows), -(-cols // 128)), -7.0, device="cuda")
    gpu_lib.quamba_fp8_quantize(xt, codes, scales, block_rows=block_rows)
    for got, first in ((codes.view(-1), want), (scales.view(-1), ws)):
        got = got.view(-1, first.size)
        assert np.array_equal(got[0].cpu().numpy(), first.reshape(-1)) and bool((got == got[0]).all())


# Rows that make whole rounds of 256 x 256 tiles go so, the others in a form of their own: a size for each of these
# (test_fp8_plans.py checks which).
WHOLE_ROUNDS = {"rows": (4100, 4000, 400), "tiles64": (4180, 4000, 768), "tiles64x128": (4200, 4224, 1024), "tiles128_one": (4240, 4500, 768),
                "tiles128_two": (4500, 4500, 768)}


@pytest.mark.parametrize("m,n,k", WHOLE_ROUNDS.values())
def test_matmul_in_whole_rounds_and_the_rest(gpu_lib, m, n, k):
    """Rows of x and y further apart than they are long, what lies between is neither read nor written."""
    import torch
    ops = _operands(m, n, k, m)
    y, top = oracle.ref_fp8_matmul(*ops)
    x, xs, w, ws = (torch.from_numpy(a).cuda() for a in ops)
    xb = torch.full((m, k + 48), 0x7f, dtype=torch.uint8, device="cuda")
    xb[:, :k] = x
    for kind in ("fp32", "fp16"):
        out = torch.full((m, n + 24), 77.0, dtype=_torch_type(kind), device="cuda")
        gpu_lib.quamba_fp8_matmul(xb[:, :k], xs, w, ws, out[:, :n])
        assert (out[:, n:] == 77.0).all()
        off = np.abs(out[:, :n].double().cpu().numpy() - y) / _bound(y, top, k, kind)
        assert off.max() <= 1.0, (kind, off.max(), np.argwhere(off > 1)[:5])


# Depths whose last block holds 64 codes (the most of which half are multiplied), 80 and 112 (the least and the most of which all are), behind 3 and 8
# whole blocks, so that either group of waves gets it; a size of each form (test_fp8_plans.py checks which).
TAILS = {"rows": [(5, 300), (30, 300), (60, 300)], "tiles64": [(100, 500)], "tiles64x128": [(500, 4001)], "tiles128_one": [(600, 4095)],
         "tiles128_two": [(2000, 2501)], "tiles256": [(4090, 4003)]}
TAIL_DEPTHS = [whole * 128 + codes for whole in (3, 8) for codes in (64, 80, 112)]


@pytest.mark.parametrize("m,n", [s for sizes in TAILS.values() for s in sizes])
def test_matmul_of_a_last_block_in_part(gpu_lib, m, n):
    """The codes behind the depth, which are read or repeated by no product, are NaN."""
    import torch
    ops = _operands(m, n, TAIL_DEPTHS[-1], m + 17)
    for depth in TAIL_DEPTHS:
        blocks = -(-depth // 128)
        x, xs, w, ws = (ops[i][:, :depth] if i % 2 == 0 else ops[i][:, :blocks].copy() for i in range(4))
        y, top = oracle.ref_fp8_matmul(x, xs, w, ws)
        xb, wb = (torch.full((v.shape[0], depth + 128), 0x7f, dtype=torch.uint8, device="cuda") for v in (x, w))
        xb[:, :depth], wb[:, :depth] = torch.from_numpy(x.copy()).cuda(), torch.from_numpy(w.copy()).cuda()
        for space in (True, False):
            size = gpu_lib.quamba_fp8_matmul_workspace_size(m, n, depth) if space else 0
            out = torch.full((m, n), float("nan"), device="cuda")
            gpu_lib.quamba_fp8_matmul(xb[:, :depth], torch.from_numpy(xs).cuda(), wb[:, :depth], torch.from_numpy(ws).cuda(), out,
                                      workspace=torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if size else None)
            off = np.abs(out.double().cpu().numpy() - y) / _bound(y, top, depth, "fp32")
            assert off.max() <= 1.0, (depth, space, off.max(), np.argwhere(off > 1)[:5])
