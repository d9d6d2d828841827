"""What the launches of the 8-bit floating-point products read and how they are cut, by the library's own arithmetic (no GPU)."""
import ctypes as C

import pytest

import paper_2503_22879_amd as q

FORMS = {"rows": 0, "tiles64": 1, "tiles64x128": 2, "tiles128_one": 3, "tiles128_two": 4, "tiles256": 5}


def _internal(name, restype, *argtypes):
    f = getattr(q.load_library(), name)      # library-internal
    f.restype, f.argtypes = restype, argtypes
    return f


@pytest.mark.parametrize("form", FORMS)
def test_no_wave_reads_behind_the_scales_of_w(form):
    """w's scales have ceil(n / 128) rows.  A 256 x 256 tile spans two of them: where 1 to 128 of its columns are left, the waves of its right
    half have none of their own."""
    last = _internal("_ZN6quamba25fp8_matmul_last_scale_rowENS_7Fp8FormEi", C.c_int32, C.c_int, C.c_int32)
    for n in [*range(1, 1100), 3352, 10576, 18560, 50021, 50280, 151936, 2 ** 20 + 1, 2 ** 26 - 200, 2 ** 26]:
        assert last(FORMS[form], n) == -(-n // 128) - 1, n


class Plan(C.Structure):
    _fields_ = [("form", C.c_int), ("splits", C.c_int), ("us", C.c_double)]


def _plan(m, n, k, workspace=True):
    f = _internal("_ZN6quamba15fp8_matmul_planEiiib", Plan, C.c_int32, C.c_int32, C.c_int32, C.c_bool)
    return f(m, n, -(-k // 128), workspace)


def test_half_filled_large_tiles_have_sizes_that_are_tested():
    from test_gpu_fp8 import HALF_FILLED
    for m, n, k in HALF_FILLED:
        assert _plan(m, n, k).form == FORMS["tiles256"] and 1 <= n % 256 <= 128


def test_the_parts_of_many_rows_are_joined_by_a_launch_that_fits():
    """A launch has at most 65535 workgroups along its second axis; the sizes are planned in parts."""
    from test_gpu_fp8 import TALL_SPLIT
    rows = _internal("_ZN6quamba20fp8_matmul_join_rowsEi", C.c_int32, C.c_int32)
    for m in (1, 17, 65535, 65536, 66096, 10 ** 6, 2 ** 29, 2 ** 31 - 1):
        assert rows(m) == min(m, 65535)
    for m, n, k in TALL_SPLIT:
        assert m > 65535 and q.quamba_fp8_matmul_workspace_size(m, n, k) > 0


class Cut(C.Structure):
    _fields_ = [("rows", C.c_int64), ("columns", C.c_int64)]


@pytest.mark.parametrize("block_rows", [1, 128])
def test_the_quantizers_launches_fit_32_bits(block_rows):
    """Threads of a launch are counted in 32 bits, and block numbers go through a division of 31; a launch of several rows of blocks holds them
    whole."""
    cut = _internal("_ZN6quamba16fp8_quantize_cutEli", Cut, C.c_int64, C.c_int32)
    threads = _internal("_ZN6quamba20fp8_quantize_threadsEli", C.c_int64, C.c_int64, C.c_int32)
    for row_blocks in (1, 2, 3, 64, 1000, 2 ** 21 + 1, 2 ** 22, 2 ** 22 + 1, 2 ** 23):
        got = cut(row_blocks, block_rows)
        assert got.rows >= 1 and 1 <= got.columns <= row_blocks and (got.rows == 1 or got.columns == row_blocks)
        assert got.rows * got.columns <= 2 ** 23 and threads(got.rows * got.columns, block_rows) < 2 ** 32, row_blocks
        assert 2 * got.rows * got.columns >= min(row_blocks, 2 ** 20)                # and there are few of them


def test_whole_rounds_and_every_form_behind_them_have_a_size_that_is_tested():
    from test_gpu_fp8 import WHOLE_ROUNDS
    whole = _internal("_ZN6quamba23fp8_matmul_whole_roundsEiiid", C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_double)
    for form, (m, n, k) in WHOLE_ROUNDS.items():
        rows = whole(m, n, -(-k // 128), _plan(m, n, k).us)
        assert 0 < rows < m and rows % 256 == 0 and _plan(m - rows, n, k, False).form == FORMS[form], (m, n, k, rows)
    assert set(WHOLE_ROUNDS) == set(FORMS) - {"tiles256"}       # its rounds would not be a rest
    for m, n, k in ((16384, 18560, 4096), (8192, 3352, 768), (2048, 18560, 4096)):
        assert whole(m, n, -(-k // 128), _plan(m, n, k).us) > 0
    assert whole(256, 50021, 20, _plan(256, 50021, 2560).us) == 0 and whole(1, 10, 1, 0.0) == 0


def test_every_form_has_depths_with_a_last_block_in_part():
    from test_gpu_fp8 import TAILS, TAIL_DEPTHS
    assert {d % 128 for d in TAIL_DEPTHS} == {64, 80, 112} and {d // 128 % 2 for d in TAIL_DEPTHS} == {0, 1}
    for form, sizes in TAILS.items():
        for m, n in sizes:
            assert all(_plan(m, n, k).form == FORMS[form] for k in TAIL_DEPTHS), (form, m, n)


def test_no_workspace_where_the_depth_is_not_split():
    unaligned = _internal("_ZN6quamba25fp8_matmul_plan_unalignedEiiii", Plan, C.c_int32, C.c_int32, C.c_int32, C.c_int32)
    split = set()
    for m in (1, 9, 17, 100, 333, 2000):
        for n in (300, 4001):
            for k in (90, 401, 517, 2101, 4113, 4112, 2048, 272):
                splits = (unaligned(m, n, -(-k // 128), 16) if k % 16 else _plan(m, n, k)).splits
                assert q.quamba_fp8_matmul_workspace_size(m, n, k) == (splits * m * -(-n // 4) * 16 if splits > 1 else 0), (m, n, k)
                split.add((splits > 1, k % 16 > 0))
    assert len(split) == 4
