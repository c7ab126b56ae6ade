"""The forms that only some sizes reach: more groups than a wave has lanes, tiles of 256 x 256 and of 128 x 128 in several rounds beside
adapters, ranks that are no whole pieces.  Whole numbers, so that every sum is exact."""
import numpy as np
import pytest

import gemm_inputs as gi
import routed_util as ru
from test_gpu_adapters import run
from test_gpu_grouped import cuts, run_grouped, run_wgrad

pytestmark = pytest.mark.gpu
COLS, ROWS = (gi.COL_MAJOR,) * 3, (gi.ROW_MAJOR,) * 3


@pytest.mark.parametrize("kind", ["f16f16", "bf16f32", "f32"])
@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("G,rows,M,N", [(130, 3000, 96, 72), (200, 2500, 200, 300), (65, 700, 260, 40)])
def test_gradients_of_many_groups(kind, odd, G, rows, M, N):
    rng = np.random.default_rng(G + odd)
    a, c = ru.KINDS[kind]
    for layout in (gi.ROW_MAJOR, gi.COL_MAJOR):
        offsets = cuts(rng, G, rows)
        A, D = ru.values(rng, (150, M), a, "int"), ru.values(rng, (rows, N), a, "int")
        for row_map in (rng.integers(0, 150, size=rows), None):
            X = A if row_map is not None else ru.values(rng, (rows, M), a, "int")
            ref, _ = ru.wgrad(X, offsets, rows, row_map, D)
            assert np.array_equal(run_wgrad(kind, X, offsets, rows, row_map, D, layout, (odd,) * 3), ru.rounded(ref, c))


@pytest.mark.parametrize("kind", ["f16f32", "bf16bf16"])
def test_sums_of_many_rows_in_few_tiles(kind):
    """Long enough that odd rows are copied first, though there is little to compute."""
    rng = np.random.default_rng(3)
    a, c = ru.KINDS[kind]
    offsets, rows = np.array([0, 2900, 2900, 5800], dtype=np.int32), 5900
    A, D = ru.values(rng, (rows, 65), a, "int"), ru.values(rng, (rows, 77), a, "int")
    row_map = rng.integers(-1, rows, size=rows)
    for m in (None, row_map):
        ref, _ = ru.wgrad(A, offsets, rows, m, D)
        assert np.array_equal(run_wgrad(kind, A, offsets, rows, m, D, gi.ROW_MAJOR), ru.rounded(ref, c))
    B = np.sign(ru.values(rng, (3, 65, 77), a, "int"))
    ref, there, _ = ru.grouped(A, offsets, rows, row_map, B)
    assert np.array_equal(run_grouped(kind, A, offsets, rows, row_map, B, gi.ROW_MAJOR)[there], ru.rounded(ref, c)[there])


def ids(rng, rows, n):
    of = np.repeat(rng.integers(-1, n, size=rows // 150 + 1), 150)[:rows]
    if rows >= 700:
        of[500:700] = np.arange(200) % (n + 1) - 1
    return of


@pytest.mark.parametrize("kind", ["f16f32", "bf16bf16", "f32"])
@pytest.mark.parametrize("rows,N,K,n,r", [(4000, 2100, 1100, 4, 16), (3900, 2200, 1090, 3, 72), (4700, 2300, 64, 5, 40)])
def test_tiles_of_many_rows(kind, rows, N, K, n, r):
    """256 x 256 (long sums in one round), 128 x 128 in two rounds."""
    rng = np.random.default_rng(rows)
    a, c = ru.KINDS[kind]
    A, B = ru.values(rng, (rows, K), a, "int"), ru.values(rng, (K, N), a, "int")
    down, up = ru.values(rng, (n, K, r), a, "int") * (rng.random((n, K, r)) < 0.2), np.sign(ru.values(rng, (n, r, N), a, "int"))
    of = ids(rng, rows, n)
    ref, _, _ = ru.adapters(A, B, of, None, down, up)
    want = ru.rounded(ref, c)
    for lay in (COLS, ROWS):
        assert np.array_equal(run(kind, A, B, of, None, down, up, lay), want)


@pytest.mark.parametrize("kind", ["f16f32", "bf16bf16", "f32"])
@pytest.mark.parametrize("r", [1, 5, 9, 38, 60, 203])
def test_ranks_of_few_rows(kind, r):
    rng = np.random.default_rng(r)
    a, c = ru.KINDS[kind]
    for rows, N, K, n in ((37, 200, 530, 5), (3, 70, 1100, 2)):
        A, B = ru.values(rng, (rows, K), a, "int"), ru.values(rng, (K, N), a, "int")
        down, up = ru.values(rng, (n, K, r), a, "int") * (rng.random((n, K, r)) < 0.1), np.sign(ru.values(rng, (n, r, N), a, "int"))
        of = rng.integers(-1, n, size=rows)
        ref, _, _ = ru.adapters(A, B, of, None, down, up)
        for lay in (COLS, ROWS):
            assert np.array_equal(run(kind, A, B, of, None, down, up, lay), ru.rounded(ref, c))


def test_a_rank_in_the_middle_of_a_piece_reads_nothing_behind_it():
    """The element behind a row of up^T is infinite: a piece that reaches over the rank takes only its own part of it."""
    rng = np.random.default_rng(8)
    rows, N, K, n, r = 9, 40, 64, 1, 11
    A, B = ru.values(rng, (rows, K), "f16", "int"), ru.values(rng, (K, N), "f16", "int")
    down, up = ru.values(rng, (n, K, r), "f16", "int"), np.sign(ru.values(rng, (n, r, N), "f16", "int"))
    wide = np.full((n, 16, N), np.inf)
    wide[:, :r] = up
    import torch
    import paper_2003_06324_amd as g
    t = [ru.put(A, "f16", K), ru.put(B, "f16", K, 0, gi.COL_MAJOR), ru.put(down, "f16", K, 0, gi.COL_MAJOR), ru.put(wide, "f16", 16, 0, gi.COL_MAJOR)]
    tC, pC, ldc = ru.room(rows, N, "f32", N)
    of = torch.zeros(rows, dtype=torch.int32, device="cuda")
    g.gemm_adapters(g.KIND_F16F32, rows, N, K, t[0][1], K, t[1][1], gi.COL_MAJOR, K, n, r, of, None, t[2][1], gi.COL_MAJOR, K, 0,
                    t[3][1], gi.COL_MAJOR, 16, 0, pC, ldc, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    got, clean = ru.back(tC, rows, N, ldc, 0)
    ref, _, _ = ru.adapters(A, B, np.zeros(rows, int), None, down, up)
    assert clean and np.array_equal(got, ref)
