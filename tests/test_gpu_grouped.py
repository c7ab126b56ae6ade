"""The experts' products, their gradients and the sum of a token's experts on the GPU against plain 64-bit implementations.

Operands of small whole numbers make every sum exact, so results are compared bit for bit; random ones are within the bound of
their sums in binary32."""
import numpy as np
import pytest

import gemm_inputs as gi
import routed_util as ru

pytestmark = pytest.mark.gpu

KINDS = list(ru.KINDS)
LAYOUTS = [gi.ROW_MAJOR, gi.COL_MAJOR]


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def ints(x):
    import torch
    return None if x is None else torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()


def cuts(rng, groups, rows, empty=0.3):
    """Offsets of groups of very different sizes, some of them empty, some rows in no group."""
    share = rng.random(groups) ** 3 * (rng.random(groups) > empty)
    n = np.floor(share / max(share.sum(), 1e-9) * rows * 0.97).astype(int) if groups else np.zeros(0, int)
    first = (rows - n.sum()) // 2
    return np.concatenate([[first], first + np.cumsum(n)]).astype(np.int32)


def run_grouped(kind, A, offsets, rows, row_map, B, layout, pads=(0, 0, 0), shift=(0, 0, 0), gap=0):
    import torch
    import paper_2003_06324_amd as g
    a, c = ru.KINDS[kind]
    G, K, N = B.shape
    tA, pA, lda, _ = ru.put(A, a, A.shape[1] + pads[0], shift[0])
    minor, major = (N, K) if layout == gi.ROW_MAJOR else (K, N)
    if gap:   # matrices further apart than they are long
        full = np.full((G, major + gap, minor), np.nan)
        full[:, :major] = B if layout == gi.ROW_MAJOR else B.transpose(0, 2, 1)
        tB, pB, ldb, stride = ru.put(full, a, minor + pads[1], shift[1])
    else:
        tB, pB, ldb, stride = ru.put(B, a, minor + pads[1], shift[1], layout)
    tC, pC, ldc = ru.room(rows, N, c, N + pads[2], shift[2])
    g.gemm_grouped(ru.kind_of(kind), G, ints(offsets), rows, N, K, pA, len(A), lda, ints(row_map), pB, layout, ldb, stride, pC, ldc, stream())
    torch.cuda.synchronize()
    got, clean = ru.back(tC, rows, N, ldc, shift[2])
    assert clean, "wrote outside C"
    return got


def check(got, ref, there, mag, kind, K, dist):
    c = ru.KINDS[kind][1]
    assert (got[~there] == 12288.0).all(), "wrote rows of no group"
    if dist == "int":
        assert np.array_equal(got[there], ru.rounded(ref, c)[there])
    else:
        assert (np.abs(got - ref) <= ru.bound(mag, K, c, ref))[there].all()


# rows for a group on average: each of the kernel's forms, and their edges
SIZES = [(1, 1, 1, 1, 1), (3, 5, 7, 9, 2), (8, 40, 64, 128, 8), (16, 130, 200, 72, 16), (4, 300, 130, 136, 4), (5, 700, 256, 520, 5), (2, 1100, 132, 64, 2),
         (128, 512, 48, 64, 40), (70, 9, 128, 256, 70), (200, 3000, 40, 192, 9), (1, 33, 1, 65, 1), (3, 260, 520, 1, 3), (1030, 2000, 16, 16, 64)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("G,rows,N,K,a_rows", SIZES)
def test_grouped(kind, G, rows, N, K, a_rows):
    rng = np.random.default_rng(G * rows + N)
    a = ru.KINDS[kind][0]
    for layout in LAYOUTS:
        for mapped in (False, True):
            for dist in ("int", "normal"):
                offsets = cuts(rng, G, rows)
                A = ru.values(rng, (a_rows if mapped else rows, K), a, dist)
                B = ru.values(rng, (G, K, N), a, dist)
                row_map = rng.integers(0, a_rows, size=rows) if mapped else None
                if mapped and rows > 4:
                    row_map[rows // 2] = -1
                    row_map[rows // 3] = a_rows
                ref, there, mag = ru.grouped(A, offsets, rows, row_map, B)
                check(run_grouped(kind, A, offsets, rows, row_map, B, layout), ref, there, mag, kind, K, dist)


@pytest.mark.parametrize("kind", ["f32", "f16f32", "bf16bf16"])
@pytest.mark.parametrize("pads,shift,gap", [((8, 8, 8), (0, 0, 0), 0), ((1, 3, 5), (0, 0, 0), 0), ((2, 6, 2), (2, 4, 6), 0), ((0, 0, 0), (1, 1, 1), 0),
                                            ((5, 0, 0), (0, 0, 3), 3), ((0, 2, 1), (0, 2, 0), 1)])
def test_grouped_strides_and_alignments(kind, pads, shift, gap):
    rng = np.random.default_rng(sum(pads) + 7)
    a = ru.KINDS[kind][0]
    for rows, G in ((50, 6), (900, 4)):
        for K in (64, 70, 129):
            for layout in LAYOUTS:
                offsets = cuts(rng, G, rows)
                A, B = ru.values(rng, (31, K), a, "int"), ru.values(rng, (G, K, 90), a, "int")
                row_map = rng.integers(0, 31, size=rows)
                ref, there, mag = ru.grouped(A, offsets, rows, row_map, B)
                check(run_grouped(kind, A, offsets, rows, row_map, B, layout, pads, shift, gap), ref, there, mag, kind, K, "int")


@pytest.mark.parametrize("kind", ["f16f32", "bf16bf16", "f32"])
@pytest.mark.parametrize("odd", [0, 1])
def test_full_chips(kind, odd):
    """Enough tiles that the chip is full: larger ones, rows on and off 4-byte words."""
    rng = np.random.default_rng(21 + odd)
    a, c = ru.KINDS[kind]
    for G, rows, N, K in ((3, 4000, 2050, 72), (40, 4500, 900, 70)):
        for layout in LAYOUTS:
            offsets = cuts(rng, G, rows)
            A, B = ru.values(rng, (500, K), a, "int"), ru.values(rng, (G, K, N), a, "int")
            row_map = rng.integers(0, 500, size=rows)
            ref, there, mag = ru.grouped(A, offsets, rows, row_map, B)
            check(run_grouped(kind, A, offsets, rows, row_map, B, layout, (odd,) * 3), ref, there, mag, kind, K, "int")
    for G, rows, M, N in ((5, 700, 1030, 1000), (36, 900, 500, 390)):
        for layout in LAYOUTS:
            offsets = cuts(rng, G, rows)
            A, D = ru.values(rng, (200, M), a, "int"), ru.values(rng, (rows, N), a, "int")
            row_map = rng.integers(0, 200, size=rows)
            ref, _ = ru.wgrad(A, offsets, rows, row_map, D)
            assert np.array_equal(run_wgrad(kind, A, offsets, rows, row_map, D, layout, (odd,) * 3), ru.rounded(ref, c))


@pytest.mark.parametrize("kind", ["f16f32", "bf16bf16"])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_long_products_of_odd_rows(kind, layout):
    """Rows in the middle of 4-byte words in products long enough that they are copied first; called twice, with other operands in
    between, so that nothing of one call is left for the next."""
    rng = np.random.default_rng(31)
    a, c = ru.KINDS[kind]
    for trial in range(2):
        for mapped in (False, True):
            G, rows, N, K = 3, 3000, 1003, 1001
            offsets = cuts(rng, G, rows, 0.0)
            A, B = ru.values(rng, (700 if mapped else rows, K), a, "int"), ru.values(rng, (G, K, N), a, "int")
            row_map = rng.integers(-1, 701, size=rows) if mapped else None
            ref, there, mag = ru.grouped(A, offsets, rows, row_map, B)
            check(run_grouped(kind, A, offsets, rows, row_map, B, layout, (0, 2 * trial, 1), (1, 0, 3)), ref, there, mag, kind, K, "int")
            M = 905
            A, D = ru.values(rng, (900 if mapped else rows, M), a, "int"), ru.values(rng, (rows, N), a, "int")
            row_map = rng.integers(-1, 901, size=rows) if mapped else None
            ref, _ = ru.wgrad(A, offsets, rows, row_map, D)
            assert np.array_equal(run_wgrad(kind, A, offsets, rows, row_map, D, layout, (0, 0, 2), (1, 0, 0)), ru.rounded(ref, c))


def test_grouped_without_rows_columns_or_k():
    rng = np.random.default_rng(5)
    B = ru.values(rng, (3, 8, 16), "f16", "int")
    assert (run_grouped("f16f32", np.zeros((4, 8)), [0, 0, 0, 0], 4, None, B, gi.ROW_MAJOR) == 12288.0).all()
    got = run_grouped("f16f32", np.zeros((0, 8)), [0, 2, 3, 4], 4, [0, 1, 2, 3], B, gi.ROW_MAJOR)     # no row of A: zeros
    assert (got == 0).all()
    got = run_grouped("f16f32", np.ones((2, 8)), [0, 2, 3, 4], 4, None, B, gi.COL_MAJOR)              # A shorter than the groups' rows
    assert np.array_equal(got[:2], np.ones((2, 8)) @ B[0]) and (got[2:] == 0).all()
    got = run_grouped("bf16f32", np.zeros((4, 0)), [0, 1, 4], 4, None, np.zeros((2, 0, 24)), gi.ROW_MAJOR)   # empty sums
    assert (got == 0).all()


def test_grouped_offsets_out_of_range_are_cut():
    rng = np.random.default_rng(6)
    A, B = ru.values(rng, (40, 32), "bf16", "int"), ru.values(rng, (4, 32, 20), "bf16", "int")
    got = run_grouped("bf16f32", A, [-5, 10, 30, 60, 90], 40, None, B, gi.COL_MAJOR)
    ref, there, mag = ru.grouped(A, np.array([0, 10, 30, 40, 40]), 40, None, B)
    check(got, ref, there, mag, "bf16f32", 32, "int")


def test_a_nan_row_stays_its_own():
    """Rows behind a tile's last one, K's tail and other groups' matrices hold NaN and never reach a result."""
    rng = np.random.default_rng(7)
    for K in (40, 64, 100):
        A, B = ru.values(rng, (70, K), "f16", "int"), ru.values(rng, (3, K, 33), "f16", "int")
        A[20:41] = np.nan
        B[1] = np.nan
        offsets = [0, 20, 41, 70]
        got = run_grouped("f16f32", A, offsets, 70, None, B, gi.ROW_MAJOR, pads=(8, 8, 0))
        assert np.array_equal(got[:20], A[:20] @ B[0]) and np.isnan(got[20:41]).all() and np.array_equal(got[41:], A[41:] @ B[2])


# ---------------------------------------------------------------------------- the gradient of B
def run_wgrad(kind, A, offsets, rows, row_map, D, layout, pads=(0, 0, 0), shift=(0, 0, 0)):
    import torch
    import paper_2003_06324_amd as g
    a, c = ru.KINDS[kind]
    G, M, N = len(offsets) - 1, A.shape[1], D.shape[1]
    tA, pA, lda, _ = ru.put(A, a, M + pads[0], shift[0])
    tD, pD, ldd, _ = ru.put(D, a, N + pads[1], shift[1])
    r, cc = (M, N) if layout == gi.ROW_MAJOR else (N, M)
    tC, pC, ldc = ru.room(G * r, cc, c, cc + pads[2], shift[2])
    g.gemm_grouped_wgrad(ru.kind_of(kind), G, ints(offsets), rows, M, N, pA, len(A), lda, ints(row_map), pD, ldd, pC, layout, ldc, 0, stream())
    torch.cuda.synchronize()
    got, clean = ru.back(tC, G * r, cc, ldc, shift[2])
    assert clean, "wrote outside C"
    got = got.reshape(G, r, cc)
    return got if layout == gi.ROW_MAJOR else got.transpose(0, 2, 1)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("G,rows,M,N,a_rows", [(1, 1, 1, 1, 1), (3, 5, 7, 9, 2), (8, 300, 64, 128, 40), (5, 700, 200, 72, 700), (2, 260, 130, 136, 9), (7, 400, 515, 334, 100),
                                               (16, 20, 256, 128, 8), (1, 9000, 65, 40, 300)])
def test_wgrad(kind, G, rows, M, N, a_rows):
    rng = np.random.default_rng(G * rows + M)
    a, c = ru.KINDS[kind]
    for layout in LAYOUTS:
        for mapped in (False, True):
            for dist in ("int", "normal"):
                offsets = cuts(rng, G, rows)
                A = ru.values(rng, (a_rows if mapped else rows, M), a, dist)
                D = ru.values(rng, (rows, N), a, dist)
                row_map = rng.integers(0, a_rows, size=rows) if mapped else None
                if mapped and rows > 4:
                    row_map[rows // 2] = -1
                    row_map[rows // 3] = a_rows
                ref, mag = ru.wgrad(A, offsets, rows, row_map, D)
                got = run_wgrad(kind, A, offsets, rows, row_map, D, layout)
                if dist == "int":
                    assert np.array_equal(got, ru.rounded(ref, c))
                else:
                    assert (np.abs(got - ref) <= ru.bound(mag, max(1, rows), c, ref)).all()


@pytest.mark.parametrize("kind", ["f32", "f16f16", "bf16f32"])
@pytest.mark.parametrize("pads,shift", [((8, 8, 8), (0, 0, 0)), ((1, 3, 5), (0, 0, 0)), ((2, 6, 2), (2, 4, 6)), ((0, 0, 0), (1, 1, 1)), ((0, 2, 1), (0, 2, 0))])
def test_wgrad_strides_and_alignments(kind, pads, shift):
    rng = np.random.default_rng(sum(pads) + 3)
    a, c = ru.KINDS[kind]
    for M, N in ((64, 40), (130, 33)):
        for layout in LAYOUTS:
            for mapped in (False, True):
                offsets = cuts(rng, 5, 400)
                A, D = ru.values(rng, (77 if mapped else 400, M), a, "int"), ru.values(rng, (400, N), a, "int")
                row_map = rng.integers(0, 77, size=400) if mapped else None
                ref, _ = ru.wgrad(A, offsets, 400, row_map, D)
                assert np.array_equal(run_wgrad(kind, A, offsets, 400, row_map, D, layout, pads, shift), ru.rounded(ref, c))


def test_wgrad_rows_behind_the_end_of_A():
    rng = np.random.default_rng(9)
    A, D = ru.values(rng, (150, 64), "bf16", "int"), ru.values(rng, (400, 32), "bf16", "int")
    offsets = [0, 100, 260, 300, 400]
    ref, _ = ru.wgrad(A, np.array(offsets), 400, None, D)
    assert np.array_equal(run_wgrad("bf16f32", A, offsets, 400, None, D, gi.ROW_MAJOR), ref)
    assert np.array_equal(run_wgrad("bf16f32", A[:0], offsets, 400, None, D, gi.COL_MAJOR), 0 * ref)


# ---------------------------------------------------------------------------- sums of a token's rows
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,k,N", [(1, 1, 1), (5, 3, 7), (64, 8, 256), (33, 9, 1000), (3, 17, 515), (200, 2, 2048), (2, 1, 4104)])
def test_combine(kind, T, k, N):
    import torch
    import paper_2003_06324_amd as g
    a, c = ru.KINDS[kind]
    rng = np.random.default_rng(T * k + N)
    for pad, shift in ((0, 0), (8, 0), (3, 1)):
        for weighted in (True, False):
            Y = ru.values(rng, (T * k, N), a)
            slots = rng.permutation(T * k).reshape(T, k)
            slots[rng.random((T, k)) < 0.15] = -1
            if T > 2:
                slots[1, 0], slots[2] = T * k, -1       # beyond the rows; a token with none
            w = rng.standard_normal((T, k)).astype(np.float32) if weighted else None
            if weighted:
                w[slots < 0] = np.nan                   # weights of nothing do not matter
            tY, pY, ldy, _ = ru.put(Y, a, N + pad, shift)
            out, po, ldo = ru.room(T, N, c, N + pad, shift)
            g.gemm_combine(ru.kind_of(kind), T, k, N, pY, T * k, ldy, ints(slots), None if w is None else torch.from_numpy(w).cuda(), po, ldo, stream())
            torch.cuda.synchronize()
            got, clean = ru.back(out, T, N, ldo, shift)
            ref, mag = ru.combine(Y, slots, w)
            assert clean and (np.abs(got - ref) <= ru.bound(mag, k, c, ref)).all()


@pytest.mark.parametrize("elem", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,k,N", [(1, 1, 1), (5, 3, 7), (64, 8, 256), (33, 9, 1000), (3, 17, 515), (200, 2, 2048)])
def test_combine_backward(elem, T, k, N):
    import torch
    import paper_2003_06324_amd as g
    rng = np.random.default_rng(T * k + N)
    for pad, shift in ((0, 0), (8, 0), (3, 1)):
        for weighted in (True, False):
            Y, d = ru.values(rng, (T * k, N), elem), ru.values(rng, (T, N), elem)
            slots = rng.permutation(T * k).reshape(T, k)
            slots[rng.random((T, k)) < 0.15] = -1
            w = rng.standard_normal((T, k)).astype(np.float32) if weighted else None
            tY, pY, ldy, _ = ru.put(Y, elem, N + pad, shift)
            td, pd, ldd, _ = ru.put(d, elem, N + pad, shift)
            out, po, ldo = ru.room(T * k, N, elem, N + pad, shift)
            dw = torch.full((T * k + 4,), -7.0, device="cuda")
            tw = None if w is None else torch.from_numpy(w).cuda()
            g.gemm_combine_backward(ru.elem_of(elem), T, k, N, pd, ldd, pY, T * k, ldy, ints(slots), tw, po, ldo, dw, stream())
            torch.cuda.synchronize()
            got, clean = ru.back(out, T * k, N, ldo, shift)
            written = np.zeros(T * k, dtype=bool)
            dy, rdw, mag = np.zeros((T * k, N)), np.zeros((T, k)), np.zeros((T, k))
            for t in range(T):
                for j in range(k):
                    s = slots[t, j]
                    if s >= 0:
                        written[s] = True
                        dy[s] = (1.0 if w is None else float(w[t, j])) * d[t]
                        rdw[t, j], mag[t, j] = d[t] @ Y[s], np.abs(d[t]) @ np.abs(Y[s])
            assert clean and (got[~written] == 12288.0).all()
            assert (np.abs(got - dy) <= ru.bound(np.abs(dy), 1, elem, dy))[written].all()
            h = dw.cpu().numpy()
            assert (h[T * k:] == -7).all() and (np.abs(h[:T * k].reshape(T, k) - rdw) <= ru.bound(mag, N, "f32", rdw)).all()
            # without the weights' gradient Y is not needed
            out, po, ldo = ru.room(T * k, N, elem, N + pad, shift)
            g.gemm_combine_backward(ru.elem_of(elem), T, k, N, pd, ldd, None, T * k, ldy, ints(slots), tw, po, ldo, None, stream())
            torch.cuda.synchronize()
            assert np.array_equal(ru.back(out, T * k, N, ldo, shift)[0], got)
