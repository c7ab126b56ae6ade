"""Low-rank adapters beside a shared product on the GPU against the plain 64-bit implementation: bit for bit on small whole numbers
(every sum is exact, and so are the 16-bit parts of the rows' projections), within the bound of the sums on random operands."""
import numpy as np
import pytest

import gemm_inputs as gi
import routed_util as ru

pytestmark = pytest.mark.gpu

KINDS = list(ru.KINDS)


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def run(kind, A, B, of, scales, down, up, lay=(gi.COL_MAJOR, gi.COL_MAJOR, gi.COL_MAJOR), pads=(0, 0, 0, 0, 0), shift=(0, 0, 0, 0, 0)):
    import torch
    import paper_2003_06324_amd as g
    a, c = ru.KINDS[kind]
    rows, K = A.shape
    N, n, r = B.shape[1], len(down), down.shape[2]
    tA, pA, lda, _ = ru.put(A, a, K + pads[0], shift[0])
    tB, pB, ldb, _ = ru.put(B, a, (N if lay[0] == gi.ROW_MAJOR else K) + pads[1], shift[1], lay[0])
    td, pd, ldd, sd = ru.put(down, a, (r if lay[1] == gi.ROW_MAJOR else K) + pads[2], shift[2], lay[1])
    tu, pu, ldu, su = ru.put(up, a, (N if lay[2] == gi.ROW_MAJOR else r) + pads[3], shift[3], lay[2])
    tC, pC, ldc = ru.room(rows, N, c, N + pads[4], shift[4])
    ts = None if scales is None else torch.from_numpy(np.asarray(scales, dtype=np.float32)).cuda()
    to = torch.from_numpy(np.asarray(of, dtype=np.int32)).cuda()
    g.gemm_adapters(ru.kind_of(kind), rows, N, K, pA, lda, pB, lay[0], ldb, n, r, to, ts, pd, lay[1], ldd, sd, pu, lay[2], ldu, su, pC, ldc, stream())
    torch.cuda.synchronize()
    got, clean = ru.back(tC, rows, N, ldc, shift[4])
    assert clean, "wrote outside C"
    return got


def bound(kind, K, r, ref, mag, add):
    # the product and the additions as sums of K and K + r terms (and three factors), what the parts leave out, and one rounding
    err = 1.01 * ru.U32 * (K + 1) * mag + (1.01 * ru.U32 * (K + r + 4) + 2.0 ** -21) * add
    return err + ru.HALF_ULP[ru.KINDS[kind][1]] * (np.abs(ref) + err) + ru.SMALLEST[ru.KINDS[kind][1]]


SIZES = [(1, 1, 1, 1, 1), (3, 7, 9, 2, 3), (16, 200, 128, 5, 8), (40, 130, 72, 40, 16), (64, 256, 512, 3, 64), (129, 300, 264, 2, 33), (300, 264, 200, 7, 16), (270, 136, 1100, 1, 100),
         (33, 64, 64, 33, 256), (5, 515, 333, 9, 13), (600, 100, 128, 200, 4)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,N,K,n,r", SIZES)
def test_adapters(kind, rows, N, K, n, r):
    rng = np.random.default_rng(rows * N + K)
    a, c = ru.KINDS[kind]
    for lay in ((1, 1, 1), (0, 0, 0), (1, 0, 1)):
        for dist in ("int", "normal"):
            A, B = ru.values(rng, (rows, K), a, dist), ru.values(rng, (K, N), a, dist)
            if dist == "int":   # sums below 2^24 with everything that is added up on the way
                keep = rng.random((n, K, r)) < min(1.0, 20.0 / K)
                down, up = ru.values(rng, (n, K, r), a, "int") * keep, np.sign(ru.values(rng, (n, r, N), a, "int"))
            else:
                down, up = ru.values(rng, (n, K, r), a, "normal", K ** -0.5), ru.values(rng, (n, r, N), a, "normal", 0.5)
            of = rng.integers(-1, n, size=rows)
            if rows > 20:
                of[rows // 3:rows // 2] = n - 1      # a run of one adapter
                of[3], of[4] = n, -7                 # numbers that name nothing
            scales = None if dist == "normal" and lay[0] else 2.0 ** rng.integers(-1, 3, size=n)
            ref, mag, add = ru.adapters(A, B, of, scales, down, up)
            got = run(kind, A, B, of, scales, down, up, lay)
            if dist == "int":
                assert np.array_equal(got, ru.rounded(ref, c))
            else:
                assert (np.abs(got - ref) <= bound(kind, K, r, ref, mag, add)).all()


@pytest.mark.parametrize("kind", ["f32", "f16f16", "bf16f32"])
@pytest.mark.parametrize("pads,shift", [((8, 8, 8, 8, 8), (0, 0, 0, 0, 0)), ((1, 3, 5, 1, 3), (0, 0, 0, 0, 0)), ((2, 6, 3, 2, 1), (2, 4, 1, 2, 6)), ((0, 0, 0, 0, 0), (1, 1, 1, 1, 1))])
def test_strides_and_alignments(kind, pads, shift):
    rng = np.random.default_rng(sum(pads))
    a, c = ru.KINDS[kind]
    for rows in (20, 400):
        for lay in ((1, 1, 1), (0, 0, 0)):
            A, B = ru.values(rng, (rows, 66), a, "int"), ru.values(rng, (66, 90), a, "int")
            down, up = ru.values(rng, (6, 66, 10), a, "int") * (rng.random((6, 66, 10)) < 0.3), ru.values(rng, (6, 10, 90), a, "int")
            of = rng.integers(-1, 6, size=rows)
            ref, _, _ = ru.adapters(A, B, of, None, down, up)
            assert np.array_equal(run(kind, A, B, of, None, down, up, lay, pads, shift), ru.rounded(ref, c))


@pytest.mark.parametrize("kind", ["f16f32", "bf16bf16", "f32"])
@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("rows,N,K,n,r", [(2100, 2050, 136, 3, 16), (2049, 2048, 70, 5, 72), (4100, 4200, 66, 9, 8),
                                            (2100, 2050, 1000, 4, 16), (2300, 1601, 999, 3, 70)])
def test_many_rows(kind, odd, rows, N, K, n, r):
    """Enough tiles that the chip is full: larger ones, rows on and off 4-byte words; runs of rows, alternating rows, rows without any."""
    rng = np.random.default_rng(rows + odd)
    a, c = ru.KINDS[kind]
    A, B = ru.values(rng, (rows, K), a, "int"), ru.values(rng, (K, N), a, "int")
    down, up = ru.values(rng, (n, K, r), a, "int") * (rng.random((n, K, r)) < 0.2), np.sign(ru.values(rng, (n, r, N), a, "int"))
    of = np.repeat(rng.integers(-1, n, size=rows // 150 + 1), 150)[:rows]
    of[500:700] = np.arange(200) % (n + 1) - 1
    ref, _, _ = ru.adapters(A, B, of, None, down, up)
    for lay in ((1, 1, 1), (0, 0, 0)):
        assert np.array_equal(run(kind, A, B, of, None, down, up, lay, (odd,) * 5), ru.rounded(ref, c))


@pytest.mark.parametrize("kind", ["f16f32", "bf16f32", "f32"])
def test_projections_of_any_size(kind):
    """What lies between the two products is neither cut off at the operand type's largest number nor lost below its smallest."""
    rng = np.random.default_rng(11)
    a = ru.KINDS[kind][0]
    rows, N, K, r = 40, 64, 128, 16
    A, B = ru.values(rng, (rows, K), a), np.zeros((K, N))
    down, up = ru.values(rng, (2, K, r), a), ru.values(rng, (2, r, N), a)
    of = rng.integers(0, 2, size=rows)
    A[::2] = ru.rounded(A[::2] * 2.0 ** 12, a)            # rows of very different sizes
    for scale in (2.0 ** -40, 1.0, 2.0 ** 30):
        ref, mag, add = ru.adapters(A, B, of, [scale, scale], down, up)
        got = run(kind, A, B, of, [scale, scale], down, up)
        assert (np.abs(got - ref) <= bound(kind, K, r, ref, mag, add) * np.ones_like(ref)).all() and np.isfinite(got).all()


def test_no_adapters_and_empty_sizes():
    rng = np.random.default_rng(12)
    A, B = ru.values(rng, (9, 40), "f16", "int"), ru.values(rng, (40, 30), "f16", "int")
    import torch
    import paper_2003_06324_amd as g
    tA, pA, lda, _ = ru.put(A, "f16")
    tB, pB, ldb, _ = ru.put(B, "f16", layout=gi.COL_MAJOR)
    for n, r in ((0, 4), (3, 0)):
        tC, pC, ldc = ru.room(9, 30, "f32")
        g.gemm_adapters(g.KIND_F16F32, 9, 30, 40, pA, lda, pB, 1, ldb, n, r, None, None, None, 1, 0, 0, None, 1, 0, 0, pC, ldc, stream())
        torch.cuda.synchronize()
        assert np.array_equal(ru.back(tC, 9, 30, ldc)[0], A @ B)
    got = run("f16f32", A, B, [-1] * 9, None, np.full((2, 40, 4), np.nan), np.full((2, 4, 30), np.nan))    # nobody's adapters are not looked at
    assert np.array_equal(got, A @ B)
    got = run("f16f32", np.zeros((5, 0)), np.zeros((0, 30)), [0] * 5, None, np.zeros((1, 0, 4)), np.zeros((1, 4, 30)))
    assert (got == 0).all()


def test_nan_of_one_adapter_stays_in_its_rows():
    rng = np.random.default_rng(13)
    for kind in ("f32", "f16f32", "bf16f32"):
        a = ru.KINDS[kind][0]
        A, B = ru.values(rng, (50, 64), a, "int"), ru.values(rng, (64, 70), a, "int")
        down, up = ru.values(rng, (3, 64, 8), a, "int") * (rng.random((3, 64, 8)) < 0.3), ru.values(rng, (3, 8, 70), a, "int")
        of = rng.integers(-1, 3, size=50)
        ref, _, _ = ru.adapters(A, B, of, None, down, up)
        up[1] = np.nan
        down[2, 5] = np.inf
        got = run(kind, A, B, of, None, down, up)
        assert np.array_equal(got[of <= 0], ref[of <= 0]) and np.isnan(got[of == 1]).all()
        assert not np.isfinite(got[(of == 2) & (A[:, 5] != 0)]).any(axis=1).all()


def test_gradients_by_the_same_calls():
    """dA is the call with every matrix transposed; the adapters' own gradients are grouped products over rows sorted by adapter."""
    import torch
    import paper_2003_06324_amd as g
    rng = np.random.default_rng(14)
    rows, N, K, n, r = 90, 48, 64, 4, 8
    A, B = ru.values(rng, (rows, K), "f32", "int"), ru.values(rng, (K, N), "f32", "int")
    down, up = ru.values(rng, (n, K, r), "f32", "int"), ru.values(rng, (n, r, N), "f32", "int")
    of, dC = rng.integers(-1, n, size=rows), ru.values(rng, (rows, N), "f32", "int")
    # the call for A's gradient: matrices as they lie in memory, other layouts
    tB, pB, ldb, _ = ru.put(B, "f32", layout=gi.COL_MAJOR)
    td, pd, ldd, sd = ru.put(down, "f32", layout=gi.COL_MAJOR)
    tu, pu, ldu, su = ru.put(up, "f32", layout=gi.COL_MAJOR)
    tC, pC, ldc, _ = ru.put(dC, "f32")
    tA, pA, lda, _ = ru.put(A, "f32")
    to = torch.from_numpy(of.astype(np.int32)).cuda()
    out, po, ldo = ru.room(rows, K, "f32")
    g.gemm_adapters(g.KIND_F32, rows, K, N, pC, ldc, pB, gi.ROW_MAJOR, ldb, n, r, to, None, pu, gi.ROW_MAJOR, ldu, su, pd, gi.ROW_MAJOR, ldd, sd,
                    po, ldo, stream())
    dA = dC @ B.T
    for a in range(n):
        dA[of == a] += dC[of == a] @ up[a].T @ down[a].T
    torch.cuda.synchronize()
    assert np.array_equal(ru.back(out, rows, K, ldo)[0], dA)
    # rows sorted by adapter, T = A down and S = dC up^T for the sorted rows, then d_up = T^T dC and d_down = A^T S
    offsets, row_of, slot_of = (torch.zeros(x, dtype=torch.int32, device="cuda") for x in (n + 1, rows, rows))
    g.gemm_route_plan(rows, 1, n, to, offsets, row_of, slot_of, stream())
    T, S = (torch.zeros((rows, r), device="cuda") for _ in range(2))
    g.gemm_grouped(g.KIND_F32, n, offsets, rows, r, K, pA, rows, lda, row_of, pd, gi.COL_MAJOR, ldd, sd, T, 0, stream())
    g.gemm_grouped(g.KIND_F32, n, offsets, rows, r, N, pC, rows, ldc, row_of, pu, gi.ROW_MAJOR, ldu, su, S, 0, stream())
    d_up, d_down = torch.zeros((n, N, r), device="cuda"), torch.zeros((n, K, r), device="cuda")
    g.gemm_grouped_wgrad(g.KIND_F32, n, offsets, rows, N, r, pC, rows, ldc, row_of, T, 0, d_up, gi.ROW_MAJOR, 0, 0, stream())
    g.gemm_grouped_wgrad(g.KIND_F32, n, offsets, rows, K, r, pA, rows, lda, row_of, S, 0, d_down, gi.ROW_MAJOR, 0, 0, stream())
    torch.cuda.synchronize()
    for a in range(n):
        i = of == a
        assert np.array_equal(d_up[a].cpu().numpy().T, (A[i] @ down[a]).T @ dC[i])
        assert np.array_equal(d_down[a].cpu().numpy(), A[i].T @ (dC[i] @ up[a].T))
