"""Routing to experts, its gradient and the plan on the GPU against plain 64-bit implementations."""
import numpy as np
import pytest

import routed_util as ru

pytestmark = pytest.mark.gpu


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def apart(rng, T, E, elem):
    """Logits whose scores are far apart (whatever a 32-bit evaluation does, their order is the same): every row a permutation of
    a grid, in steps that the element type has; some equal, which have to go to the lowest index."""
    x = np.tile((np.arange(E) - E // 2) / 16.0, (T, 1))
    x = rng.permuted(x, axis=1)
    if E > 3:
        x[::3, 1] = x[::3, 3]
    return ru.rounded(x, elem)


def run_route(logits, elem, softmax, top_k, bias=None, groups=1, top_groups=1, group_top=1, renormalise=True, scale=1.0, ld=0, offset=0):
    import torch
    import paper_2003_06324_amd as g
    T, E = logits.shape
    _, at, ld, _ = keep = ru.put(logits, elem, ld, offset)
    b = None if bias is None else torch.from_numpy(np.asarray(bias, dtype=np.float32)).cuda()
    w = torch.full((T * top_k + 4,), -7.0, device="cuda")
    i = torch.full((T * top_k + 4,), -7, dtype=torch.int32, device="cuda")
    g.gemm_route(ru.elem_of(elem), T, E, at, ld, b, g.SCORE_SOFTMAX if softmax else g.SCORE_SIGMOID, groups, top_groups, group_top, top_k,
                 int(renormalise), scale, w, i, stream())
    torch.cuda.synchronize()
    del keep
    w, i = w.cpu().numpy(), i.cpu().numpy()
    assert (w[T * top_k:] == -7).all() and (i[T * top_k:] == -7).all()
    return w[:T * top_k].reshape(T, top_k), i[:T * top_k].reshape(T, top_k)


def weight_tolerance(ref, E, logits):
    # every factor relative: exp (two units, and what the rounded difference in its argument makes of it), a sum of E terms, the
    # quotients, the sum of the chosen ones
    return (2 * E + 16 + 2 * np.abs(logits[np.isfinite(logits)]).max()) * ru.U32 * np.abs(ref) + 1e-37


SHAPES = [(1, 1, 1), (1, 7, 3), (5, 8, 8), (33, 16, 2), (64, 60, 4), (17, 128, 8), (16, 255, 5), (9, 256, 16), (7, 257, 6), (6, 300, 17), (3, 1024, 64)]


@pytest.mark.parametrize("elem", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,E,k", SHAPES)
def test_experts_and_weights(T, E, k, elem):
    rng = np.random.default_rng(E * 100 + k)
    for softmax in (True, False):
        for renormalise in (True, False):
            x = apart(rng, T, E, elem)
            if not softmax:
                x = x / 4 if elem == "f32" else x     # (scores that 32 bits tell apart)
                x = ru.rounded(np.clip(x, -8, 8), elem)
            w, i = run_route(x, elem, softmax, k, renormalise=renormalise, scale=2.5, ld=E + 3, offset=1)
            rw, ri = ru.route(x, softmax, k, renormalise=renormalise, scale=2.5)
            assert np.array_equal(i, ri)
            assert (np.abs(w - rw) <= weight_tolerance(rw, E, x)).all()


@pytest.mark.parametrize("E,groups,top_groups,group_top,k", [(256, 8, 4, 2, 8), (64, 8, 3, 1, 6), (60, 4, 2, 2, 5), (12, 12, 5, 2, 4), (256, 32, 3, 2, 9),
                                                            (96, 3, 1, 2, 7), (1024, 64, 9, 2, 33), (40, 20, 4, 2, 8), (512, 16, 8, 1, 8), (6, 2, 2, 1, 6)])
def test_groups_and_bias(E, groups, top_groups, group_top, k):
    """The bias makes the choice values a grid of their own, so that sums of two are told apart as well."""
    rng = np.random.default_rng(E + groups)
    T = 19
    x = rng.integers(-4, 5, size=(T, E)) / 4.0
    s = ru.scores(x, False)
    # equal logits everywhere: choice values are one score plus distinct multiples of 1/4
    x[:] = 0.25
    s = ru.scores(x, False)[0, 0]
    bias = rng.permutation(E) / 4.0
    w, i = run_route(x, "f32", False, k, bias, groups, top_groups, group_top, True, 1.0)
    rw, ri = ru.route(x, False, k, bias, groups, top_groups, group_top, True, 1.0)
    assert np.array_equal(i, ri)
    assert (np.abs(w - rw) <= weight_tolerance(rw, E, x)).all() and s > 0
    # scores decide: rows of distinct grid values, groups by their best
    x = apart(rng, T, E, "f32") / 8
    w, i = run_route(x, "f32", False, k, None, groups, top_groups, 1, False, 1.0)
    rw, ri = ru.route(x, False, k, None, groups, top_groups, 1, False, 1.0)
    assert np.array_equal(i, ri)
    assert (np.abs(w - rw) <= weight_tolerance(rw, E, x)).all()


def test_all_equal_goes_to_the_lowest_indices():
    x = np.zeros((5, 100))
    for groups in (1, 4):
        w, i = run_route(x, "bf16", True, 6, None, groups, groups, 2)
        assert np.array_equal(i, np.tile(np.arange(6), (5, 1)))
        assert (np.abs(w - 1 / 6) <= 4 * ru.U32).all()
    w, i = run_route(x, "f32", True, 6, None, 4, 2, 2)
    assert np.array_equal(i, np.tile(np.arange(6), (5, 1)))


@pytest.mark.parametrize("elem", ["f32", "f16", "bf16"])
def test_masked_experts(elem):
    """Minus infinity masks an expert, a row of nothing else has zero scores; the type's lowest value is a number like any other."""
    lowest = {"f32": -3.4028234663852886e38, "f16": -65504.0, "bf16": -3.3895313892515355e38}[elem]
    x = np.zeros((6, 20))
    x[0, :] = -np.inf
    x[1, :] = -np.inf
    x[1, 7] = 3.0
    x[2, 4:] = -np.inf
    x[3, :] = lowest
    x[4, :10] = lowest
    x[5, ::2] = -np.inf
    for softmax in (True, False):
        for renormalise in (True, False):
            w, i = run_route(x, elem, softmax, 5, renormalise=renormalise)
            rw, ri = ru.route(x, softmax, 5, renormalise=renormalise)
            assert np.array_equal(i, ri), (softmax, renormalise)
            assert np.isfinite(w).all() and (np.abs(w - rw) <= 64 * ru.U32 * np.abs(rw)).all()


def test_nan_and_infinity_reach_their_own_row_only():
    x = np.tile(np.arange(24) / 4.0, (4, 1))
    x[1, 5] = np.nan
    x[2, 9] = np.inf
    for softmax in (True, False):
        w, i = run_route(x, "f32", softmax, 24, renormalise=False)
        for t in range(4):
            assert sorted(i[t]) == list(range(24))
        rw, ri = ru.route(x[[0, 3]], softmax, 24, renormalise=False)
        assert np.array_equal(i[[0, 3]], ri) and (np.abs(w[[0, 3]] - rw) <= 64 * ru.U32 * rw).all()
        if softmax:
            assert np.isnan(w[1]).all() and np.isnan(w[2]).all()
        else:
            assert i[1, 23] == 5 and np.isnan(w[1, 23]) and np.isfinite(w[1, :23]).all()   # NaN ranks below every number
            assert i[2, 0] == 9 and w[2, 0] == 1.0


@pytest.mark.parametrize("elem", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,E,k", SHAPES)
def test_gradient(T, E, k, elem):
    import torch
    import paper_2003_06324_amd as g
    rng = np.random.default_rng(E * 10 + k)
    x = ru.values(rng, (T, E), elem)
    dw = rng.standard_normal((T, k)).astype(np.float32)
    at = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    for softmax in (True, False):
        for renormalise in (True, False):
            for pad, offset in ((0, 0), (5, 3)):
                _, px, ld, _ = keep = ru.put(x, elem, E + pad, offset)
                out, po, ldo = ru.room(T, E, elem, E + pad, offset)
                g.gemm_route_backward(ru.elem_of(elem), T, E, px, ld, g.SCORE_SOFTMAX if softmax else g.SCORE_SIGMOID, k, int(renormalise), 1.5,
                                      torch.from_numpy(at).cuda(), torch.from_numpy(dw).cuda(), po, ldo, stream())
                torch.cuda.synchronize()
                del keep
                got, clean = ru.back(out, T, E, ldo, offset)
                ref = ru.route_backward(x, softmax, at, dw, renormalise, 1.5)
                # every score is off by (E + 16 + |x|) units at most, relative; what they enter are these magnitudes
                s = ru.scores(x, softmax)
                chosen = np.take_along_axis(s, at, 1)
                z = chosen.sum(axis=1, keepdims=True) if renormalise else 1.0
                mag = 1.5 * s * (np.abs(dw).max(axis=1, keepdims=True) / z * 2 + (np.abs(dw) * chosen / z).sum(axis=1, keepdims=True))
                assert clean and (np.abs(got - ref) <= 4 * (E + 24) * ru.U32 * mag + ru.HALF_ULP[elem] * np.abs(ref) + ru.SMALLEST[elem]).all()


def test_gradient_of_masked_rows_is_zero_and_bad_indices_are_passed_over():
    import torch
    import paper_2003_06324_amd as g
    x = np.zeros((3, 16))
    x[0] = -np.inf
    at = np.array([[0, 1], [-1, 3], [99, 2]], dtype=np.int32)
    dw = np.ones((3, 2), dtype=np.float32)
    dw[1, 0] = dw[2, 0] = np.nan
    for softmax in (g.SCORE_SOFTMAX, g.SCORE_SIGMOID):
        for renormalise in (0, 1):
            out = torch.full((3, 16), 5.0, device="cuda")
            g.gemm_route_backward(g.ELEM_F32, 3, 16, torch.from_numpy(x).float().cuda(), 0, softmax, 2, renormalise, 1.0, torch.from_numpy(at).cuda(),
                                  torch.from_numpy(dw).cuda(), out, 0, stream())
            torch.cuda.synchronize()
            got = out.cpu().numpy()
            assert np.isfinite(got).all() and (got[0] == 0).all()
            if renormalise:
                assert (np.abs(got[1:]) <= 1e-6).all()     # one expert that counts: its weight is constant


@pytest.mark.parametrize("T,k,E", [(0, 2, 5), (1, 1, 1), (1, 8, 8), (3, 5, 7), (64, 8, 128), (1000, 3, 17), (1025, 8, 256), (2500, 4, 1000), (700, 16, 1024), (20000, 7, 60), (40000, 8, 1024)])
def test_plan(T, k, E):
    import torch
    import paper_2003_06324_amd as g
    rng = np.random.default_rng(T + E)
    idx = rng.integers(0, max(1, E * 3 // 4), size=(T, k)).astype(np.int32)     # (some experts have nothing)
    if T > 4:
        idx[::5, 0] = -1
        idx[1::7, k - 1] = E
        idx[2, :] = np.iinfo(np.int32).max
        idx[3, :] = np.iinfo(np.int32).min
    for _ in range(2):    # (the second time with what the first left behind)
        offsets = torch.full((E + 3,), -9, dtype=torch.int32, device="cuda")
        token_of = torch.full((T * k + 2,), -9, dtype=torch.int32, device="cuda")
        slot_of = torch.full((T * k + 2,), -9, dtype=torch.int32, device="cuda")
        g.gemm_route_plan(T, k, E, torch.from_numpy(idx).cuda(), offsets, token_of, slot_of, stream())
        torch.cuda.synchronize()
        o, to, so = (x.cpu().numpy() for x in (offsets, token_of, slot_of))
        assert (o[E + 1:] == -9).all() and (to[T * k:] == -9).all() and (so[T * k:] == -9).all()
        flat = idx.reshape(-1).astype(np.int64)
        ok = (flat >= 0) & (flat < E)
        order = np.nonzero(ok)[0][np.argsort(flat[ok], kind="stable")]
        ro = np.concatenate([[0], np.cumsum(np.bincount(flat[ok], minlength=E))])
        rt = np.full(T * k, -1)
        rt[:len(order)] = order // k
        rs = np.full(T * k, -1)
        rs[order] = np.arange(len(order))
        assert np.array_equal(o[:E + 1], ro) and np.array_equal(to[:T * k], rt) and np.array_equal(so[:T * k], rs)
