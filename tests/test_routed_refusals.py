"""What the calls of include/gemm_routed.h refuse, before anything is enqueued (no GPU needed), and that the header is plain C."""
import ctypes
import os
import re
import subprocess

import pytest

import paper_2003_06324_amd as g
from paper_2003_06324_amd import routed

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096   # an address that no refused or empty call looks at
INVALID, UNSUPPORTED = -1, -3

# a call of each that would be served but for its having nothing to do, as {argument: value} in order
ROUTE = dict(elem=g.ELEM_F32, tokens=0, experts=16, logits=P, ld=0, bias=None, score=g.SCORE_SOFTMAX, groups=4, top_groups=2, group_top=2, top_k=4,
             renormalise=1, scale=1.0, weights=P, indices=P)
ROUTE_BACKWARD = dict(elem=g.ELEM_F16, tokens=0, experts=16, logits=P, ld=0, score=g.SCORE_SIGMOID, top_k=4, renormalise=1, scale=1.0, indices=P,
                      d_weights=P, d_logits=P, ld_d=0)
PLAN = dict(tokens=0, top_k=4, experts=16, indices=P, offsets=P, token_of=P, slot_of=P)
GROUPED = dict(kind=g.KIND_BF16BF16, groups=4, offsets=P, rows=0, N=32, K=48, A=P, a_rows=9, lda=0, row_map=None, B=P, layoutB=g.COL_MAJOR, ldb=0, strideB=0,
               C=P, ldc=0)
WGRAD = dict(kind=g.KIND_F32, groups=4, offsets=P, rows=8, M=0, N=48, A=P, a_rows=9, lda=0, row_map=None, D=P, ldd=0, C=P, layoutC=g.ROW_MAJOR, ldc=0, strideC=0)
COMBINE = dict(kind=g.KIND_F16F16, tokens=0, top_k=2, N=32, Y=P, y_rows=8, ldy=0, slot_of=P, weights=None, out=P, ldo=0)
COMBINE_BACKWARD = dict(elem=g.ELEM_BF16, tokens=0, top_k=2, N=32, d_out=P, ldo=0, Y=P, y_rows=8, ldy=0, slot_of=P, weights=None, dY=P, lddy=0, d_weights=None)
ADAPTERS = dict(kind=g.KIND_F16F32, rows=0, N=32, K=48, A=P, lda=0, B=P, layoutB=g.ROW_MAJOR, ldb=0, adapters=3, rank=8, adapter_of=P, scales=None, down=P,
                layout_down=g.COL_MAJOR, ld_down=0, stride_down=0, up=P, layout_up=g.COL_MAJOR, ld_up=0, stride_up=0, C=P, ldc=0)
CALLS = {"gemm_route": ROUTE, "gemm_route_backward": ROUTE_BACKWARD, "gemm_grouped": GROUPED, "gemm_grouped_wgrad": WGRAD, "gemm_combine": COMBINE,
         "gemm_combine_backward": COMBINE_BACKWARD, "gemm_adapters": ADAPTERS}
BIG = 2 ** 31

REFUSED = {
    "gemm_route": [(INVALID, dict(elem=3)), (INVALID, dict(elem=-1)), (INVALID, dict(tokens=-1)), (INVALID, dict(experts=0, groups=1)), (INVALID, dict(score=2)),
                   (INVALID, dict(groups=3)), (INVALID, dict(groups=0)), (INVALID, dict(top_groups=0)), (INVALID, dict(top_groups=5)), (INVALID, dict(group_top=3)),
                   (INVALID, dict(group_top=0)), (INVALID, dict(top_k=0)), (INVALID, dict(top_k=9)), (INVALID, dict(top_k=17, groups=1, top_groups=1)),
                   (INVALID, dict(ld=15)), (INVALID, dict(ld=-1)), (INVALID, dict(tokens=1, logits=None)), (INVALID, dict(tokens=1, weights=None)),
                   (INVALID, dict(tokens=1, indices=None)), (UNSUPPORTED, dict(experts=1028)), (UNSUPPORTED, dict(tokens=BIG)),
                   (UNSUPPORTED, dict(experts=1000, top_k=65, groups=1, top_groups=1)), (UNSUPPORTED, dict(experts=130, groups=65, top_groups=65)),
                   (UNSUPPORTED, dict(tokens=2, ld=2 ** 62))],
    "gemm_route_backward": [(INVALID, dict(elem=4)), (INVALID, dict(tokens=-2)), (INVALID, dict(ld_d=3)), (INVALID, dict(ld=3)), (INVALID, dict(top_k=17)),
                            (INVALID, dict(tokens=1, indices=None)), (INVALID, dict(tokens=1, d_weights=None)), (INVALID, dict(tokens=1, d_logits=None)),
                            (INVALID, dict(tokens=1, logits=None)), (UNSUPPORTED, dict(experts=1025)), (UNSUPPORTED, dict(tokens=3, ld_d=2 ** 62))],
    "gemm_grouped": [(INVALID, dict(kind=5)), (INVALID, dict(kind=-1)), (INVALID, dict(groups=-1)), (INVALID, dict(rows=-1)), (INVALID, dict(N=-1)), (INVALID, dict(K=-1)),
                     (INVALID, dict(a_rows=-1)), (INVALID, dict(lda=47)), (INVALID, dict(ldb=47)), (INVALID, dict(ldb=31, layoutB=g.ROW_MAJOR)), (INVALID, dict(ldc=31)),
                     (INVALID, dict(strideB=-1)), (INVALID, dict(layoutB=2)), (INVALID, dict(rows=1, offsets=None)), (INVALID, dict(rows=1, A=None)),
                     (INVALID, dict(rows=1, B=None)), (INVALID, dict(rows=1, C=None)), (UNSUPPORTED, dict(rows=BIG)), (UNSUPPORTED, dict(N=BIG)),
                     (UNSUPPORTED, dict(strideB=2 ** 61)), (UNSUPPORTED, dict(rows=2 ** 30, N=2 ** 20, ldc=2 ** 20))],
    "gemm_grouped_wgrad": [(INVALID, dict(kind=9)), (INVALID, dict(M=-1)), (INVALID, dict(layoutC=-1)), (INVALID, dict(M=3, ldc=47)), (INVALID, dict(ldd=47)),
                           (INVALID, dict(M=3, lda=2)), (INVALID, dict(M=3, strideC=143)), (INVALID, dict(M=3, strideC=-1)), (INVALID, dict(M=3, offsets=None)), (INVALID, dict(M=3, A=None)),
                           (INVALID, dict(M=3, D=None)), (INVALID, dict(M=3, C=None)), (UNSUPPORTED, dict(M=BIG)), (UNSUPPORTED, dict(M=2 ** 20, N=2 ** 20)),
                           (UNSUPPORTED, dict(M=3, strideC=2 ** 61))],
    "gemm_combine": [(INVALID, dict(kind=5)), (INVALID, dict(tokens=-1)), (INVALID, dict(top_k=-1)), (INVALID, dict(ldy=31)), (INVALID, dict(ldo=31)),
                     (INVALID, dict(tokens=1, slot_of=None)), (INVALID, dict(tokens=1, Y=None)), (INVALID, dict(tokens=1, out=None)), (UNSUPPORTED, dict(tokens=BIG)),
                     (UNSUPPORTED, dict(y_rows=4, ldy=2 ** 62))],
    "gemm_combine_backward": [(INVALID, dict(elem=3)), (INVALID, dict(N=-1)), (INVALID, dict(lddy=31)), (INVALID, dict(tokens=1, slot_of=None)),
                              (INVALID, dict(tokens=1, d_out=None)), (INVALID, dict(tokens=1, dY=None)), (INVALID, dict(tokens=1, d_weights=P, Y=None)),
                              (UNSUPPORTED, dict(tokens=2 ** 28)), (UNSUPPORTED, dict(N=BIG))],
    "gemm_adapters": [(INVALID, dict(kind=5)), (INVALID, dict(rows=-1)), (INVALID, dict(rank=-1)), (INVALID, dict(adapters=-1)), (INVALID, dict(layoutB=3)),
                      (INVALID, dict(layout_down=3)), (INVALID, dict(layout_up=-1)), (INVALID, dict(ld_down=47)), (INVALID, dict(ld_up=7)), (INVALID, dict(lda=47)),
                      (INVALID, dict(stride_up=-1)), (INVALID, dict(rows=1, adapter_of=None)), (INVALID, dict(rows=1, down=None)), (INVALID, dict(rows=1, up=None)),
                      (INVALID, dict(rows=1, A=None)), (INVALID, dict(rows=1, B=None)), (INVALID, dict(rows=1, C=None)), (UNSUPPORTED, dict(rank=257)),
                      (UNSUPPORTED, dict(rows=BIG)), (UNSUPPORTED, dict(stride_down=2 ** 61))],
}


@pytest.mark.parametrize("name", CALLS)
def test_refusals(name):
    fn, plain = getattr(g, name), CALLS[name]
    assert fn(*plain.values(), check=False) == 0
    for status, change in REFUSED[name]:
        assert set(change) <= set(plain)
        assert fn(*{**plain, **change}.values(), check=False) == status, change
        with pytest.raises(g.GemmError) as e:
            fn(*{**plain, **change}.values())
        assert e.value.status == status


def test_plan_refusals():
    def call(**change):
        return g.gemm_route_plan(*{**PLAN, **change}.values(), check=False)
    for change in (dict(tokens=-1), dict(top_k=0), dict(experts=0), dict(offsets=None), dict(tokens=1, indices=None), dict(tokens=1, token_of=None),
                   dict(tokens=1, slot_of=None)):
        assert call(**change) == INVALID, change
    for change in (dict(experts=1025), dict(tokens=2 ** 28, top_k=1), dict(tokens=2 ** 20, top_k=2 ** 20)):
        assert call(**change) == UNSUPPORTED, change


def test_every_declared_call_is_exported_and_bound():
    text = open(os.path.join(ROOT, "include", "gemm_routed.h")).read()
    names = set(re.findall(r"\b(gemm_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert names == set(routed.SIGNATURES)
    lib = g.load_library()
    for name in names:
        assert isinstance(getattr(lib, name), ctypes._CFuncPtr)
        assert name in g.__all__ and callable(getattr(g, name))
    for constant, value in re.findall(r"\bGEMM_([A-Z0-9_]+)\s*(?:=)?\s*(\d+)\b", re.sub(r"/\*.*?\*/", "", text, flags=re.S)):
        assert getattr(g, constant) == int(value), constant


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "gemm_routed.h"\nint kinds(void) { return GEMM_KIND_BF16BF16 + GEMM_SCORE_SIGMOID + GEMM_ELEM_BF16 + GEMM_ADAPTERS_MAX_RANK; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-fsyntax-only", "-I" + os.path.join(ROOT, "include"), str(src)], check=True)


@pytest.mark.parametrize("name", list(CALLS) + ["gemm_route_plan"])
def test_plain_and_general_calls_agree(name):
    """The calls through the C extension and the ctypes functions behind it (any keyword argument goes there)."""
    import inspect
    fn, plain = getattr(g, name), CALLS.get(name, {**PLAN, "tokens": -1})   # (a plan of no entries still writes its offsets)
    status = 0 if name in CALLS else INVALID
    assert list(inspect.signature(fn).parameters) == list(plain) + ["stream", "check"]
    args = tuple(plain.values())
    for stream in (0, None):
        assert fn(*args, stream, False) == status
        if status == 0:
            assert fn(*args) == fn(*args, stream) == fn(*args, stream, True) == 0
    for at in range(0 if status == 0 else 1, len(args)):   # (the plan's first argument is what has it refused)
        for value in ("x", 1.5j, 2 ** 70):
            bad = args[:at] + (value,) + args[at + 1:]
            errors = []
            for call in (lambda: fn(*bad, 0, False), lambda: fn(*bad, check=False, stream=0)):
                try:
                    errors.append(call())
                except Exception as e:
                    errors.append(type(e))
            assert errors[0] == errors[1], (name, at, value, errors)
    with pytest.raises(TypeError):
        fn(*args[:-1])
    with pytest.raises(TypeError):
        fn(*args, 0, True, 1)
