"""Python binding of include/gemm_routed.h: products whose rows choose their right operand (experts, adapters).

Argument marshalling only, as in gemm.py: device addresses (ints) or objects with ``data_ptr()``; names and argument order follow
the C header, which says what each call computes.
"""
import ctypes

from .gemm import _binding, _check, _ptr, load_library as _load_library

ELEM_F32, ELEM_F16, ELEM_BF16 = 0, 1, 2
KIND_BF16BF16 = 4
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
ROUTE_MAX_EXPERTS, ROUTE_MAX_GROUPS, ROUTE_MAX_TOP_K = 1024, 64, 64
ADAPTERS_MAX_RANK = 256

_P, _I, _L, _F = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float
SIGNATURES = {
    "gemm_route": [_I, _L, _L, _P, _L, _P, _I, _L, _L, _I, _L, _I, _F, _P, _P, _P],
    "gemm_route_backward": [_I, _L, _L, _P, _L, _I, _L, _I, _F, _P, _P, _P, _L, _P],
    "gemm_route_plan": [_L, _L, _L, _P, _P, _P, _P, _P],
    "gemm_grouped": [_I, _L, _P, _L, _L, _L, _P, _L, _L, _P, _P, _I, _L, _L, _P, _L, _P],
    "gemm_grouped_wgrad": [_I, _L, _P, _L, _L, _L, _P, _L, _L, _P, _P, _L, _P, _I, _L, _L, _P],
    "gemm_combine": [_I, _L, _L, _L, _P, _L, _L, _P, _P, _P, _L, _P],
    "gemm_combine_backward": [_I, _L, _L, _L, _P, _L, _P, _L, _L, _P, _P, _P, _L, _P, _P],
    "gemm_adapters": [_I, _L, _L, _L, _P, _L, _P, _I, _L, _L, _L, _P, _P, _P, _I, _L, _L, _P, _I, _L, _L, _P, _L, _P],
}
_bound = None
_plain = hasattr(_binding, "routed_bind")   # (an extension that was built before these calls leaves them to ctypes)


def _lib():
    global _bound
    if _bound is None:
        lib = _load_library()
        for name, signature in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.argtypes = signature
            fn.restype = ctypes.c_int
        _bound = lib
        if _plain:
            _binding.routed_bind(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in SIGNATURES))
    return _bound


def gemm_route(elem, tokens, experts, logits, ld, bias, score, groups, top_groups, group_top, top_k, renormalise, scale,
               weights, indices, stream=None, check=True):
    """Scores of a router, the top_k experts of every token and their weights."""
    rc = _lib().gemm_route(elem, tokens, experts, _ptr(logits), ld, _ptr(bias), score, groups, top_groups, group_top, top_k,
                           renormalise, scale, _ptr(weights), _ptr(indices), stream or None)
    return _check(rc) if check else rc


def gemm_route_backward(elem, tokens, experts, logits, ld, score, top_k, renormalise, scale, indices, d_weights, d_logits, ld_d,
                        stream=None, check=True):
    """Gradient of gemm_route's weights for the logits."""
    rc = _lib().gemm_route_backward(elem, tokens, experts, _ptr(logits), ld, score, top_k, renormalise, scale, _ptr(indices),
                                    _ptr(d_weights), _ptr(d_logits), ld_d, stream or None)
    return _check(rc) if check else rc


def gemm_route_plan(tokens, top_k, experts, indices, offsets, token_of, slot_of, stream=None, check=True):
    """The tokens' entries sorted by expert: offsets of the experts' slots, a slot's token, an entry's slot."""
    rc = _lib().gemm_route_plan(tokens, top_k, experts, _ptr(indices), _ptr(offsets), _ptr(token_of), _ptr(slot_of), stream or None)
    return _check(rc) if check else rc


def gemm_grouped(kind, groups, offsets, rows, N, K, A, a_rows, lda, row_map, B, layoutB, ldb, strideB, C, ldc, stream=None, check=True):
    """C(i,:) = A(row_map[i],:) * B_e for the rows i of every group e."""
    rc = _lib().gemm_grouped(kind, groups, _ptr(offsets), rows, N, K, _ptr(A), a_rows, lda, _ptr(row_map), _ptr(B), layoutB, ldb, strideB,
                             _ptr(C), ldc, stream or None)
    return _check(rc) if check else rc


def gemm_grouped_wgrad(kind, groups, offsets, rows, M, N, A, a_rows, lda, row_map, D, ldd, C, layoutC, ldc, strideC, stream=None, check=True):
    """C_e = sum over the rows i of group e of A(row_map[i],:)^T * D(i,:)."""
    rc = _lib().gemm_grouped_wgrad(kind, groups, _ptr(offsets), rows, M, N, _ptr(A), a_rows, lda, _ptr(row_map), _ptr(D), ldd, _ptr(C),
                                   layoutC, ldc, strideC, stream or None)
    return _check(rc) if check else rc


def gemm_combine(kind, tokens, top_k, N, Y, y_rows, ldy, slot_of, weights, out, ldo, stream=None, check=True):
    """out(t,:) = sum over j of weights[t][j] * Y(slot_of[t][j],:)."""
    rc = _lib().gemm_combine(kind, tokens, top_k, N, _ptr(Y), y_rows, ldy, _ptr(slot_of), _ptr(weights), _ptr(out), ldo, stream or None)
    return _check(rc) if check else rc


def gemm_combine_backward(elem, tokens, top_k, N, d_out, ldo, Y, y_rows, ldy, slot_of, weights, dY, lddy, d_weights, stream=None, check=True):
    """Gradients of gemm_combine for Y and the weights."""
    rc = _lib().gemm_combine_backward(elem, tokens, top_k, N, _ptr(d_out), ldo, _ptr(Y), y_rows, ldy, _ptr(slot_of), _ptr(weights), _ptr(dY),
                                      lddy, _ptr(d_weights), stream or None)
    return _check(rc) if check else rc


def gemm_adapters(kind, rows, N, K, A, lda, B, layoutB, ldb, adapters, rank, adapter_of, scales, down, layout_down, ld_down, stride_down,
                  up, layout_up, ld_up, stride_up, C, ldc, stream=None, check=True):
    """C(i,:) = A(i,:) * B + scales[a] * (A(i,:) * down_a) * up_a with a = adapter_of[i]."""
    rc = _lib().gemm_adapters(kind, rows, N, K, _ptr(A), lda, _ptr(B), layoutB, ldb, adapters, rank, _ptr(adapter_of), _ptr(scales), _ptr(down),
                              layout_down, ld_down, stride_down, _ptr(up), layout_up, ld_up, stride_up, _ptr(C), ldc, stream or None)
    return _check(rc) if check else rc


if _plain:
    for _i, _name in enumerate(SIGNATURES):
        _binding.routed_general(_i, globals()[_name])   # before the library is loaded, and for arguments that are not plain
    from ._binding import (gemm_adapters, gemm_combine, gemm_combine_backward, gemm_grouped, gemm_grouped_wgrad, gemm_route,  # noqa: F811
                           gemm_route_backward, gemm_route_plan)
