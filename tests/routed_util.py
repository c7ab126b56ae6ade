"""Plain 64-bit implementations of what include/gemm_routed.h describes (numpy, host only), and helpers of its GPU tests."""
import numpy as np

import gemm_inputs as gi

U32 = 2.0 ** -24                                   # half a unit in the last place of binary32, relative
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
SMALLEST = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}   # half the smallest number

KINDS = {"f32": ("f32", "f32"), "f16f32": ("f16", "f32"), "f16f16": ("f16", "f16"), "bf16f32": ("bf16", "f32"), "bf16bf16": ("bf16", "bf16")}


def kind_of(name):
    import paper_2003_06324_amd as g
    return {"f32": g.KIND_F32, "f16f32": g.KIND_F16F32, "f16f16": g.KIND_F16F16, "bf16f32": g.KIND_BF16F32, "bf16bf16": g.KIND_BF16BF16}[name]


def elem_of(name):
    import paper_2003_06324_amd as g
    return {"f32": g.ELEM_F32, "f16": g.ELEM_F16, "bf16": g.ELEM_BF16}[name]


def torch_type(elem):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[elem]


def rounded(x, elem):
    """float64 values rounded once, to nearest even, to the element type (as float64)."""
    x = np.asarray(x, dtype=np.float64)
    if elem == "f32":
        return x.astype(np.float32).astype(np.float64)
    if elem == "f16":
        with np.errstate(over="ignore"):
            return x.astype(np.float16).astype(np.float64)
    m, e = np.frexp(x)                      # 8 significant bits
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


def values(rng, shape, elem, dist="normal", scale=1.0):
    """Host values of the element type, as float64."""
    x = rng.standard_normal(shape) * scale if dist == "normal" else rng.integers(-3, 4, size=shape).astype(np.float64)
    return rounded(x, elem)


def put(x, elem, ld=0, offset=0, layout=gi.ROW_MAJOR, count=None):
    """The matrix (or, with a leading axis, matrices one after the other) on the device: (flat tensor, address, ld, stride).
    Rows are padded to ld, and `offset` elements lie before them; padding holds NaN."""
    import torch
    x = np.asarray(x, dtype=np.float64)
    mats = x if x.ndim == 3 else x[None]
    if layout == gi.COL_MAJOR:
        mats = mats.transpose(0, 2, 1)
    n, rows, cols = mats.shape
    ld = ld or cols
    buf = np.full(offset + n * rows * ld, np.nan)
    buf[offset:].reshape(n, rows, ld)[:, :, :cols] = mats
    t = torch.from_numpy(buf).to(torch_type(elem)).cuda()
    return t, t.data_ptr() + offset * t.element_size(), ld, rows * ld


def room(rows, cols, elem, ld=0, offset=0, guard=64):
    """Device memory for a rows x cols result, filled with a value that no result has: (tensor, address, ld)."""
    import torch
    ld = ld or cols
    t = torch.full((offset + rows * ld + guard,), 12288.0, dtype=torch_type(elem), device="cuda")
    return t, t.data_ptr() + offset * t.element_size(), ld


def back(t, rows, cols, ld, offset=0, guard=64):
    """The result as float64, and whether everything around it is untouched."""
    h = t.float().cpu().numpy().astype(np.float64)
    body = h[offset:offset + rows * ld].reshape(rows, ld)
    clean = (h[:offset] == 12288.0).all() and (h[offset + rows * ld:] == 12288.0).all() and (body[:, cols:] == 12288.0).all()
    return body[:, :cols].copy(), bool(clean)


# ---------------------------------------------------------------------------- routing
def scores(logits, softmax):
    l = np.asarray(logits, dtype=np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if not softmax:
            return 1.0 / (1.0 + np.exp(-l))
        m = l.max(axis=1, keepdims=True)
        e = np.exp(l - np.where(np.isneginf(m), 0.0, m))
        z = e.sum(axis=1, keepdims=True)
        return np.where(z == 0.0, 0.0, e / np.where(z == 0.0, 1.0, z))


def route(logits, softmax, top_k, bias=None, groups=1, top_groups=1, group_top=1, renormalise=True, scale=1.0):
    s = scores(logits, softmax)
    c = s if bias is None else s + np.asarray(bias, dtype=np.float64)
    T, E = c.shape
    weights, indices = np.zeros((T, top_k)), np.zeros((T, top_k), dtype=np.int64)
    size = E // groups
    for t in range(T):
        allowed = list(range(E))
        if groups > 1:
            best = [sum(sorted(c[t, g * size:(g + 1) * size], reverse=True)[:group_top]) for g in range(groups)]
            chosen = sorted(range(groups), key=lambda g: (-best[g], g))[:top_groups]
            allowed = [e for e in allowed if e // size in chosen]
        order = sorted(allowed, key=lambda e: (np.inf if np.isnan(c[t, e]) else -c[t, e] if not np.isneginf(c[t, e]) else 1e300, e))
        indices[t] = order[:top_k]
        w = s[t, indices[t]]
        if renormalise:
            z = w.sum()
            w = np.zeros(top_k) if z == 0.0 else w / z
        weights[t] = w * scale
    return weights, indices


def route_backward(logits, softmax, indices, d_weights, renormalise=True, scale=1.0):
    s = scores(logits, softmax)
    T, E = s.shape
    out = np.zeros((T, E))
    for t in range(T):
        at, dw = indices[t], np.asarray(d_weights[t], dtype=np.float64)
        ds = np.zeros(E)
        if renormalise:
            z = s[t, at].sum()
            ds[at] = 0.0 if z == 0.0 else scale / z * (dw - (dw * s[t, at]).sum() / z)
        else:
            ds[at] = scale * dw
        out[t] = s[t] * (ds - (ds * s[t]).sum()) if softmax else ds * s[t] * (1.0 - s[t])
    return out


def plan(indices, experts):
    T, k = indices.shape
    offsets, token_of, slot_of = [0], np.full(T * k, -1, dtype=np.int64), np.full((T, k), -1, dtype=np.int64)
    slot = 0
    for e in range(experts):
        for t, j in zip(*np.nonzero(indices == e)):
            token_of[slot], slot_of[t, j] = t, slot
            slot += 1
        offsets.append(slot)
    return np.array(offsets), token_of, slot_of


# ---------------------------------------------------------------------------- products
def rows_of(A, row_map, i):
    r = i if row_map is None else row_map[i]
    ok = (r >= 0) & (r < len(A))
    return np.where(ok[:, None], A[np.where(ok, r, 0)], 0.0) if len(A) else np.zeros((len(i), A.shape[1]))


def grouped(A, offsets, rows, row_map, B):
    """(result, which rows belong to a group, sum of the products' magnitudes)"""
    out, mag, there = np.zeros((rows, B.shape[2])), np.zeros((rows, B.shape[2])), np.zeros(rows, dtype=bool)
    for e in range(len(B)):
        i = np.arange(max(0, offsets[e]), min(rows, offsets[e + 1]))
        a = rows_of(A, row_map, i)
        out[i], mag[i], there[i] = a @ B[e], np.abs(a) @ np.abs(B[e]), True
    return out, there, mag


def wgrad(A, offsets, rows, row_map, D):
    n = len(offsets) - 1
    out, mag = np.zeros((n, A.shape[1], D.shape[1])), np.zeros((n, A.shape[1], D.shape[1]))
    for e in range(n):
        i = np.arange(max(0, offsets[e]), min(rows, offsets[e + 1]))
        a = rows_of(A, row_map, i)
        out[e], mag[e] = a.T @ D[i], np.abs(a).T @ np.abs(D[i])
    return out, mag


def combine(Y, slot_of, weights):
    T, k = slot_of.shape
    out, mag = np.zeros((T, Y.shape[1])), np.zeros((T, Y.shape[1]))
    for t in range(T):
        for j in range(k):
            if 0 <= slot_of[t, j] < len(Y):
                w = 1.0 if weights is None else float(weights[t, j])
                out[t] += w * Y[slot_of[t, j]]
                mag[t] += abs(w) * np.abs(Y[slot_of[t, j]])
    return out, mag


def adapters(A, B, adapter_of, scales, down, up):
    """(result, magnitudes of the product, of the additions)"""
    out, mag, add = A @ B, np.abs(A) @ np.abs(B), np.zeros((len(A), B.shape[1]))
    for a in range(len(down)):
        i = np.nonzero(adapter_of == a)[0]
        s = 1.0 if scales is None else float(scales[a])
        out[i] += s * (A[i] @ down[a]) @ up[a]
        add[i] = abs(s) * (np.abs(A[i]) @ np.abs(down[a])) @ np.abs(up[a])
    return out, mag, add


def bound(mag, terms, elem, ref):
    """What a sum of `terms` products may differ by from the exact one: every product and addition in binary32 (the standard bound, terms
    times the unit roundoff times the magnitudes), and the rounding of the result."""
    return 1.01 * terms * U32 * mag + HALF_ULP[elem] * (np.abs(ref) + terms * U32 * mag) + SMALLEST[elem]
