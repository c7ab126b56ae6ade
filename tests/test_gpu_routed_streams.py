"""Routed products on streams other than the default one, under graph capture, in a row as a layer of experts runs them, and with
operands whose offsets pass 32 bits."""
import numpy as np
import pytest

import gemm_inputs as gi
import routed_util as ru

pytestmark = pytest.mark.gpu


class Layer:
    """A layer of experts with an adapted projection in front, in bfloat16, on buffers of its own."""

    def __init__(self, seed, T=150, E=24, k=4, D=136, F=72, n=5, r=8):
        import torch
        g = torch.Generator().manual_seed(seed)

        def some(*shape, scale=1.0):
            return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16).cuda()
        self.T, self.E, self.k, self.D, self.F, self.n, self.r = T, E, k, D, F, n, r
        self.x, self.w, self.down, self.up = some(T, D), some(D, D, scale=D ** -0.5), some(n, r, D, scale=D ** -0.5), some(n, D, r, scale=0.3)
        self.of = torch.randint(-1, n, (T,), generator=g).int().cuda()
        self.router, self.w1, self.w2 = some(E, D, scale=D ** -0.5), some(E, F, D, scale=D ** -0.5), some(E, D, F, scale=F ** -0.5)
        f32, i32, bf = torch.float32, torch.int32, torch.bfloat16

        def room(*shape, type=bf):
            return torch.zeros(shape, dtype=type, device="cuda")
        self.h, self.logits, self.weights, self.indices = room(T, D), room(T, E, type=f32), room(T, k, type=f32), room(T, k, type=i32)
        self.offsets, self.token_of, self.slot_of = room(E + 1, type=i32), room(T * k, type=i32), room(T, k, type=i32)
        self.mid, self.act, self.y, self.out = room(T * k, F), room(T * k, F), room(T * k, D), room(T, D, type=f32)

    def run(self, stream):
        import paper_2003_06324_amd as g
        import torch
        T, E, k, D, F = self.T, self.E, self.k, self.D, self.F
        g.gemm_adapters(g.KIND_BF16BF16, T, D, D, self.x, 0, self.w, 1, 0, self.n, self.r, self.of, None, self.down, 1, 0, 0, self.up, 1, 0, 0, self.h, 0, stream)
        g.gemm_bf16f32(T, E, D, self.h, 0, 0, self.router, 1, 0, self.logits, 0, 0, stream)
        g.gemm_route(g.ELEM_F32, T, E, self.logits, 0, None, g.SCORE_SOFTMAX, 1, 1, 1, k, 1, 1.0, self.weights, self.indices, stream)
        g.gemm_route_plan(T, k, E, self.indices, self.offsets, self.token_of, self.slot_of, stream)
        g.gemm_grouped(g.KIND_BF16BF16, E, self.offsets, T * k, F, D, self.h, T, 0, self.token_of, self.w1, 1, 0, 0, self.mid, 0, stream)
        torch.clamp(self.mid, min=0, out=self.act)
        g.gemm_grouped(g.KIND_BF16BF16, E, self.offsets, T * k, D, F, self.act, T * k, 0, None, self.w2, 1, 0, 0, self.y, 0, stream)
        g.gemm_combine(g.KIND_BF16F32, T, k, D, self.y, T * k, 0, self.slot_of, self.weights, self.out, 0, stream)
        return self.out

    def expected(self):
        """Layer by layer from what the library has made of the one before: the error of every step is its own."""
        f = {k: v.float().cpu().numpy().astype(np.float64) for k, v in self.__dict__.items() if hasattr(v, "cpu")}
        of, idx = f["of"].astype(int), f["indices"].astype(int)
        h, mag, add = ru.adapters(f["x"], f["w"].T, of, None, f["down"].transpose(0, 2, 1), f["up"].transpose(0, 2, 1))
        err = 1.01 * ru.U32 * (self.D + 1) * mag + 2.0 ** -20 * add
        assert (np.abs(f["h"] - h) <= err + ru.HALF_ULP["bf16"] * (np.abs(h) + err)).all()
        w, _ = ru.route(f["logits"], True, self.k)
        assert (np.abs(f["weights"] - w) <= 1e-5).all()
        offsets, token_of, slot_of = ru.plan(idx, self.E)
        assert np.array_equal(f["offsets"], offsets) and np.array_equal(f["slot_of"], slot_of)
        mid, there, mag = ru.grouped(f["h"], offsets, self.T * self.k, token_of, f["w1"].transpose(0, 2, 1))
        assert (np.abs(f["mid"] - mid) <= ru.bound(mag, self.D, "bf16", mid)).all()
        y, there, mag = ru.grouped(f["act"], offsets, self.T * self.k, None, f["w2"].transpose(0, 2, 1))
        assert (np.abs(f["y"] - y) <= ru.bound(mag, self.F, "bf16", y)).all()
        out, mag = ru.combine(f["y"], slot_of, f["weights"])
        assert (np.abs(f["out"] - out) <= ru.bound(mag, self.k, "f32", out)).all()


def test_a_layer_of_experts():
    import torch
    layer = Layer(1)
    layer.run(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    layer.expected()


def test_two_streams_do_not_meet():
    """Both use workspaces of their own: results are those of each alone."""
    import torch
    layers = [Layer(2), Layer(3, T=700, E=40), Layer(4, T=9, D=256)]
    alone = []
    for layer in layers:
        alone.append(layer.run(torch.cuda.current_stream().cuda_stream).clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(5):
        for layer in layers:
            layer.out.fill_(7.0)
        torch.cuda.synchronize()
        for layer, s in zip(layers, streams):
            with torch.cuda.stream(s):
                layer.run(s.cuda_stream)
        torch.cuda.synchronize()
        for layer, want in zip(layers, alone):
            assert torch.equal(layer.out, want)


def test_capture_and_replays():
    import torch
    import paper_2003_06324_amd as g
    layer = Layer(5)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        layer.run(s.cuda_stream)      # the workspace, outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        layer.run(s.cuda_stream)
    for seed in range(4):
        layer.x.copy_(torch.randn(layer.x.shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16))
        layer.out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = layer.out.clone()
        layer.run(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(got, layer.out)
        layer.expected()
    # on a stream whose workspace would have to grow the call is refused, and the capture goes on
    fresh = torch.cuda.Stream()
    status = []
    with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=fresh):
        status.append(g.gemm_adapters(g.KIND_BF16BF16, layer.T, layer.D, layer.D, layer.x, 0, layer.w, 1, 0, layer.n, layer.r, layer.of, None, layer.down, 1, 0, 0,
                                      layer.up, 1, 0, 0, layer.h, 0, fresh.cuda_stream, check=False))
        layer.out.fill_(1.0)
    assert status == [-4]


def test_results_are_the_same_every_time():
    """No result depends on the order in which workgroups run."""
    import torch
    layer = Layer(6, T=900, E=16, D=320, F=264)
    stream = torch.cuda.current_stream().cuda_stream
    want = layer.run(stream).clone()
    for _ in range(10):
        assert torch.equal(layer.run(stream), want)


@pytest.mark.parametrize("mapped", [False, True])
def test_offsets_beyond_32_bits(mapped):
    """Rows and matrices further apart than 32-bit offsets reach: the first, some in the middle and the last ones."""
    import torch
    import paper_2003_06324_amd as g
    stream = torch.cuda.current_stream().cuda_stream
    rows, ld, K, N, G = 60000, 40008, 72, 40, 3
    look = torch.tensor([0, 1, 777, 30000, 53690, 53700, rows - 2, rows - 1], device="cuda")
    A = torch.empty(rows * ld, dtype=torch.float16, device="cuda").view(rows, ld)      # 4.8 GB: element 2^31 lies in row 53676
    A[:, :K] = torch.randint(-3, 4, (rows, K), device="cuda").half()
    stride = (1 << 31) + 8
    B = torch.empty(2 * stride + K * N, dtype=torch.float16, device="cuda")
    mats = torch.randint(-3, 4, (G, K, N), device="cuda").half()
    for e in range(G):
        B[e * stride:e * stride + K * N] = mats[e].flatten()
    C = torch.empty(rows * ld, dtype=torch.float32, device="cuda").view(rows, ld)      # 9.6 GB
    offsets = torch.tensor([0, 20000, 53695, rows], dtype=torch.int32, device="cuda")
    perm = torch.randperm(rows, device="cuda").int() if mapped else None
    g.gemm_grouped(g.KIND_F16F32, G, offsets, rows, N, K, A, rows, ld, perm, B, gi.ROW_MAJOR, 0, stride, C, ld, stream)
    group = (look >= 20000).long() + (look >= 53695).long()
    src = A[:, :K][perm[look].long()] if mapped else A[look, :K]
    want = (src.double().unsqueeze(1) @ mats.double()[group]).squeeze(1)
    assert torch.equal(C[look, :N].double(), want)
    # the gradient: D's and A's rows as far apart
    D = C[:, :N]
    D.copy_(torch.randint(-2, 3, (rows, N), device="cuda").float())
    A32 = torch.empty(rows * 40000, dtype=torch.float32, device="cuda").view(rows, 40000)
    A32[:, :K] = A[:, :K].float()
    out = torch.zeros(G, K, N, device="cuda")
    g.gemm_grouped_wgrad(g.KIND_F32, G, offsets, rows, K, N, A32, rows, 40000, perm, C, ld, out, gi.ROW_MAJOR, 0, 0, stream)
    a = A32[:, :K].double()
    a = a[perm.long()] if mapped else a
    for e in range(G):
        lo, hi = offsets[e].item(), offsets[e + 1].item()
        assert torch.equal(out[e].double(), a[lo:hi].t().contiguous() @ D[lo:hi].double().contiguous())
    # sums of rows
    slots = torch.stack([look, look.flip(0)], 1).int().contiguous()
    total = torch.zeros(len(look), N, device="cuda")
    g.gemm_combine(g.KIND_F32, len(look), 2, N, C, rows, ld, slots, None, total, 0, stream)
    assert torch.equal(total, D[look] + D[look.flip(0)])


def test_adapters_with_offsets_beyond_32_bits():
    import torch
    import paper_2003_06324_amd as g
    stream = torch.cuda.current_stream().cuda_stream
    rows, ld, K, N, r = 60000, 40008, 72, 40, 8
    look = torch.tensor([0, 1, 777, 30000, 53690, 53700, rows - 2, rows - 1], device="cuda")
    A = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    A[:, :K] = torch.randint(-3, 4, (rows, K), device="cuda").to(torch.bfloat16)
    B = torch.randint(-3, 4, (K, N), device="cuda").to(torch.bfloat16)
    stride = (1 << 31) + 8
    up, down = torch.empty(stride + N * r, dtype=torch.bfloat16, device="cuda"), torch.randint(-1, 2, (2, r, K), device="cuda").to(torch.bfloat16)
    ups = torch.randint(-1, 2, (2, N, r), device="cuda").to(torch.bfloat16)
    up[:N * r], up[stride:stride + N * r] = ups[0].flatten(), ups[1].flatten()
    of = (torch.arange(rows, device="cuda") // 100 % 3 - 1).int()
    C = torch.empty(rows * ld, dtype=torch.float32, device="cuda").view(rows, ld)
    g.gemm_adapters(g.KIND_BF16F32, rows, N, K, A, ld, B, gi.ROW_MAJOR, 0, 2, r, of, None, down, gi.COL_MAJOR, 0, 0, up, gi.COL_MAJOR, 0, stride, C, ld, stream)
    want = A[look, :K].double() @ B.double()
    for i, row in enumerate(look.tolist()):
        a = of[row].item()
        if a >= 0:
            want[i] += A[row, :K].double() @ down[a].double().t().contiguous() @ ups[a].double().t().contiguous()
    assert torch.equal(C[look, :N].double(), want)
