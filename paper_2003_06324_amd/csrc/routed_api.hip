// C entries of the grouped products and the adapters: checks, forms, launches.
#include "routed_launch.h"

#include <algorithm>

using namespace gemm_gfx950;

namespace gemm_gfx950 {
ROUTED_FORMS(extern, float, float)
ROUTED_FORMS(extern, _Float16, float)
ROUTED_FORMS(extern, _Float16, _Float16)
ROUTED_FORMS(extern, __bf16, float)
ROUTED_FORMS(extern, __bf16, __bf16)
}  // namespace gemm_gfx950

namespace {

int64_t elem_size(int kind) { return kind == GEMM_KIND_F32 ? 4 : 2; }

// Whether direct loads serve a matrix: rows begin on 4-byte words, and offsets in a tile of 256 rows (or 64 k-rows) fit 32 bits.
bool direct(const void *p, int64_t ld, int64_t stride, int64_t esz)
{
    return (((uintptr_t)p | (uintptr_t)(ld * esz) | (uintptr_t)(stride * esz)) & 3) == 0 && 256 * ld * esz < (1LL << 31);
}
// whether gathered rows' offsets fit 32 bits (with what the loader adds to them)
bool gathers(int64_t rows, int64_t ld, int64_t esz) { return ld * esz < (1LL << 31) && rows * (ld * esz) < (1LL << 31) - (1 << 16); }

template <typename F> int by_kind(int kind, const F &f)
{
    switch (kind) {
    case GEMM_KIND_F32: return f((float *)nullptr, (float *)nullptr);
    case GEMM_KIND_F16F32: return f((_Float16 *)nullptr, (float *)nullptr);
    case GEMM_KIND_F16F16: return f((_Float16 *)nullptr, (_Float16 *)nullptr);
    case GEMM_KIND_BF16F32: return f((__bf16 *)nullptr, (float *)nullptr);
    default: return f((__bf16 *)nullptr, (__bf16 *)nullptr);
    }
}

}  // namespace

extern "C" {

int gemm_grouped(int kind, int64_t groups, const int32_t *offsets, int64_t rows, int64_t N, int64_t K,
                 const void *A, int64_t a_rows, int64_t lda, const int32_t *row_map,
                 const void *B, int layoutB, int64_t ldb, int64_t strideB, void *C, int64_t ldc, void *hip_stream)
{
    if (!valid_kind(kind) || groups < 0 || rows < 0 || N < 0 || K < 0 || a_rows < 0 || lda < 0 || ldb < 0 || ldc < 0 || strideB < 0 || !valid_layout(layoutB))
        return GEMM_ERR_INVALID_ARG;
    if (!fill_ld(GEMM_ROW_MAJOR, lda, a_rows, K) || !fill_ld(layoutB, ldb, K, N) || !fill_ld(GEMM_ROW_MAJOR, ldc, rows, N)) return GEMM_ERR_INVALID_ARG;
    if (groups > kMaxExtent || rows > kMaxExtent || N > kMaxExtent || K > kMaxExtent || a_rows > kMaxExtent || too_far(a_rows, lda) ||
        too_far(layoutB == GEMM_ROW_MAJOR ? K : N, ldb) || too_far(rows, ldc))
        return GEMM_ERR_UNSUPPORTED;
    if (strideB == 0) strideB = layoutB == GEMM_ROW_MAJOR ? K * ldb : N * ldb;
    if (too_far(groups, strideB)) return GEMM_ERR_UNSUPPORTED;
    if (groups == 0 || rows == 0 || N == 0) return GEMM_OK;
    if (offsets == nullptr || C == nullptr || (K > 0 && (B == nullptr || (a_rows > 0 && A == nullptr)))) return GEMM_ERR_INVALID_ARG;
    const int64_t esz = elem_size(kind);
    int form = GROUPED_ANY;
    int64_t BM = 64, BN = 64;
    if (direct(A, lda, 0, esz) && direct(B, ldb, strideB, esz) && (row_map == nullptr || gathers(a_rows, lda, esz))) {
        const int64_t each = ceil_div(rows, groups);
        form = each <= 32 ? GROUPED_32x128 : (each <= 64 ? GROUPED_64x128 : GROUPED_128x128);
        BM = each <= 32 ? 32 : (each <= 64 ? 64 : 128);
        BN = 128;
    }
    const int64_t tiles_n = ceil_div(N, BN), grid = grouped_grid(groups, rows, BM, tiles_n);
    if (grid > (1LL << 24) - 1) return GEMM_ERR_UNSUPPORTED;
    const GroupedArgs a = {A, B, C, offsets, row_map, lda, ldb, ldc, strideB, (int)groups, (int)rows, (int)a_rows, (int)N, (int)K, (int)tiles_n};
    return by_kind(kind, [&](auto *t, auto *tc) {
        return launch_grouped<std::remove_pointer_t<decltype(t)>, std::remove_pointer_t<decltype(tc)>>(form, layoutB == GEMM_COL_MAJOR, dim3((unsigned)grid),
                                                                                                       (hipStream_t)hip_stream, a);
    });
}

int gemm_grouped_wgrad(int kind, int64_t groups, const int32_t *offsets, int64_t rows, int64_t M, int64_t N,
                       const void *A, int64_t a_rows, int64_t lda, const int32_t *row_map,
                       const void *D, int64_t ldd, void *C, int layoutC, int64_t ldc, int64_t strideC, void *hip_stream)
{
    if (!valid_kind(kind) || groups < 0 || rows < 0 || M < 0 || N < 0 || a_rows < 0 || lda < 0 || ldd < 0 || ldc < 0 || strideC < 0 || !valid_layout(layoutC))
        return GEMM_ERR_INVALID_ARG;
    if (!fill_ld(GEMM_ROW_MAJOR, lda, a_rows, M) || !fill_ld(GEMM_ROW_MAJOR, ldd, rows, N) || !fill_ld(layoutC, ldc, M, N)) return GEMM_ERR_INVALID_ARG;
    if (groups > kMaxExtent || rows > kMaxExtent || N > kMaxExtent || M > kMaxExtent || a_rows > kMaxExtent || too_far(a_rows, lda) || too_far(rows, ldd) ||
        too_far(layoutC == GEMM_ROW_MAJOR ? M : N, ldc))
        return GEMM_ERR_UNSUPPORTED;
    if (strideC == 0) strideC = layoutC == GEMM_ROW_MAJOR ? M * ldc : N * ldc;
    if (groups > 1 && strideC < extent_of(layoutC, ldc, M, N)) return GEMM_ERR_INVALID_ARG;
    if (too_far(groups, strideC)) return GEMM_ERR_UNSUPPORTED;
    if (groups == 0 || M == 0 || N == 0) return GEMM_OK;
    if (offsets == nullptr || C == nullptr || (rows > 0 && (D == nullptr || (a_rows > 0 && A == nullptr)))) return GEMM_ERR_INVALID_ARG;
    const int64_t esz = elem_size(kind);
    // The kernels write rows of C: a column-major C is the row-major C^T = D^T A.
    WgradArgs a = {A, D, C, offsets, row_map, nullptr, lda, ldd, ldc, strideC, (int)groups, (int)rows, (int)a_rows, (int)rows, (int)M, (int)N, 0, 0};
    if (layoutC == GEMM_COL_MAJOR) {
        std::swap(a.X, a.Y);
        std::swap(a.map_x, a.map_y);
        std::swap(a.ldx, a.ldy);
        std::swap(a.x_rows, a.y_rows);
        std::swap(a.M, a.N);
    }
    const bool fast = direct(A, lda, 0, esz) && direct(D, ldd, 0, esz) && (row_map == nullptr || gathers(a_rows, lda, esz));
    const int64_t edge = fast ? 128 : 64;
    a.tiles_m = (int)ceil_div(a.M, edge);
    a.tiles_n = (int)ceil_div(a.N, edge);
    const int64_t per = (int64_t)a.tiles_m * a.tiles_n;
    if (per > (1LL << 24) || per * groups > (1LL << 24) - 8) return GEMM_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)(8 * ceil_div(per * groups, 8)));
    return by_kind(kind, [&](auto *t, auto *tc) {
        return launch_wgrad<std::remove_pointer_t<decltype(t)>, std::remove_pointer_t<decltype(tc)>>(fast ? WGRAD_128x128 : WGRAD_ANY, grid, (hipStream_t)hip_stream, a);
    });
}

int gemm_adapters(int kind, int64_t rows, int64_t N, int64_t K, const void *A, int64_t lda, const void *B, int layoutB, int64_t ldb,
                  int64_t adapters, int64_t rank, const int32_t *adapter_of, const float *scales,
                  const void *down, int layout_down, int64_t ld_down, int64_t stride_down,
                  const void *up, int layout_up, int64_t ld_up, int64_t stride_up, void *C, int64_t ldc, void *hip_stream)
{
    if (!valid_kind(kind) || rows < 0 || N < 0 || K < 0 || lda < 0 || ldb < 0 || ldc < 0 || adapters < 0 || rank < 0 || ld_down < 0 || ld_up < 0 ||
        stride_down < 0 || stride_up < 0 || !valid_layout(layoutB) || !valid_layout(layout_down) || !valid_layout(layout_up))
        return GEMM_ERR_INVALID_ARG;
    if (!fill_ld(GEMM_ROW_MAJOR, lda, rows, K) || !fill_ld(layoutB, ldb, K, N) || !fill_ld(GEMM_ROW_MAJOR, ldc, rows, N) ||
        !fill_ld(layout_down, ld_down, K, rank) || !fill_ld(layout_up, ld_up, rank, N))
        return GEMM_ERR_INVALID_ARG;
    if (rank > GEMM_ADAPTERS_MAX_RANK || rows > kMaxExtent || N > kMaxExtent || K > kMaxExtent || adapters > kMaxExtent || too_far(rows, lda) ||
        too_far(rows, ldc) || too_far(layoutB == GEMM_ROW_MAJOR ? K : N, ldb) || too_far(layout_down == GEMM_ROW_MAJOR ? K : rank, ld_down) ||
        too_far(layout_up == GEMM_ROW_MAJOR ? rank : N, ld_up))
        return GEMM_ERR_UNSUPPORTED;
    if (stride_down == 0) stride_down = (layout_down == GEMM_ROW_MAJOR ? K : rank) * ld_down;
    if (stride_up == 0) stride_up = (layout_up == GEMM_ROW_MAJOR ? rank : N) * ld_up;
    if (too_far(adapters, stride_down) || too_far(adapters, stride_up)) return GEMM_ERR_UNSUPPORTED;
    if (rows == 0 || N == 0) return GEMM_OK;
    const bool some = adapters > 0 && rank > 0 && K > 0;  // whether there is anything to add
    if (C == nullptr || (K > 0 && (A == nullptr || B == nullptr)) || (some && (adapter_of == nullptr || down == nullptr || up == nullptr)))
        return GEMM_ERR_INVALID_ARG;
    return no_throw([&]() -> int {
        const hipStream_t s = (hipStream_t)hip_stream;
        const int64_t esz = elem_size(kind);
        AdaptersArgs a = {A, B, down, up, C, adapter_of, scales, nullptr, lda, ldb, ldc, ld_down, stride_down, ld_up, stride_up, (int)rows, (int)N, (int)K,
                          some ? (int)adapters : 0, (int)rank, 0, 1, (int)K, layout_up == GEMM_COL_MAJOR, 0, 0, {}, {}};
        const bool fast = direct(A, lda, 0, esz) && direct(B, ldb, 0, esz);
        const int form = !fast ? ADAPTERS_ANY : (rows <= 256 ? ADAPTERS_32x128 : ADAPTERS_128x128);
        const int64_t BM = form == ADAPTERS_ANY ? 64 : (form == ADAPTERS_32x128 ? 32 : 128), BN = form == ADAPTERS_ANY ? 64 : 128;
        const int64_t tiles_m = ceil_div(rows, BM), tiles_n = ceil_div(N, BN);
        if (tiles_m > (1LL << 24) || tiles_n > (1LL << 24) || tiles_m * tiles_n > (1LL << 24) - 8) return GEMM_ERR_UNSUPPORTED;
        StreamScratch scratch;
        if (some) {
            const int64_t row_tiles = ceil_div(rows, DOWN_ROWS);
            const int64_t turns = std::min<int64_t>(adapters, row_tiles >= 64 ? 1 : DOWN_ROWS);
            a.t_pitch = (int)(ceil_div(rank, 32) * 32);
            // K in slices while there are fewer workgroups than CUs, of at least 256 k
            const int64_t slices = std::max<int64_t>(1, std::min<int64_t>(256 / std::max<int64_t>(1, row_tiles), ceil_div(K, 256)));
            a.t_k = (int)(ceil_div(ceil_div(K, slices), 64) * 64);
            a.t_splits = (int)ceil_div(K, a.t_k);
            const int rc = stream_scratch(s, (size_t)a.t_splits * rows * a.t_pitch * sizeof(float), scratch);
            if (rc != GEMM_OK) return rc;
            a.t = (float *)scratch.ptr;
            const dim3 grid((unsigned)(row_tiles * a.t_splits), (unsigned)turns);
            const bool kc = layout_down == GEMM_COL_MAJOR;
            const int sent = kind == GEMM_KIND_F32 ? launch_adapters_down<float>(kc, grid, s, a)
                             : elem_of_kind(kind) == GEMM_ELEM_F16 ? launch_adapters_down<_Float16>(kc, grid, s, a)
                                                                   : launch_adapters_down<__bf16>(kc, grid, s, a);
            if (sent != GEMM_OK) return sent;
        }
        a.tiles_m = (int)tiles_m;
        a.tiles_n = (int)tiles_n;
        a.by_band = divisor(GM * tiles_n);
        a.by_last_rows = divisor(tiles_m % GM > 0 ? tiles_m % GM : 1);
        const dim3 grid((unsigned)(8 * ceil_div(tiles_m * tiles_n, 8)));
        return by_kind(kind, [&](auto *t, auto *tc) {
            return launch_adapters<std::remove_pointer_t<decltype(t)>, std::remove_pointer_t<decltype(tc)>>(form, layoutB == GEMM_COL_MAJOR, grid, s, a);
        });
    });
}

}  // extern "C"
